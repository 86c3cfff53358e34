"""GPU parity of the experts' side of a layer (fb_quantize_rows, fb_expert_matmul, fb_combine) against plain
implementations in 64 bits.

Tolerances, all derived from the number formats.  bf16: half a step is 2^-8 of the value.  e4m3: 2^-4 of the value, or
2^-10 (half the step of its subnormal numbers) of the block's scale.  A 32-bit sum of n products differs from the exact one
by at most n * 2^-23 * sum |products| (a step of 2^-23 per addition covers rounding and truncation alike).  SwiGLU:
|d silu(g) / dg| <= 1.1, so an error dg, du of the sums becomes at most 1.1 |u| dg + |silu(g)| du, and 2^-19 of the value
covers exp (2 ulp and the rounding of its argument for |g| < 32), the division and the products."""
import pytest
import torch

from paper_2608_14205_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda", 0)
E4M3 = torch.float8_e4m3fn
SMALLEST = 2.0 ** -100


def make_ctx(k=2, E=8):
    return B.Context(1 << 16, 64, E, k, 1)


def blocks_of(n):
    return -(-n // 128)


def spread(scale, rows, cols, row_block):
    """Block scales [ceil(rows / row_block), ceil(cols / 128)] as a 64-bit matrix [rows, cols]."""
    s = scale.double().repeat_interleave(128, dim=1)[:, :cols]
    return s.repeat_interleave(row_block, dim=0)[:rows] if row_block > 1 else s


def offsets_of(counts, base=0):
    return torch.tensor([base] + [base + sum(counts[: i + 1]) for i in range(len(counts))], dtype=torch.int32, device=DEV)


class Case:
    """Random operands of one product; integers when exact results are wanted."""

    def __init__(self, counts, K, n, e4m3, swiglu, perm, seed=0, whole=False, k=2, base=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        E, P = len(counts), sum(counts)
        self.counts, self.K, self.n, self.e4m3, self.swiglu, self.k, self.base, self.P = counts, K, n, e4m3, swiglu, k, base, P
        self.n_out = n // 2 if swiglu else n
        self.x_rows = max(1, -(-(P + base) // k) if perm else P)
        if whole:
            draw = lambda *s: torch.randint(-2, 3, s, generator=g, device=DEV).float()
        else:
            draw = lambda *s: torch.randn(*s, generator=g, device=DEV)
        x, w = draw(self.x_rows, K), draw(E, n, K)
        self.xs = self.ws = None
        if e4m3:
            self.x, self.w = x.to(E4M3), w.to(E4M3)
            rb = 2 * blocks_of(n // 2) if swiglu else blocks_of(n)
            if whole:                                        # powers of two: products and sums stay exact
                self.xs = 2.0 ** torch.randint(-2, 3, (self.x_rows, blocks_of(K)), generator=g, device=DEV).float()
                self.ws = 2.0 ** torch.randint(-2, 3, (E, rb, blocks_of(K)), generator=g, device=DEV).float()
            else:
                self.xs = torch.rand(self.x_rows, blocks_of(K), generator=g, device=DEV) + 0.5
                self.ws = (torch.rand(E, rb, blocks_of(K), generator=g, device=DEV) + 0.5) * K ** -0.5
        else:
            self.x, self.w = x.bfloat16(), w.bfloat16() if whole else (w * K ** -0.5).bfloat16()
        self.offsets = offsets_of(counts, base)
        self.perm = None
        if perm:
            self.perm = torch.randperm(self.x_rows * k, generator=g, device=DEV)[: P + base].int()

    def values(self):
        """64-bit values of x and of the matrices."""
        x, w = self.x.double(), self.w.double()
        if self.e4m3:
            x = x * spread(self.xs, self.x_rows, self.K, 1)
            rows = [self.n // 2] * 2 if self.swiglu else [self.n]
            at, parts = 0, []
            for r in rows:
                parts.append(torch.stack([spread(self.ws[e, at: at + blocks_of(r)], r, self.K, 128) for e in range(len(self.counts))]))
                at += blocks_of(r)
            w = w * torch.cat(parts, dim=1)
        return x, w

    def expected(self):
        """(result before its rounding, bound on the error of the 32-bit sums)."""
        x, w = self.values()
        rows = self.perm[self.base:].long() // self.k if self.perm is not None else torch.arange(self.P, device=DEV)
        out, err = [], []
        at = 0
        steps = (self.K + blocks_of(self.K) + 4) * 2.0 ** -23
        for e, c in enumerate(self.counts):
            xe = x[rows[at: at + c]]
            at += c
            y, size = xe @ w[e].t(), xe.abs() @ w[e].abs().t() * steps
            if self.swiglu:
                gate, up = y.chunk(2, dim=1)
                dg, du = size.chunk(2, dim=1)
                silu = gate * torch.sigmoid(gate)
                y = silu * up
                size = 1.1 * up.abs() * dg + silu.abs() * du + 1.1 * dg * du + y.abs() * 2.0 ** -19
            out.append(y)
            err.append(size)
        return torch.cat(out), torch.cat(err)

    def matrix(self):
        return B.make_expert_matrix(self.w, self.ws, B.FB_ACT_SWIGLU if self.swiglu else B.FB_ACT_NONE)

    def run(self, ctx, quantize=False, extra=3, stream=None):
        """Rows behind the last slot keep what they held."""
        rows = self.P + extra
        if quantize:
            self.out = torch.full((rows, self.n_out), 7.0, device=DEV).to(E4M3)
            self.out_scale = torch.full((rows, blocks_of(self.n_out)), -1.0, device=DEV)
        else:
            self.out = torch.full((rows, self.n_out), 7.0, dtype=torch.bfloat16, device=DEV)
            self.out_scale = None
        x, xs = self.x, self.xs
        if self.perm is None:                                # x holds `rows` rows as well
            x = torch.cat([x[: self.P].view(torch.uint8 if self.e4m3 else torch.int16),
                           x.new_zeros(1).view(torch.uint8 if self.e4m3 else torch.int16)[0].expand(extra, self.K)]).view(x.dtype)
            xs = torch.cat([xs[: self.P], xs.new_ones(extra, xs.shape[1])]) if self.e4m3 else None
        self.kept = (x, xs)
        ctx.fb_expert_matmul(self.matrix(), x.contiguous(), xs, self.offsets, self.perm, rows, self.out, self.out_scale, stream=stream)
        torch.cuda.synchronize()
        assert ctx.fb_device_status() == 0
        assert (self.out[self.P:].float() == 7.0).all(), "rows behind the last slot are left as they were"
        return self.out[: self.P], self.out_scale[: self.P] if quantize else None


COUNTS = [[1], [5, 0, 3], [0, 16, 17, 0], [31, 32, 33], [255, 1, 256, 257], [300, 0, 0, 513, 64], [1000, 40]]
SHAPES = [(64, 128), (8, 8), (72, 136), (200, 264), (1040, 520)]
SHAPES_8BIT = [(128, 128), (16, 8), (144, 136), (272, 264), (1040, 520)]


@pytest.mark.parametrize("perm", [False, True])
@pytest.mark.parametrize("counts", COUNTS, ids=str)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_whole_numbers_give_exact_products(e4m3, shape, counts, perm):
    # products of small integers (and powers of two) are exact in 32 bits: the result is the exact one, rounded
    K, n = (SHAPES_8BIT if e4m3 else SHAPES)[shape]
    ctx = make_ctx(k=3)
    c = Case(counts, K, n, e4m3, False, perm, seed=shape, whole=True, k=3)
    got, _ = c.run(ctx)
    want, _ = c.expected()
    assert torch.equal(got, want.float().bfloat16())
    ctx.close()


@pytest.mark.parametrize("perm", [False, True])
@pytest.mark.parametrize("counts", COUNTS, ids=str)
@pytest.mark.parametrize("shape", [(64, 128), (16, 32), (80, 96), (208, 544), (1040, 288)], ids=str)
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_swiglu(e4m3, shape, counts, perm):
    K, n = shape
    ctx = make_ctx()
    c = Case(counts, K, n, e4m3, True, perm, seed=3)
    got, _ = c.run(ctx)
    want, err = c.expected()
    assert ((got.double() - want).abs() <= err + (want.abs() + err) * 2.0 ** -8 + 2.0 ** -133).all()
    ctx.close()


@pytest.mark.parametrize("counts", COUNTS, ids=str)
@pytest.mark.parametrize("shape", [(128, 256), (16, 32), (80, 96), (208, 544), (1040, 1056)], ids=str)
def test_swiglu_quantized(shape, counts):
    K, n = shape
    ctx = make_ctx()
    c = Case(counts, K, n, True, True, True, seed=4)
    q, scale = c.run(ctx, quantize=True)
    want, err = c.expected()
    s = spread(scale, c.P, c.n_out, 1)
    # the scale: the block's largest value / 448, that value off by at most the largest error in the block
    pad = torch.nn.functional.pad
    by_block = lambda v: pad(v, (0, blocks_of(c.n_out) * 128 - c.n_out)).view(c.P, -1, 128)
    top, e_top = by_block(want).abs().amax(2).clamp(min=SMALLEST), by_block(err).amax(2)
    assert ((scale.double() * 448 - top).abs() <= e_top + top * 2.0 ** -22).all()
    got = q.double() * s
    assert ((got - want).abs() <= err + (want.abs() + err) * (2.0 ** -4 + 2.0 ** -20) + s * 2.0 ** -10).all()
    ctx.close()


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_products_of_real_numbers(e4m3):
    ctx = make_ctx()
    c = Case([700, 3, 0, 250, 256], 2048, 768, e4m3, False, True, seed=5)
    got, _ = c.run(ctx)
    want, err = c.expected()
    assert ((got.double() - want).abs() <= err + (want.abs() + err) * 2.0 ** -8).all()
    ctx.close()


@pytest.mark.parametrize("perm", [False, True])
@pytest.mark.parametrize("counts", [[1100], [3000, 0, 200], [2047, 2], [1025, 1279, 1024]], ids=str)
@pytest.mark.parametrize("form", ["whole", "swiglu", "quantized"])
def test_many_rows_per_slot(form, counts, perm):
    # 1024 rows a slot and more on average: e4m3 products by pairs of blocks
    ctx = make_ctx(k=3)
    c = Case(counts, 272, 264 if form == "whole" else 288, True, form != "whole", perm, seed=8, whole=form == "whole", k=3)
    got, scale = c.run(ctx, quantize=form == "quantized")
    want, err = c.expected()
    if form == "whole":
        assert torch.equal(got, want.float().bfloat16())
    elif form == "swiglu":
        assert ((got.double() - want).abs() <= err + (want.abs() + err) * 2.0 ** -8 + 2.0 ** -133).all()
    else:
        s = spread(scale, c.P, c.n_out, 1)
        assert ((got.double() * s - want).abs() <= err + (want.abs() + err) * (2.0 ** -4 + 2.0 ** -20) + s * 2.0 ** -10).all()
    ctx.close()


@pytest.mark.parametrize("perm", [False, True])
@pytest.mark.parametrize("counts", [[1], [40], [3, 0, 130], [256], [300, 20]], ids=str)
@pytest.mark.parametrize("K", [512, 1040, 2064, 7168])
@pytest.mark.parametrize("form", ["bf16", "bf16 swiglu", "e4m3", "e4m3 swiglu", "quantized"])
def test_few_tiles_share_their_k_range(form, K, counts, perm):
    # so few tiles that clusters share them: pieces of equal and of different length
    e4m3, swiglu = form != "bf16" and form != "bf16 swiglu", form not in ("bf16", "e4m3")
    ctx = make_ctx(k=2)
    c = Case(counts, K, 320, e4m3, swiglu, perm, seed=K, whole=not swiglu)
    got, scale = c.run(ctx, quantize=form == "quantized")
    want, err = c.expected()
    if not swiglu:
        assert torch.equal(got, want.float().bfloat16())
    elif scale is None:
        assert ((got.double() - want).abs() <= err + (want.abs() + err) * 2.0 ** -8 + 2.0 ** -133).all()
    else:
        s = spread(scale, c.P, c.n_out, 1)
        assert ((got.double() * s - want).abs() <= err + (want.abs() + err) * (2.0 ** -4 + 2.0 ** -20) + s * 2.0 ** -10).all()
    again, _ = c.run(ctx, quantize=form == "quantized")
    assert torch.equal(got.view(torch.uint8), again.view(torch.uint8))
    ctx.close()


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("perm", [False, True])
def test_256_slots_and_one_token(e4m3, perm):
    ctx = make_ctx(k=8, E=256)
    counts = [0] * 256
    for e in (0, 3, 31, 32, 100, 200, 254, 255):
        counts[e] = 1
    c = Case(counts, 128, 64, e4m3, False, perm, seed=1, whole=True, k=8)
    got, _ = c.run(ctx)
    assert torch.equal(got, c.expected()[0].float().bfloat16())
    ctx.close()


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_a_rank_passes_its_own_slots(e4m3):
    # offsets that do not begin at zero: positions of perm are those of the whole batch, rows of out the rank's own
    ctx = make_ctx()
    c = Case([7, 300, 0, 33], 64, 128, e4m3, False, True, seed=2, whole=True, base=517)
    got, _ = c.run(ctx)
    assert torch.equal(got, c.expected()[0].float().bfloat16())
    ctx.close()


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("rows", [1, 127, 129, 1500])
def test_one_matrix_without_offsets(e4m3, rows):
    ctx = make_ctx(k=2)
    c = Case([rows], 144, 264, e4m3, False, False, seed=3, whole=True)
    out = torch.zeros(rows, 264, dtype=torch.bfloat16, device=DEV)
    ctx.fb_expert_matmul(c.matrix(), c.x, c.xs, None, None, rows, out)
    torch.cuda.synchronize()
    assert ctx.fb_device_status() == 0
    assert torch.equal(out, c.expected()[0].float().bfloat16())
    ctx.close()


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("swiglu", [False, True], ids=["none", "swiglu"])
def test_numbers_that_are_none_stay_in_their_row(e4m3, swiglu):
    # a NaN or an infinity in one token's row, beside it in the same tile and behind the slot's last row
    ctx = make_ctx(k=1)
    c = Case([40, 100], 128, 64, e4m3, swiglu, True, seed=4, k=1)
    clean, _ = c.run(ctx)
    clean = clean.clone()
    bad = c.perm[[3, 39, 77]].long()
    c.x.view(torch.uint8 if e4m3 else torch.int16)[bad, 5] = 0x7F if e4m3 else 0x7FC0
    if not e4m3:
        c.x[bad[1], 5] = float("inf")
    got, _ = c.run(ctx)
    hit = torch.zeros(140, dtype=torch.bool, device=DEV)
    hit[[3, 39, 77]] = True
    assert torch.equal(got[~hit], clean[~hit])
    assert got[3].isnan().all() and got[77].isnan().all()
    ctx.close()


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_extreme_gates(e4m3):
    # exp overflows, underflows and vanishes: silu(g) -> 0, g / 2 near 0, g
    ctx = make_ctx(k=1)
    c = Case([8], 16, 32, e4m3, True, False, seed=5, k=1)
    x, w = torch.zeros(8, 16), torch.zeros(1, 32, 16)
    x[:, 0] = torch.tensor([-448.0, -100.0, -20.0, -1.0, 0.0, 1.0, 20.0, 448.0])
    w[0, :16, 0], w[0, 16:, 1] = 1.0, 1.0
    x[:, 1] = 1.0
    c.x, c.w = (x.to(DEV).to(E4M3), w.to(DEV).to(E4M3)) if e4m3 else (x.to(DEV).bfloat16(), w.to(DEV).bfloat16())
    if e4m3:
        c.xs, c.ws = torch.ones(8, 1, device=DEV), torch.ones(1, 2, 1, device=DEV)
    got, _ = c.run(ctx)
    g = c.x.double()[:, :1].expand(8, 16)
    want = g / (1 + torch.exp(-g))
    # half a step of bf16, exp's rounding (|g| 2^-23, twice for the argument) and 2^-19; below the smallest 32-bit number: zero
    assert ((got.double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -19 + g.abs() * 2.0 ** -22) + 2.0 ** -126).all()
    ctx.close()


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_bad_offsets_and_rows_are_reported_and_nothing_else_is_written(e4m3):
    ctx = make_ctx(k=1)
    c = Case([20, 30, 10], 64, 64, e4m3, False, True, seed=6, whole=True, k=1)
    want = c.expected()[0].float().bfloat16()
    run = lambda: (ctx.fb_expert_matmul(c.matrix(), c.x, c.xs, c.offsets, c.perm, 60, out), torch.cuda.synchronize())
    out = torch.full((64, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    good = c.offsets.clone()
    c.offsets[2] = 90                                        # beyond the rows: slot 1 ends there, slot 2 falls
    run()
    assert ctx.fb_device_status() == B.FB_ERR_RANGE
    assert torch.equal(out[:20], want[:20]) and (out[20:] == 7.0).all()
    many = Case([20] * 40, 64, 64, e4m3, False, False, seed=6, whole=True, k=1)       # every other slot claims all rows
    many.offsets[:40:2], many.offsets[1::2] = 0, 800
    big = torch.full((800, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    ctx.fb_expert_matmul(many.matrix(), many.x, many.xs, many.offsets, None, 800, big)
    torch.cuda.synchronize()
    assert ctx.fb_device_status() == B.FB_ERR_RANGE
    assert (big == 7.0).all()
    c.offsets.copy_(good + 1000)                             # positions that perm cannot have
    out.fill_(7.0)
    run()
    assert ctx.fb_device_status() == B.FB_ERR_RANGE and (out == 7.0).all()
    c.offsets.copy_(good)
    c.perm[25], c.perm[26] = -5, 10 ** 9                     # outside x: row 0 instead
    run()
    assert ctx.fb_device_status() == B.FB_ERR_RANGE
    keep = torch.ones(60, dtype=torch.bool, device=DEV)
    keep[[25, 26]] = False
    assert torch.equal(out[:60][keep], want[keep])
    ctx.close()


def test_weights_and_results_beyond_32_bits():
    ctx = make_ctx(k=1)
    # three slots 2.2 GB apart, in part of a 6.7 GB buffer
    E, n, K, apart = 3, 128, 64, 1_100_000_000
    buf = torch.empty(2 * apart + n * K, dtype=torch.bfloat16, device=DEV)
    w = buf.as_strided((E, n, K), (apart, K, 1))
    g = torch.Generator(device=DEV).manual_seed(1)
    for e in range(E):
        w[e] = torch.randint(-2, 3, (n, K), generator=g, device=DEV).bfloat16()
    x = torch.randint(-2, 3, (90, K), generator=g, device=DEV).bfloat16()
    out = torch.empty(90, n, dtype=torch.bfloat16, device=DEV)
    ctx.fb_expert_matmul(B.make_expert_matrix(w), x, None, offsets_of([30, 30, 30]), None, 90, out)
    want = torch.cat([x[30 * e: 30 * e + 30].double() @ w[e].double().t() for e in range(E)])
    assert torch.equal(out, want.float().bfloat16())
    del buf, w
    # 4.6 billion results
    n, K, rows = 8192, 16, 560_000
    w = torch.randint(-2, 3, (1, n, K), generator=g, device=DEV).bfloat16()
    x = torch.randint(-2, 3, (rows, K), generator=g, device=DEV).bfloat16()
    out = torch.empty(rows, n, dtype=torch.bfloat16, device=DEV)
    ctx.fb_expert_matmul(B.make_expert_matrix(w), x, None, None, None, rows, out)
    for at in (0, 262_100, 559_900):
        part = slice(at, at + 100)
        assert torch.equal(out[part], (x[part].double() @ w[0].double().t()).float().bfloat16())
    assert ctx.fb_device_status() == 0
    ctx.close()


# ---------------------------------------------------------------- rows to e4m3
@pytest.mark.parametrize("rows,n", [(1, 16), (1, 128), (3, 144), (5, 2048), (77, 1040), (1000, 7168), (4097, 112)])
def test_quantized_rows(rows, n):
    ctx = make_ctx()
    g = torch.Generator(device=DEV).manual_seed(rows + n)
    x = (torch.randn(rows, n, generator=g, device=DEV) * torch.exp2(torch.randint(-30, 30, (rows, 1), generator=g, device=DEV).float())).bfloat16()
    x[0, : min(n, 128)] = 0.0                                # a block of zeros
    if rows > 2:
        x[2] = 2.0 ** -130                                   # below the smallest scale
    q = torch.full((rows + 1, n), 7.0, device=DEV).to(E4M3)
    scale = torch.full((rows + 1, blocks_of(n)), -1.0, device=DEV)
    ctx.fb_quantize_rows(x, rows, n, q, scale)
    torch.cuda.synchronize()
    assert (q[rows].float() == 7.0).all() and (scale[rows] == -1.0).all()
    pad = torch.nn.functional.pad(x.double(), (0, blocks_of(n) * 128 - n)).view(rows, -1, 128)
    top = pad.abs().amax(2).clamp(min=SMALLEST)
    # the scale is one 32-bit division; q is off by half a step, after a division and a product in 32 bits
    assert ((scale[:rows].double() - top / 448).abs() <= top / 448 * 2.0 ** -24).all()
    s = spread(scale[:rows], rows, n, 1)
    assert ((q[:rows].double() * s - x.double()).abs() <= x.double().abs() * (2.0 ** -4 + 2.0 ** -21) + s * 2.0 ** -10).all()
    assert not q[:rows].float().isnan().any()
    ctx.close()


def test_quantized_rows_with_numbers_that_are_none():
    ctx = make_ctx()
    x = torch.ones(3, 256, dtype=torch.bfloat16, device=DEV)
    x[0, 7], x[1, 200] = float("nan"), float("-inf")
    q, scale = torch.empty(3, 256, dtype=E4M3, device=DEV), torch.empty(3, 2, device=DEV)
    ctx.fb_quantize_rows(x, 3, 256, q, scale)
    torch.cuda.synchronize()
    v = q.float() * scale.repeat_interleave(128, dim=1)
    assert v[0, 7].isnan() and v[0].isnan().sum() == 1 and (v[2] == 1.0).all() and (v[1, :128] == 1.0).all()
    assert scale[1, 1].isinf() and not v[1, 200].isfinite()
    ctx.close()


def test_quantized_rows_beyond_32_bits():
    ctx = make_ctx()
    rows, n = 600_000, 7168                                  # 4.3 billion numbers
    x = torch.empty(rows, n, dtype=torch.bfloat16, device=DEV)
    for at in (0, 299_600, 599_900):
        x[at: at + 100] = torch.randn(100, n, device=DEV).bfloat16()
    q, scale = torch.empty(rows, n, dtype=E4M3, device=DEV), torch.empty(rows, n // 128, device=DEV)
    ctx.fb_quantize_rows(x, rows, n, q, scale)
    q1, scale1 = torch.empty(100, n, dtype=E4M3, device=DEV), torch.empty(100, n // 128, device=DEV)
    for at in (0, 299_600, 599_900):
        ctx.fb_quantize_rows(x[at: at + 100].contiguous(), 100, n, q1, scale1)
        assert torch.equal(q[at: at + 100].view(torch.uint8), q1.view(torch.uint8)) and torch.equal(scale[at: at + 100], scale1)
    ctx.close()


# ---------------------------------------------------------------- weighted sum
@pytest.mark.parametrize("k", range(1, 9))
@pytest.mark.parametrize("T,n", [(1, 8), (3, 1032), (130, 2048)])
@pytest.mark.parametrize("add", ["none", "other", "itself"])
def test_combination(k, T, n, add):
    ctx = make_ctx(k=k)
    g = torch.Generator(device=DEV).manual_seed(k)
    rows = torch.randn(T * k, n, generator=g, device=DEV).bfloat16()
    w = torch.rand(T, k, generator=g, device=DEV)
    inv = torch.randperm(T * k, generator=g, device=DEV).int()
    more = torch.randn(T, n, generator=g, device=DEV).bfloat16()
    out = more.clone() if add == "itself" else torch.zeros(T, n, dtype=torch.bfloat16, device=DEV)
    ctx.fb_combine(rows, w, inv, T, n, None if add == "none" else out if add == "itself" else more, out)
    torch.cuda.synchronize()
    terms = rows[inv.long()].view(T, k, n).double() * w.double()[:, :, None]
    want, size = terms.sum(1), terms.abs().sum(1)
    if add != "none":
        want, size = want + more.double(), size + more.double().abs()
    err = size * (k + 1) * 2.0 ** -24
    assert ((out.double() - want).abs() <= err + (want.abs() + err) * 2.0 ** -8).all()
    assert ctx.fb_device_status() == 0
    ctx.close()


def test_combination_beyond_32_bits_and_bad_positions():
    ctx = make_ctx(k=2)
    T, n = 300_000, 8192                                     # 4.9 billion numbers in rows
    rows = torch.zeros(2 * T, n, dtype=torch.bfloat16, device=DEV)
    rows[-1], rows[5] = 3.0, 1.0
    inv = torch.zeros(2 * T, dtype=torch.int32, device=DEV)
    inv[0], inv[1] = 2 * T - 1, 5
    w = torch.ones(T, 2, device=DEV)
    out = torch.empty(T, n, dtype=torch.bfloat16, device=DEV)
    ctx.fb_combine(rows, w, inv, T, n, None, out)
    assert (out[0] == 4.0).all() and (out[1:] == 0).all()
    assert ctx.fb_device_status() == 0
    inv[7], inv[8] = 2 * T, -1
    ctx.fb_combine(rows, w, inv, T, n, None, out)
    assert ctx.fb_device_status() == B.FB_ERR_RANGE and (out[0] == 4.0).all()
    ctx.close()


# ---------------------------------------------------------------- calls
def test_refusals():
    ctx = make_ctx(k=2, E=8)
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=DEV)
    f8 = lambda *s: torch.zeros(*s, device=DEV).to(E4M3)
    f32 = lambda *s: torch.zeros(*s, device=DEV)
    off = offsets_of([4, 4])
    cases = []

    def matmul(want, w, ws=None, act=0, x=None, xs=None, offsets=off, perm=None, rows=8, out=None, out_scale=None, edit=None):
        m = B.make_expert_matrix(w, ws, act)
        if edit:
            edit(m)
        cases.append((want, lambda: ctx.fb_expert_matmul(m, x, xs, offsets, perm, rows, out, out_scale)))

    A, U = B.FB_ERR_INVALID_ARG, B.FB_ERR_UNSUPPORTED_SHAPE
    good = dict(w=bf(2, 32, 64), x=bf(8, 64), out=bf(8, 32))
    matmul(U, bf(2, 32, 60), x=bf(8, 60), out=bf(8, 32))                                   # rows of 120 bytes
    matmul(U, f8(2, 32, 72), f32(2, 1, 1), x=f8(8, 72), xs=f32(8, 1), out=bf(8, 32))       # rows of 72 bytes
    matmul(U, bf(2, 12, 64), x=bf(8, 64), out=bf(8, 12))                                   # columns
    matmul(U, bf(2, 48, 64), act=1, x=bf(8, 64), out=bf(8, 24))                            # SwiGLU: 24 outputs
    matmul(U, bf(257, 8, 8), x=bf(8, 8), out=bf(8, 8), offsets=offsets_of([0] * 257))
    matmul(A, f8(2, 32, 64), None, x=f8(8, 64), xs=f32(8, 1), out=bf(8, 32))               # e4m3 without scales
    matmul(A, f8(2, 32, 64), f32(2, 1, 1), x=f8(8, 64), out=bf(8, 32))
    matmul(A, **{**good, "x": bf(8, 64)}, xs=f32(8, 1))                                    # bf16 with scales
    matmul(A, **{**good, "out": f8(8, 32)}, out_scale=f32(8, 1))                            # bf16 operands give bf16 results
    matmul(A, f8(2, 32, 64), f32(2, 1, 1), x=f8(8, 64), xs=f32(8, 1), out=f8(8, 32), out_scale=f32(8, 1))   # nor without SwiGLU
    matmul(A, **good, offsets=None)                                                        # two slots without offsets
    matmul(A, **{**good, "x": bf(7, 64)})                                                  # fewer rows of x than of out
    matmul(A, **{**good, "x": bf(8 * 64 + 1)[1:].view(8, 64)})                             # not on 16 bytes
    matmul(A, **{**good, "out": bf(8 * 32 + 1)[1:].view(8, 32)})
    matmul(A, **{**good, "out": None})
    matmul(A, **good, rows=-1)
    matmul(A, **good, edit=lambda m: setattr(m, "act", 2))
    matmul(A, **good, edit=lambda m: setattr(m, "dtype", 1))
    matmul(A, **good, edit=lambda m: setattr(m, "slot_bytes", 64))                         # slots that overlap
    matmul(A, **good, edit=lambda m: setattr(m, "slot_bytes", m.slot_bytes + 8))
    matmul(U, **good, edit=lambda m: setattr(m, "slot_bytes", 1 << 40))
    matmul(A, **good, edit=lambda m: setattr(m, "w", None))
    x, q, s = bf(4, 64), f8(4, 64), f32(4, 1)
    for want, rows, n, xx, qq in ((A, -1, 64, x, q), (A, 4, 24, x, q), (A, 4, 0, x, q), (A, 4, 64, None, q), (A, 4, 64, bf(257)[1:], q),
                                  (U, 2 ** 40, 7168, x, q)):
        cases.append((want, lambda rows=rows, n=n, xx=xx, qq=qq: ctx.fb_quantize_rows(xx if xx is not None else bf(0), rows, n, qq, s)))
    w, inv, o = f32(4, 2), torch.zeros(8, dtype=torch.int32, device=DEV), bf(4, 64)
    for want, T, n, rr, oo, aa in ((A, -1, 64, x, o, None), (A, 4, 60, x, o, None), (A, 4, 64, None, o, None), (A, 4, 64, x, None, None),
                                   (A, 4, 64, x, o, bf(257)[1:]), (U, 2 ** 30, 64, x, o, None)):
        cases.append((want, lambda T=T, n=n, rr=rr, oo=oo, aa=aa: ctx.fb_combine(rr, w, inv, T, n, aa, oo)))
    launches = ctx.fb_launch_count()
    for i, (want, call) in enumerate(cases):
        with pytest.raises(B.FbError) as e:
            call()
        assert e.value.status == want, i
    # nothing to do is no error and no launch
    ctx.fb_expert_matmul(B.make_expert_matrix(good["w"]), bf(0, 64), None, off, None, 0, bf(0, 32))
    ctx.fb_quantize_rows(bf(0, 64), 0, 64, f8(0, 64), f32(0, 1))
    ctx.fb_combine(bf(0, 64), w, inv, 0, 64, None, bf(0, 64))
    assert ctx.fb_launch_count() == launches
    # a launch that fails is reported; the next one is not affected
    ctx.fb_fail_launch(1)
    with pytest.raises(B.FbError) as e:
        ctx.fb_expert_matmul(B.make_expert_matrix(good["w"]), good["x"], None, off, None, 8, good["out"])
    assert e.value.status == B.FB_ERR_CUDA
    ctx.fb_expert_matmul(B.make_expert_matrix(good["w"]), good["x"], None, off, None, 8, good["out"])
    torch.cuda.synchronize()
    assert ctx.fb_device_status() == 0
    ctx.close()


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_captured_calls_follow_their_buffers(e4m3):
    ctx = make_ctx()
    c = Case([40, 0, 300, 5], 256, 256, e4m3, True, True, seed=7)
    quantize = e4m3
    first, s1 = c.run(ctx, quantize=quantize)
    first = first.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.fb_expert_matmul(c.matrix(), c.x, c.xs, c.offsets, c.perm, c.P + 3, c.out, c.out_scale)
    d = Case([300, 40, 3, 2], 256, 256, e4m3, True, True, seed=9)          # as many rows, other counts
    for name in ("x", "w", "perm", "offsets", *(["xs", "ws"] if e4m3 else [])):
        getattr(c, name).view(torch.uint8).copy_(getattr(d, name).view(torch.uint8))
    c.out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    got = c.out[: c.P].clone()
    want, _ = d.run(ctx, quantize=quantize)
    assert torch.equal(got.view(torch.uint8), want.view(torch.uint8))
    ctx.close()


def test_calls_of_one_context_overlap_on_two_streams():
    ctx = make_ctx()
    cases = [Case([30, 500, 7, 90], 512, 512, e4m3, True, True, seed=int(e4m3)) for e4m3 in (False, True)]
    want = [c.run(ctx, quantize=c.e4m3)[0].clone() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [[torch.empty_like(w) for _ in range(20)] for w in want]
    scales = [torch.empty(c.P, blocks_of(c.n_out), device=DEV) if c.e4m3 else None for c in cases]
    torch.cuda.synchronize()
    for i in range(20):
        for c, s, o, sc in zip(cases, streams, outs, scales):
            ctx.fb_expert_matmul(c.matrix(), c.x, c.xs, c.offsets, c.perm, c.P, o[i], sc, stream=s)
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert all(torch.equal(w.view(torch.uint8), t.view(torch.uint8)) for t in o)
    assert ctx.fb_device_status() == 0
    ctx.close()
