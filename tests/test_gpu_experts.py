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
