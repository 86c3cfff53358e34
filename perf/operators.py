"""The experts' side of an MoE layer: what follows the dispatch index of ``fb_route_dispatch``.

Four operators, as a serving program calls them between the router of a layer and the next layer:

``quantize``  rows of hidden states to 8-bit floats (e4m3) with one scale per 128 columns
``experts``   products grouped by expert: every row of the dispatch order with the matrix of its
              slot; "up" is gate and up projection with SwiGLU (rows gathered by token), "down" the
              projection back to the hidden size (rows in dispatch order); bf16 weights, or e4m3
              weights with one scale per 128 x 128 block and e4m3 rows
``combine``   the experts' rows of a token, weighted and added

Sizes are those of ``paper_2608_14205_b200/inputs.py``: an expert of the qwen3 workload is 9 MiB, three
matrices of 2048 x 768 in bf16; one of dsv3 is 44 040 192 bytes, three of 7168 x 2048 in e4m3.
"""
import functools
import math

import torch

own = False

QWEN3 = dict(d=2048, E=128, k=8, inter=768, dtype="bf16")
DSV3 = dict(d=7168, E=256, k=8, inter=2048, dtype="e4m3")
SKEW = 0.5                    # popularity of the experts: rank ** -SKEW
BLOCK = 128
E4M3_MAX = 448.0
SMALLEST = 2.0 ** -100        # a block of zeros takes this for its largest value


def listed():
    return [
        # Quantisation of a nearly drained batch: launch and latency.
        dict(name="quantize 40x2048", op="quantize", T=40, n=2048),
        # Of the hidden states of a whole prefill step.
        dict(name="quantize 16384x7168", op="quantize", T=16384, n=7168),
        # Eight experts' rows of each token of a small decode batch.
        dict(QWEN3, name="combine qwen3 40", op="combine", T=40),
        # Of a prefill step: the largest traffic of a layer that no product hides.
        dict(DSV3, name="combine dsv3 16384", op="combine", T=16384),
        # One token in decode: eight experts' matrices are read for one row each.
        dict(QWEN3, name="up qwen3 1", op="experts", way="up", T=1),
        # A decode batch: nearly all experts, a few rows each; bound by the weights.
        dict(QWEN3, name="down qwen3 40", op="experts", way="down", T=40),
        # A short ragged prefill.
        dict(QWEN3, name="down qwen3 1733", op="experts", way="down", T=1733),
        # An ordinary prefill step.
        dict(QWEN3, name="up qwen3 8192", op="experts", way="up", T=8192),
        # 16 sequences of 8K tokens: the largest call.
        dict(QWEN3, name="up qwen3 131072", op="experts", way="up", T=131072),
        # 8-bit weights, decode; the rows come out quantised for the down projection.
        dict(DSV3, name="up dsv3 64", op="experts", way="up", T=64),
        # The headline prefill step of that model.
        dict(DSV3, name="up dsv3 16384", op="experts", way="up", T=16384),
        # The way back, ragged.
        dict(DSV3, name="down dsv3 5003", op="experts", way="down", T=5003),
    ]


def _between(rng, lo, hi):
    """Spread over the logarithm of the range."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "combine", "experts", "experts", "experts", "experts"])
    if op == "quantize":
        return dict(op=op, T=_between(rng, 1, 16384), n=16 * _between(rng, 8, 448))
    E = _between(rng, 1, 256)
    k = min(E, rng.randint(1, 8))
    dtype = rng.choice(["bf16", "e4m3"])
    step = 16 if dtype == "e4m3" else 8
    c = dict(op=op, d=step * _between(rng, 256 // step, 7168 // step), E=E, k=k, inter=16 * _between(rng, 8, 128), dtype=dtype,
             T=_between(rng, 1, 16384))
    if op == "experts":
        c["way"] = rng.choice(["up", "down"])
        while c["T"] * c["k"] * c["d"] * c["inter"] > 5e11:
            c["T"] //= 2
    return c


def _popularity(E):
    w = torch.arange(1, E + 1, dtype=torch.float64) ** -SKEW
    return w / w.sum()


def work(case):
    if case["op"] == "quantize":
        n = case["T"] * case["n"]
        return {"bytes": 3 * n + 4 * case["T"] * -(-case["n"] // BLOCK), "flops": 2 * n}
    T, k, d = case["T"], case["k"], case["d"]
    if case["op"] == "combine":
        return {"bytes": 2 * T * k * d + 8 * T * k + 2 * T * d, "flops": 2 * T * k * d}
    # experts that at least one token chose, on average
    touched = float((1 - (1 - (k * _popularity(case["E"])).clamp(max=1)) ** T).sum())
    up, e4m3 = case["way"] == "up", case["dtype"] == "e4m3"
    K, n_w, n_out = (d, 2 * case["inter"], case["inter"]) if up else (case["inter"], d, d)
    rows_in, rows = T if up else T * k, T * k
    blocks_k = -(-K // BLOCK)
    size = 1 if e4m3 else 2
    nbytes = touched * n_w * K * size + rows_in * K * size + (4 * rows if up else 0) + 4 * (case["E"] + 1)
    nbytes += rows * n_out * (1 if up and e4m3 else 2)
    if e4m3:
        nbytes += 4 * touched * blocks_k * -(-n_w // BLOCK) + 4 * rows_in * blocks_k + (4 * rows * -(-n_out // BLOCK) if up else 0)
    return {"bytes": nbytes, "flops": 2 * rows * n_w * K}


# ------------------------------------------------------------------ inputs
def _quantized_rows(x):
    """e4m3 values and block scales of the rows of x (32-bit floats)."""
    rows, n = x.shape
    blocks = -(-n // BLOCK)
    x = torch.nn.functional.pad(x, (0, blocks * BLOCK - n)).view(rows, blocks, BLOCK)
    top = x.abs().amax(dim=2, keepdim=True).clamp(min=SMALLEST)
    q = (x * (E4M3_MAX / top)).to(torch.float8_e4m3fn)
    return q.view(rows, blocks * BLOCK)[:, :n].contiguous(), (top / E4M3_MAX).view(rows, blocks)


def _matrices(E, n, K, e4m3, g):
    """A matrix [n][K] for each slot; e4m3: with a scale for each 128 x 128 block."""
    dev = g.device
    if not e4m3:
        w = torch.empty(E, n, K, dtype=torch.bfloat16, device=dev)
        for e in range(E):
            w[e] = torch.randn(n, K, generator=g, device=dev) * 0.02
        return w, None
    bn, bk = -(-n // BLOCK), -(-K // BLOCK)
    w = torch.empty(E, n, K, dtype=torch.float8_e4m3fn, device=dev)
    scale = torch.empty(E, bn, bk, device=dev)
    for e in range(E):
        full = torch.zeros(bn * BLOCK, bk * BLOCK, device=dev)
        full[:n, :K] = torch.randn(n, K, generator=g, device=dev) * 0.02
        full = full.view(bn, BLOCK, bk, BLOCK)
        scale[e] = full.abs().amax(dim=(1, 3)).clamp(min=SMALLEST) / E4M3_MAX
        w[e] = (full / scale[e][:, None, :, None]).view(bn * BLOCK, bk * BLOCK)[:n, :K].to(torch.float8_e4m3fn)
    return w, scale


def _gate_up(E, inter, K, e4m3, g):
    """Gate rows, then up rows, of each slot; the scales' blocks start afresh at the up rows."""
    gate, gs = _matrices(E, inter, K, e4m3, g)
    up, us = _matrices(E, inter, K, e4m3, g)
    return torch.cat([gate, up], dim=1), torch.cat([gs, us], dim=1) if e4m3 else None


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    T = case["T"]
    if case["op"] == "quantize":
        n = case["n"]
        x = torch.randn(T, n, generator=g, device=dev).to(torch.bfloat16)
        return dict(case=case, x=x, q=torch.empty(T, n, dtype=torch.float8_e4m3fn, device=dev),
                    scale=torch.empty(T, -(-n // BLOCK), device=dev))
    E, k, d, inter = case["E"], case["k"], case["d"], case["inter"]
    P, e4m3 = T * k, case["dtype"] == "e4m3"
    # the outcome of routing: k different experts per token, and the dispatch index of them
    order = torch.randperm(E, generator=g, device=dev)
    noise = -torch.log(-torch.log(torch.rand(T, E, generator=g, device=dev).clamp(1e-9, 1 - 1e-7)))
    score, ids = (_popularity(E).float().to(dev)[order].log() + noise).topk(k, dim=1)
    weights = torch.softmax(score, dim=1)
    flat = ids.reshape(-1)
    perm = torch.argsort(flat, stable=True)
    inv_perm = torch.empty_like(perm)
    inv_perm[perm] = torch.arange(P, device=dev)
    slot_offsets = torch.zeros(E + 1, dtype=torch.int64, device=dev)
    slot_offsets[1:] = torch.bincount(flat, minlength=E).cumsum(0)
    s = dict(case=case, perm=perm.int(), inv_perm=inv_perm.int(), slot_offsets=slot_offsets.int(), weights=weights)
    if case["op"] == "combine":
        s["rows"] = torch.randn(P, d, generator=g, device=dev).to(torch.bfloat16)
        s["out"] = torch.empty(T, d, dtype=torch.bfloat16, device=dev)
        return s
    up = case["way"] == "up"
    s["spans"] = slot_offsets.tolist()
    s["w"], s["w_scale"] = _gate_up(E, inter, d, e4m3, g) if up else _matrices(E, d, inter, e4m3, g)
    x = torch.randn(T if up else P, d if up else inter, generator=g, device=dev).to(torch.bfloat16)
    s["x"], s["x_scale"] = _quantized_rows(x.float()) if e4m3 else (x, None)
    n_out = inter if up else d
    s["out"] = torch.empty(P, n_out, dtype=torch.float8_e4m3fn if up and e4m3 else torch.bfloat16, device=dev)
    s["out_scale"] = torch.empty(P, -(-n_out // BLOCK), device=dev) if up and e4m3 else None
    return s


# ------------------------------------------------------------------ the plain forms
def _plain_values(q, scale, rows_per_scale):
    """The 32-bit values that e4m3 numbers and the scales of their blocks stand for."""
    by_row = scale.repeat_interleave(rows_per_scale, dim=0)[: q.shape[0]] if rows_per_scale > 1 else scale
    return q.float() * by_row.repeat_interleave(BLOCK, dim=1)[:, : q.shape[1]]


def _plain_weights(s, e):
    w, scale = s["w"][e], s["w_scale"]
    if scale is None:
        return w.float()
    if s["case"]["way"] == "down":
        return _plain_values(w, scale[e], BLOCK)
    half, blocks = w.shape[0] // 2, scale.shape[1] // 2
    return torch.cat([_plain_values(w[:half], scale[e, :blocks], BLOCK), _plain_values(w[half:], scale[e, blocks:], BLOCK)])


def _plain_experts(s):
    up, e4m3 = s["case"]["way"] == "up", s["x_scale"] is not None
    x = _plain_values(s["x"], s["x_scale"], 1) if e4m3 else s["x"].float()
    if up:
        x = x[s["perm"] // s["case"]["k"]]
    n_out = s["out"].shape[1]
    y = torch.empty(x.shape[0], n_out, device=x.device)
    for e, (lo, hi) in enumerate(zip(s["spans"][:-1], s["spans"][1:])):
        if lo < hi:
            r = x[lo:hi] @ _plain_weights(s, e).t()
            y[lo:hi] = r[:, :n_out] / (1 + torch.exp(-r[:, :n_out])) * r[:, n_out:] if up else r
    if not (up and e4m3):
        return y.to(torch.bfloat16)
    q, scale = _quantized_rows(y)
    return dict(q=q, scale=scale)


def _plain(s):
    op = s["case"]["op"]
    if op == "quantize":
        q, scale = _quantized_rows(s["x"].float())
        return dict(q=q, scale=scale)
    if op == "combine":
        c = s["case"]
        rows = s["rows"][s["inv_perm"]].view(c["T"], c["k"], c["d"]).float()
        return (rows * s["weights"][:, :, None]).sum(dim=1).to(torch.bfloat16)
    return _plain_experts(s)


# ------------------------------------------------------------------ the framework's calls
@functools.lru_cache(maxsize=None)
def _context(d, E, k):
    """The one handle that a program keeps for the layers of a model."""
    from paper_2608_14205_b200 import binding as B
    return B.Context(131072, d, E, k, 1)


def _own(s):
    from paper_2608_14205_b200 import binding as B
    c = s["case"]
    if c["op"] == "quantize":
        _context(1024, 8, 2).fb_quantize_rows(s["x"], c["T"], c["n"], s["q"], s["scale"])
        return dict(q=s["q"], scale=s["scale"])
    ctx = _context(c["d"], c["E"], c["k"])
    if c["op"] == "combine":
        ctx.fb_combine(s["rows"], s["weights"], s["inv_perm"], c["T"], c["d"], None, s["out"])
        return s["out"]
    up = c["way"] == "up"
    matrix = B.make_expert_matrix(s["w"], s["w_scale"], B.FB_ACT_SWIGLU if up else B.FB_ACT_NONE)
    ctx.fb_expert_matmul(matrix, s["x"], s["x_scale"], s["slot_offsets"], s["perm"] if up else None, c["T"] * c["k"], s["out"],
                         s["out_scale"])
    return s["out"] if s["out_scale"] is None else dict(q=s["out"], scale=s["out_scale"])


def run(s):
    return _own(s) if own else _plain(s)


# ------------------------------------------------------------------ in 64 bits
def _nearest_e4m3(v):
    """v (64 bits) on the grid of e4m3: three bits behind the leading one, steps of 2^-9 below 2^-6, ties to even."""
    exponent = torch.frexp(v.abs()).exponent.clamp(min=-5) - 1
    step = torch.exp2((exponent - 3).double())
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _exact_quantized(y):
    """The grid of blocks one by one: last block of a row may be shorter."""
    n = y.shape[1]
    q, scale = torch.empty_like(y), y.new_empty(y.shape[0], -(-n // BLOCK))
    for b, at in enumerate(range(0, n, BLOCK)):
        part = y[:, at:at + BLOCK]
        scale[:, b] = part.abs().max(dim=1).values.clamp(min=SMALLEST) / E4M3_MAX
        q[:, at:at + BLOCK] = _nearest_e4m3(part / scale[:, b:b + 1])
    return dict(q=q, scale=scale)


def _exact_product(s, x, xs, e, first_row, n, first_block):
    """x times the transposed rows [first_row, first_row + n) of slot e's matrix, one 128-column block after the other."""
    w = s["w"][e, first_row:first_row + n].double()
    if xs is None:
        return x.double() @ w.t()
    blocks = torch.arange(n, device=w.device) // BLOCK + first_block
    y = torch.zeros(x.shape[0], n, dtype=torch.float64, device=w.device)
    for b, at in enumerate(range(0, w.shape[1], BLOCK)):
        part = x[:, at:at + BLOCK].double() @ w[:, at:at + BLOCK].t()
        y += part * xs[:, b:b + 1].double() * s["w_scale"][e, blocks, b].double()
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        return _exact_quantized(s["x"].double())
    if case["op"] == "combine":
        y = torch.zeros(case["T"], case["d"], dtype=torch.float64, device=s["rows"].device)
        at = s["inv_perm"].view(case["T"], case["k"]).long()
        for j in range(case["k"]):
            y += s["weights"][:, j:j + 1].double() * s["rows"][at[:, j]].double()
        return y
    up, k = case["way"] == "up", case["k"]
    n_out = s["out"].shape[1]
    y = torch.zeros(case["T"] * k, n_out, dtype=torch.float64, device=s["x"].device)
    for e in range(case["E"]):
        lo, hi = s["spans"][e], s["spans"][e + 1]
        if lo == hi:
            continue
        rows = s["perm"][lo:hi].long() // k if up else torch.arange(lo, hi, device=y.device)
        x, xs = s["x"][rows], None if s["x_scale"] is None else s["x_scale"][rows]
        if up:
            g = _exact_product(s, x, xs, e, 0, n_out, 0)
            u = _exact_product(s, x, xs, e, n_out, n_out, -(-n_out // BLOCK))
            y[lo:hi] = g * torch.sigmoid(g) * u
        else:
            y[lo:hi] = _exact_product(s, x, xs, e, 0, n_out, 0)
    return _exact_quantized(y) if up and s["x_scale"] is not None else y
