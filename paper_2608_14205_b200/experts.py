"""The routed experts of one layer as slot images: what `fb_apply_swaps` exchanges between slots and
`fb_expert_matmul` reads.

One image per slot holds an expert's three matrices (and, in e4m3, their block scales), so a swap of
two experts is one exchange of two images and the products need no other change than the placement:

    gate [inter][d] | up [inter][d] | down [d][inter] | scales of gate, up, down (e4m3 only)

This module owns the buffer and passes pointers; products, quantisation of rows and exchange run in the
library's kernels.  Only `load`, which brings a checkpoint's matrices into a slot, is torch code.
"""
from __future__ import annotations

import torch

from . import binding as B

BLOCK = 128                     # side of a block of weights that shares a scale
E4M3_MAX = 448.0
SMALLEST = 2.0 ** -100          # a block of zeros takes this for its largest value, as in fb_quantize_rows


def _blocks(n: int) -> int:
    return -(-n // BLOCK)


def quantize_matrix(w: torch.Tensor) -> tuple[torch.Tensor, torch.Tensor]:
    """e4m3 values of w [n, K] and the float32 scale of each 128 x 128 block."""
    n, K = w.shape
    bn, bk = _blocks(n), _blocks(K)
    full = torch.nn.functional.pad(w.float(), (0, bk * BLOCK - K, 0, bn * BLOCK - n)).view(bn, BLOCK, bk, BLOCK)
    top = full.abs().amax(dim=(1, 3)).clamp(min=SMALLEST)
    q = (full * (E4M3_MAX / top)[:, None, :, None]).to(torch.float8_e4m3fn)
    return q.view(bn * BLOCK, bk * BLOCK)[:n, :K].contiguous(), top / E4M3_MAX


class SlotExperts:
    """Images of E experts of hidden size d and intermediate size `inter` on one GPU."""

    def __init__(self, E: int, d: int, inter: int, e4m3: bool = False, device: int = 0):
        assert d % 16 == 0 and inter % 16 == 0, "d and inter: multiples of 16"
        self.E, self.d, self.inter, self.e4m3 = E, d, inter, e4m3
        self.dtype = torch.float8_e4m3fn if e4m3 else torch.bfloat16
        size = 1 if e4m3 else 2
        weights = 3 * d * inter * size                                   # a multiple of 256: the scales are aligned
        up_blocks, k_up, down_blocks, k_down = 2 * _blocks(inter), _blocks(d), _blocks(d), _blocks(inter)
        scales = 4 * (up_blocks * k_up + down_blocks * k_down) if e4m3 else 0
        self.image_bytes = (weights + scales + 15) // 16 * 16
        self.images = torch.zeros(E, self.image_bytes, dtype=torch.uint8, device=torch.device("cuda", device))

        def part(dtype, at, rows, cols):
            flat = self.images.view(-1).view(dtype)
            size = flat.element_size()
            return flat.as_strided((E, rows, cols), (self.image_bytes // size, cols, 1), at // size)

        self.gate_up = part(self.dtype, 0, 2 * inter, d)
        self.down = part(self.dtype, 2 * d * inter * size, d, inter)
        self.gate_up_scale = self.down_scale = None
        if e4m3:
            self.gate_up_scale = part(torch.float32, weights, up_blocks, k_up)
            self.down_scale = part(torch.float32, weights + 4 * up_blocks * k_up, down_blocks, k_down)
        self.up_matrix = B.make_expert_matrix(self.gate_up, self.gate_up_scale, B.FB_ACT_SWIGLU)
        self.down_matrix = B.make_expert_matrix(self.down, self.down_scale, B.FB_ACT_NONE)

    def load(self, slot: int, gate: torch.Tensor, up: torch.Tensor, down: torch.Tensor) -> None:
        """An expert's matrices (gate, up [inter, d], down [d, inter]) into a slot, quantised if the images are e4m3."""
        dev, inter = self.images.device, self.inter
        gate, up, down = (m.to(dev) for m in (gate, up, down))
        if not self.e4m3:
            self.gate_up[slot, :inter], self.gate_up[slot, inter:], self.down[slot] = gate, up, down
            return
        half = _blocks(inter)
        for at, blocks, m in ((slice(0, inter), slice(0, half), gate), (slice(inter, None), slice(half, None), up)):
            self.gate_up[slot, at], self.gate_up_scale[slot, blocks] = quantize_matrix(m)
        self.down[slot], self.down_scale[slot] = quantize_matrix(down)

    def apply_swaps(self, expert_to_slot: torch.Tensor, swaps: torch.Tensor, n_swaps: torch.Tensor, max_swaps: int,
                    status_word=None, stream=None) -> None:
        """The accepted swaps of a plan (expert_to_slot: the placement before it) applied to the images."""
        B.fb_apply_swaps(self.images, self.image_bytes, self.E, expert_to_slot, swaps, n_swaps, max_swaps, status_word, stream)


class ExpertBuffers:
    """What the experts' side of a step needs between its calls, for up to `tokens` tokens of k experts each."""

    def __init__(self, experts: SlotExperts, tokens: int, k: int):
        dev, d, inter, rows = experts.images.device, experts.d, experts.inter, max(1, tokens * k)
        self.hidden = torch.empty(rows, inter, dtype=experts.dtype, device=dev)
        self.rows = torch.empty(rows, d, dtype=torch.bfloat16, device=dev)
        self.out = torch.empty(max(1, tokens), d, dtype=torch.bfloat16, device=dev)
        self.x = self.x_scale = self.hidden_scale = None
        if experts.e4m3:
            self.x = torch.empty(max(1, tokens), d, dtype=experts.dtype, device=dev)
            self.x_scale = torch.empty(max(1, tokens), _blocks(d), device=dev)
            self.hidden_scale = torch.empty(rows, _blocks(inter), device=dev)


def run_experts(ctx: B.Context, experts: SlotExperts, buf: ExpertBuffers, H: torch.Tensor, T: int, k: int, topk_w: torch.Tensor,
                slot_offsets: torch.Tensor, perm: torch.Tensor, inv_perm: torch.Tensor, addend=None, stream=None) -> torch.Tensor:
    """Sum over the chosen experts of weight x expert(H[t]) (+ addend[t]) for every token, from a dispatch index.

    Up projection with SwiGLU over the tokens' rows in dispatch order, down projection, combination: three launches,
    with e4m3 images four (the rows of H are quantised once per token; the up projection quantises its own results)."""
    assert H.shape[1] == experts.d, "hidden states of another size than the experts'"
    rows = T * k
    out = buf.out[:T]
    x, x_scale, hidden_scale = H, None, None
    if experts.e4m3:
        x, x_scale, hidden_scale = buf.x[:T], buf.x_scale[:T], buf.hidden_scale[:rows]
        ctx.fb_quantize_rows(H, T, experts.d, x, x_scale, stream=stream)
    hidden = buf.hidden[:rows]
    ctx.fb_expert_matmul(experts.up_matrix, x, x_scale, slot_offsets, perm, rows, hidden, hidden_scale, stream=stream)
    ctx.fb_expert_matmul(experts.down_matrix, hidden, hidden_scale, slot_offsets, None, rows, buf.rows, stream=stream)
    ctx.fb_combine(buf.rows, topk_w, inv_perm, T, experts.d, addend, out, stream=stream)
    return out
