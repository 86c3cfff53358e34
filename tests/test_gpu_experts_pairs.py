"""The e4m3 products by pairs of blocks (1024 rows a slot and more on average) where a tile's k-blocks go round the ring several
times and every pair walks over several tiles, and guards around the results of every form.  Tolerances: see test_gpu_experts."""
import pytest
import torch

from paper_2608_14205_b200 import binding as B

from .test_gpu_experts import DEV, E4M3, SMALLEST, Case, blocks_of, make_ctx, spread

pytestmark = pytest.mark.gpu


def check(c, form, got, scale):
    want, err = c.expected()
    if form == "whole":
        assert torch.equal(got, want.float().bfloat16())
    elif form == "swiglu":
        assert ((got.double() - want).abs() <= err + (want.abs() + err) * 2.0 ** -8 + 2.0 ** -133).all()
    else:
        by_block = lambda v: torch.nn.functional.pad(v, (0, blocks_of(c.n_out) * 128 - c.n_out)).view(c.P, -1, 128)
        top, e_top = by_block(want).abs().amax(2).clamp(min=SMALLEST), by_block(err).amax(2)
        assert ((scale.double() * 448 - top).abs() <= e_top + top * 2.0 ** -22).all()
        s = spread(scale, c.P, c.n_out, 1)
        assert ((got.double() * s - want).abs() <= err + (want.abs() + err) * (2.0 ** -4 + 2.0 ** -20) + s * 2.0 ** -10).all()


# 17 k-blocks and one of 16 numbers in a ring of six; 17 tiles of W (the last with 8 or 16 rows) by 16 to 30 of x for 74 pairs
@pytest.mark.parametrize("perm", [False, True], ids=["rows", "gathered"])
@pytest.mark.parametrize("counts", [[4000], [3001, 0, 257, 1100], [1, 2100, 1999]], ids=str)
@pytest.mark.parametrize("form", ["whole", "swiglu", "quantized"])
def test_pairs_walk_over_many_tiles(form, counts, perm):
    ctx = make_ctx(k=3)
    assert sum(counts) // len(counts) >= 1024
    c = Case(counts, 2192, 4104 if form == "whole" else 4128, True, form != "whole", perm, seed=21, whole=form == "whole", k=3)
    got, scale = c.run(ctx, quantize=form == "quantized")
    check(c, form, got, scale)
    again, scale_again = c.run(ctx, quantize=form == "quantized")
    assert torch.equal(got.view(torch.uint8), again.view(torch.uint8))
    assert scale is None or torch.equal(scale, scale_again)
    ctx.close()


def guarded(shape, dtype, size, fill):
    """A buffer of this shape between two stretches of 4096 bytes, all bytes `fill`; (buffer, the bytes outside it)."""
    n = size
    for s in shape:
        n *= s
    flat = torch.full((n + 8192,), fill, dtype=torch.uint8, device=DEV)
    return flat[4096: 4096 + n].view(dtype).view(shape), (flat[:4096], flat[4096 + n:])


@pytest.mark.parametrize("counts", [[1], [40, 0, 3], [300, 20, 129], [1500, 1100]], ids=str)
@pytest.mark.parametrize("form", ["bf16", "bf16 swiglu", "e4m3", "e4m3 swiglu", "quantized"])
@pytest.mark.parametrize("K", [144, 2064])
def test_nothing_outside_the_results_is_written(K, form, counts):
    e4m3, swiglu, quantize = form[0] != "b", form not in ("bf16", "e4m3"), form == "quantized"
    ctx = make_ctx(k=2)
    c = Case(counts, K, 352, e4m3, swiglu, True, seed=22, k=2)
    want, want_scale = c.run(ctx, quantize=quantize)
    # (the form is chosen by rows: three more than the slots have, as in Case.run)
    out, edges = guarded((c.P + 3, c.n_out), E4M3 if quantize else torch.bfloat16, 1 if quantize else 2, 0x5A)
    scale, scale_edges = guarded((c.P + 3, blocks_of(c.n_out)), torch.float32, 4, 0x5A)
    ctx.fb_expert_matmul(c.matrix(), c.x, c.xs, c.offsets, c.perm, c.P + 3, out, scale if quantize else None)
    torch.cuda.synchronize()
    assert ctx.fb_device_status() == 0
    assert torch.equal(out[: c.P].view(torch.uint8), want.view(torch.uint8))
    assert all((e == 0x5A).all() for e in (*edges, *scale_edges, out[c.P:].view(torch.uint8), scale[c.P:].view(torch.uint8)))
    if quantize:
        assert torch.equal(scale[: c.P], want_scale)
    else:
        assert (scale.view(torch.uint8) == 0x5A).all()
    ctx.close()
