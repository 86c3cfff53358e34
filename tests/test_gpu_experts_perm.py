"""Entries of perm that are no rows of x: reported whatever k is, row 0 read in their place, the other rows as ever."""
import pytest
import torch

from paper_2608_14205_b200 import binding as B

from .test_gpu_experts import Case, DEV, make_ctx

pytestmark = pytest.mark.gpu


# -1 .. -(k - 1) would be row 0 if the quotient were tested; -k is the first whose quotient is negative
@pytest.mark.parametrize("entry", [-1, -7, -8, -2**31, 8 * 60, 2**31 - 1])
@pytest.mark.parametrize("swiglu", [False, True], ids=["none", "swiglu"])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_an_entry_outside_x_is_reported(e4m3, swiglu, entry):
    k = 8
    ctx = make_ctx(k=k)
    c = Case([200, 0, 250, 30], 128, 64, e4m3, swiglu, True, seed=11, whole=True, k=k)
    assert c.x_rows == 60
    clean, _ = c.run(ctx)
    clean = clean.clone()
    c.perm[205] = entry
    out = torch.full((480, c.n_out), 7.0, dtype=torch.bfloat16, device=DEV)
    ctx.fb_expert_matmul(c.matrix(), c.x, c.xs, c.offsets, c.perm, 480, out)
    torch.cuda.synchronize()
    assert ctx.fb_device_status() == B.FB_ERR_RANGE
    keep = torch.ones(480, dtype=torch.bool, device=DEV)
    keep[205] = False
    assert torch.equal(out[keep], clean[keep])
    c.perm[205] = 0
    row0, _ = c.run(ctx)
    assert torch.equal(out[205], row0[205])
    ctx.close()
