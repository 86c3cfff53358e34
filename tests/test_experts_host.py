"""Host side of the experts' products: marshalling of matrices, refusals that need no device, images' layout."""
import ctypes

import pytest
import torch

from paper_2608_14205_b200 import binding as B
from paper_2608_14205_b200 import experts as X


def test_struct_matches_the_header():
    # 5 x i32, padding, pointer, u64, pointer, u64
    assert ctypes.sizeof(B.FbExpertMatrix) == 56
    assert B.FbExpertMatrix.w.offset == 24 and B.FbExpertMatrix.slot_bytes.offset == 32
    assert B.FbExpertMatrix.scale.offset == 40 and B.FbExpertMatrix.scale_slot.offset == 48


def test_matrix_of_slots_that_lie_apart():
    images = torch.zeros(4, 10000, dtype=torch.uint8)
    w = images.view(-1).view(torch.bfloat16).as_strided((4, 32, 64), (5000, 64, 1))
    m = B.make_expert_matrix(w, None, B.FB_ACT_SWIGLU)
    assert (m.dtype, m.act, m.n_slots, m.n, m.K, m.slot_bytes) == (B.FB_DTYPE_BF16, 1, 4, 32, 64, 10000)
    assert m.w == images.data_ptr() and not m.scale
    q = torch.zeros(2, 264, 272).to(torch.float8_e4m3fn)
    m = B.make_expert_matrix(q, torch.ones(2, 3, 3))
    assert m.dtype == B.FB_DTYPE_E4M3 and m.scale_slot == 9 and m.slot_bytes == 264 * 272
    m = B.make_expert_matrix(torch.zeros(2, 288, 272).to(torch.float8_e4m3fn), torch.ones(2, 4, 3), B.FB_ACT_SWIGLU)
    assert m.scale_slot == 12


def test_matrices_that_are_refused():
    q = torch.zeros(2, 264, 272).to(torch.float8_e4m3fn)
    for w, scale in ((q, torch.ones(2, 3, 2)), (q, torch.ones(2, 3, 3).double()), (q.transpose(1, 2), None), (q.float(), None),
                     (torch.zeros(264, 272, dtype=torch.bfloat16), None)):
        with pytest.raises(AssertionError):
            B.make_expert_matrix(w, scale)


def test_calls_without_a_context_are_refused():
    L = B.lib()
    m = B.make_expert_matrix(torch.zeros(1, 8, 8, dtype=torch.bfloat16))
    assert L.fb_expert_matmul(None, ctypes.byref(m), None, None, 0, None, None, 0, None, None, None) == B.FB_ERR_INVALID_ARG
    assert L.fb_quantize_rows(None, None, 0, 16, None, None, None) == B.FB_ERR_INVALID_ARG
    assert L.fb_combine(None, None, None, None, 0, 8, None, None, None) == B.FB_ERR_INVALID_ARG


@pytest.mark.parametrize("n,K", [(128, 128), (16, 48), (300, 200)])
def test_quantized_matrix(n, K):
    g = torch.Generator().manual_seed(n)
    w = torch.randn(n, K, generator=g)
    w[: min(n, 128), : min(K, 128)] = 0.0
    q, scale = X.quantize_matrix(w)
    s = scale.double().repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :K]
    assert q.shape == (n, K) and scale.shape == (-(-n // 128), -(-K // 128))
    assert not q.float().isnan().any()
    assert ((q.double() * s - w.double()).abs() <= w.double().abs() * (2.0 ** -4 + 2.0 ** -21) + s * 2.0 ** -10).all()
