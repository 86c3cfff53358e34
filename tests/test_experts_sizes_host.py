"""Sizes whose rounding up would pass 32 bits are refused before anything is computed from them (no device is needed: a context
that is all zeros is never looked at)."""
import ctypes

import pytest

from paper_2608_14205_b200 import binding as B

BLANK = ctypes.create_string_buffer(1 << 20)
CTX = ctypes.addressof(BLANK)
SOME = 1 << 20                                  # an aligned address that is not read
MOST = 2**31 - 1024


def matmul(dtype, n, K, rows, x_rows, act=B.FB_ACT_NONE, perm=None):
    e4m3 = dtype == B.FB_DTYPE_E4M3
    m = B.FbExpertMatrix(dtype, act, 1, n, K, SOME, 0, SOME if e4m3 else None, 0)
    return B.lib().fb_expert_matmul(CTX, ctypes.byref(m), SOME, SOME if e4m3 else None, x_rows, SOME, perm, rows, SOME, None, None)


@pytest.mark.parametrize("dtype", [B.FB_DTYPE_BF16, B.FB_DTYPE_E4M3], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("act", [B.FB_ACT_NONE, B.FB_ACT_SWIGLU], ids=["none", "swiglu"])
def test_products(dtype, act):
    for n, K, rows, x_rows, perm in ((2**31 - 32, 16, 1, 1, None), (MOST + 32, 16, 1, 1, None), (32, 16, 2**31 - 1, 2**31 - 1, None),
                                     (32, 16, MOST + 1, MOST + 1, None), (32, 16, MOST + 1, 2**30, SOME), (32, 16, 1, 2**31 - 1, None)):
        assert matmul(dtype, n, K, rows, x_rows, act, perm) == B.FB_ERR_UNSUPPORTED_SHAPE, (n, K, rows, x_rows)


@pytest.mark.parametrize("K", [2**31 - 16, 2**31 - 128, MOST + 16])
def test_long_rows_of_e4m3(K):
    assert matmul(B.FB_DTYPE_E4M3, 32, K, 1, 1) == B.FB_ERR_UNSUPPORTED_SHAPE


@pytest.mark.parametrize("n", [2**31 - 16, MOST + 16])
def test_quantisation_and_combination(n):
    assert B.lib().fb_quantize_rows(CTX, SOME, 1, n, SOME, SOME, None) == B.FB_ERR_UNSUPPORTED_SHAPE
    assert B.lib().fb_combine(CTX, SOME, SOME, SOME, 1, n, None, SOME, None) == B.FB_ERR_UNSUPPORTED_SHAPE
