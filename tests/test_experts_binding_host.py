"""What the binding refuses before the library is called: tensors of another type or with too few elements, whose pointers alone
the library could not tell from good ones.  A stand-in takes the library's place: nothing is launched."""
import pytest
import torch

from paper_2608_14205_b200 import binding as B

E4M3 = torch.float8_e4m3fn
bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
f8 = lambda *s: torch.zeros(*s).to(E4M3)
f32 = lambda *s: torch.zeros(*s)
i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)


@pytest.fixture
def ctx(monkeypatch):
    """A context whose calls reach a list instead of the library."""
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.append(name) or 0

    monkeypatch.setattr(B, "lib", Library)
    monkeypatch.setattr(B, "_stream", lambda stream: None)
    monkeypatch.setattr(B, "_lib", None)
    c = B.Context.__new__(B.Context)
    c._h, c.device, c._k, c.calls = None, 0, 2, calls
    return c


def product(e4m3, quantize=False):
    """Good arguments: 8 rows of 4 tokens, 2 slots, K = 144."""
    act = B.FB_ACT_SWIGLU if quantize else B.FB_ACT_NONE
    m = B.make_expert_matrix(f8(2, 320, 144), f32(2, 4 if quantize else 3, 2), act) if e4m3 else B.make_expert_matrix(bf(2, 320, 144))
    return dict(matrix=m, x=f8(4, 144) if e4m3 else bf(4, 144), x_scale=f32(4, 2) if e4m3 else None, slot_offsets=i32(3), perm=i32(8), rows=8,
                out=f8(8, 160) if quantize else bf(8, 320), out_scale=f32(8, 2) if quantize else None)


FORMS = [(False, False), (True, False), (True, True)]      # e4m3, quantised results
has = lambda name, e4m3, quantize: (e4m3 or name != "x_scale") and (quantize or name != "out_scale")


@pytest.mark.parametrize("e4m3,quantize", FORMS)
def test_good_products_reach_the_library(ctx, e4m3, quantize):
    a = product(e4m3, quantize)
    ctx.fb_expert_matmul(**a)
    ctx.fb_expert_matmul(**{**a, "slot_offsets": a["slot_offsets"].view(torch.uint32)})
    ctx.fb_expert_matmul(**{**a, "rows": 7})                 # buffers that hold more than the call's rows
    assert ctx.calls == ["fb_expert_matmul"] * 3


WRONG_TYPE = [("x", torch.float32), ("x", torch.float16), ("x", "other"), ("slot_offsets", torch.int64), ("perm", torch.int64),
              ("out", torch.float16), ("out", torch.float32), ("x_scale", torch.float64), ("x_scale", torch.bfloat16),
              ("out_scale", torch.float64), ("out_scale", torch.bfloat16)]


@pytest.mark.parametrize("name,dtype,e4m3,quantize", [(n, t, *form) for form in FORMS for n, t in WRONG_TYPE if has(n, *form)], ids=str)
def test_products_with_tensors_of_another_type(ctx, name, dtype, e4m3, quantize):
    a = product(e4m3, quantize)
    if dtype == "other":
        dtype = torch.bfloat16 if e4m3 else E4M3
    a[name] = a[name].to(torch.float32).to(dtype)
    with pytest.raises(AssertionError):
        ctx.fb_expert_matmul(**a)
    assert ctx.calls == []


@pytest.mark.parametrize("name,e4m3,quantize", [(n, *form) for form in FORMS for n in ("out", "out_scale", "x_scale", "slot_offsets") if has(n, *form)])
def test_products_with_too_few_elements(ctx, name, e4m3, quantize):
    a = product(e4m3, quantize)
    a[name] = a[name].reshape(-1)[:-1]
    with pytest.raises(B.FbError) as e:
        ctx.fb_expert_matmul(**a)
    assert e.value.status == B.FB_ERR_INVALID_ARG and ctx.calls == []


def sum_of_rows():
    """Good arguments: 4 tokens, k = 2."""
    return dict(rows=bf(8, 64), w=f32(4, 2), inv_perm=i32(8), T=4, n=64, addend=bf(4, 64), out=bf(4, 64))


def test_good_combinations_reach_the_library(ctx):
    ctx.fb_combine(**sum_of_rows())
    ctx.fb_combine(**{**sum_of_rows(), "addend": None, "T": 3})
    assert ctx.calls == ["fb_combine"] * 2


@pytest.mark.parametrize("name,dtype", [("rows", torch.float16), ("rows", torch.float32), ("w", torch.bfloat16), ("w", torch.float64),
                                        ("inv_perm", torch.int64), ("addend", torch.float16), ("out", torch.float16), ("out", torch.float32)], ids=str)
def test_combinations_with_tensors_of_another_type(ctx, name, dtype):
    a = sum_of_rows()
    a[name] = a[name].to(dtype)
    with pytest.raises(AssertionError):
        ctx.fb_combine(**a)
    assert ctx.calls == []


@pytest.mark.parametrize("name", ["rows", "w", "inv_perm", "addend", "out"])
def test_combinations_with_too_few_elements(ctx, name):
    a = sum_of_rows()
    a[name] = a[name].reshape(-1)[:-1]
    with pytest.raises(B.FbError) as e:
        ctx.fb_combine(**a)
    assert e.value.status == B.FB_ERR_INVALID_ARG and ctx.calls == []


def rows_to_quantize():
    """Good arguments: 4 rows of 144 numbers."""
    return dict(x=bf(4, 144), rows=4, n=144, q=f8(4, 144), scale=f32(4, 2))


def test_good_quantisations_reach_the_library(ctx):
    ctx.fb_quantize_rows(**rows_to_quantize())
    ctx.fb_quantize_rows(**{**rows_to_quantize(), "rows": 3})
    ctx.fb_quantize_rows(**{**rows_to_quantize(), "rows": 2**40, "n": 7168})      # the library's own refusal
    assert ctx.calls == ["fb_quantize_rows"] * 3


@pytest.mark.parametrize("name,dtype", [("x", torch.float16), ("x", torch.float32), ("q", torch.bfloat16), ("q", torch.float8_e5m2),
                                        ("scale", torch.bfloat16)], ids=str)
def test_quantisations_with_tensors_of_another_type(ctx, name, dtype):
    a = rows_to_quantize()
    a[name] = a[name].to(torch.float32).to(dtype)
    with pytest.raises(AssertionError):
        ctx.fb_quantize_rows(**a)
    assert ctx.calls == []


@pytest.mark.parametrize("name", ["x", "q", "scale"])
def test_quantisations_with_too_few_elements(ctx, name):
    a = rows_to_quantize()
    a[name] = a[name].reshape(-1)[:-1]
    with pytest.raises(B.FbError) as e:
        ctx.fb_quantize_rows(**a)
    assert e.value.status == B.FB_ERR_INVALID_ARG and ctx.calls == []
