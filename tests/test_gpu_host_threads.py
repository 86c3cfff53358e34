"""A call of the library may be the first CUDA call of its host thread (a server's worker), which has no context yet."""
import threading

import pytest
import torch

from paper_2608_14205_b200 import binding as B
from paper_2608_14205_b200 import inputs as I

from .test_gpu_experts import Case, DEV, make_ctx

pytestmark = pytest.mark.gpu


def in_a_fresh_thread(call):
    failed = []

    def run():
        try:
            call()
        except BaseException as e:
            failed.append(e)

    t = threading.Thread(target=run)
    t.start()
    t.join()
    torch.cuda.synchronize()
    if failed:
        raise failed[0]


@pytest.mark.parametrize("perm", [False, True], ids=["rows", "gathered"])
@pytest.mark.parametrize("form", ["bf16", "e4m3", "bf16 swiglu", "e4m3 swiglu"])
def test_a_product_is_the_first_call(form, perm):
    ctx = make_ctx()
    c = Case([40, 3, 200], 256, 256, form[0] == "e", "swiglu" in form, perm, seed=31)
    want, _ = c.run(ctx, extra=0)
    out = torch.zeros_like(want)
    in_a_fresh_thread(lambda: ctx.fb_expert_matmul(c.matrix(), c.x, c.xs, c.offsets, c.perm, c.P, out))
    assert ctx.fb_device_status() == 0 and torch.equal(out, want)
    ctx.close()


def test_quantisation_and_combination_are_the_first_calls():
    ctx = make_ctx(k=2)
    x = torch.randn(50, 256, device=DEV).bfloat16()
    q, s = torch.empty(50, 256, device=DEV).to(torch.float8_e4m3fn), torch.empty(50, 2, device=DEV)
    want_q, want_s = torch.empty_like(q), torch.empty_like(s)
    ctx.fb_quantize_rows(x, 50, 256, want_q, want_s)
    in_a_fresh_thread(lambda: ctx.fb_quantize_rows(x, 50, 256, q, s))
    assert torch.equal(q.view(torch.uint8), want_q.view(torch.uint8)) and torch.equal(s, want_s)
    w, inv = torch.rand(25, 2, device=DEV), torch.randperm(50, device=DEV).int()
    out, want = torch.empty(25, 256, dtype=torch.bfloat16, device=DEV), torch.empty(25, 256, dtype=torch.bfloat16, device=DEV)
    ctx.fb_combine(x, w, inv, 25, 256, None, want)
    in_a_fresh_thread(lambda: ctx.fb_combine(x, w, inv, 25, 256, None, out))
    assert torch.equal(out, want)
    ctx.close()


@pytest.mark.parametrize("call", ["route", "predict", "static"])
def test_a_router_call_on_new_buffers_is_the_first_call(call):
    wl, T = I.WORKLOADS["tiny"], 300
    li = I.make_layer(wl, 0, 0, T=T)
    cfg = (T, wl.d, wl.E, wl.k, wl.R, wl.gate, wl.n_group, wl.topk_group, wl.renorm, wl.route_scale)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)
    pi = li.expert_to_slot.to(DEV)

    def run(ctx, thread):
        router, H = B.make_router(li.W.to(DEV).clone(), None, None), li.H.to(DEV).clone()
        outs = dict(ids=i32(T * wl.k), w=torch.zeros(T * wl.k, device=DEV), so=i32(wl.E + 1), ro=i32(wl.R + 1), perm=i32(T * wl.k),
                    inv=i32(T * wl.k), load=i32(wl.R))
        counts = i32(wl.E)

        def make():
            if call == "route":
                ctx.fb_route_dispatch(router, H, T, pi, *outs.values())
            elif call == "predict":
                ctx.fb_predict_load(router, H, T, counts)
            else:
                B.fb_predict_load_static(ctx.cfg, 0, router, H, T, counts)

        torch.cuda.synchronize()
        in_a_fresh_thread(make) if thread else make()
        torch.cuda.synchronize()
        assert ctx.fb_device_status() == 0
        return [*outs.values(), counts]

    results = []
    for thread in (True, False):
        ctx = B.Context(*cfg)                            # (maps of buffers that it has seen are kept: a new context has none)
        results.append(run(ctx, thread))
        ctx.close()
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert any(t.abs().sum() > 0 for t in results[0])
