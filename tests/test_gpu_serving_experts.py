"""ServingLoop.experts_step on a stream of its own, and with experts of two sizes, against the same steps on the current stream."""
import pytest
import torch

from paper_2608_14205_b200 import binding as B
from paper_2608_14205_b200 import inputs as I
from paper_2608_14205_b200 import serving as S

from .test_gpu_experts_layer import DEV, small

pytestmark = pytest.mark.gpu


def steps(wl, T, experts, stream_of, out_of):
    """Five steps of two layers with other hidden states each; the layers' outputs."""
    loop, outs = S.ServingLoop(wl, T), []
    lis = [[I.make_layer(wl, l, s, T=T) for l in range(2)] for s in range(3)]
    inputs = [[(li.W.to(DEV), li.h_prev.to(DEV), li.H.to(DEV), li.select_bias) for li in step] for step in lis]
    torch.cuda.synchronize()
    for s in range(5):
        for l in range(2):
            W, h_prev, H, bias = inputs[s % 3][l]
            router = B.make_router(W, None, bias.to(DEV) if bias is not None else None)
            torch.cuda._sleep(200_000)                       # the step's index is not there yet when experts_step is called
            r = loop.layer_step(l, router, h_prev, H, S.make_budget_for(wl, T))
            outs.append(out_of(loop.experts_step(r, H, experts[l], stream=stream_of())))
    torch.cuda.synchronize()
    assert loop.ctx.fb_device_status() == 0
    loop.close()
    return outs


@pytest.mark.parametrize("given", ["stream", "handle", "current"])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_a_stream_of_its_own(e4m3, given):
    wl, T = small("qwen3", e4m3, 512, 128), 900
    make = lambda: [S.random_experts(wl, l, 3, DEV) for l in range(2)]
    want = steps(wl, T, make(), lambda: None, lambda o: o.clone())
    side = torch.cuda.Stream()
    stream_of = {"stream": lambda: side, "handle": lambda: side.cuda_stream, "current": torch.cuda.current_stream}[given]
    got = steps(wl, T, make(), stream_of, lambda o: o.clone())      # (copied on the current stream)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert not torch.equal(want[0], want[2])


def test_a_captured_step_outlives_experts_of_another_size():
    wl, T = small("qwen3", False, 512, 128), 400
    wide = small("qwen3", True, 512, 256)
    loop, li = S.ServingLoop(wl, T), I.make_layer(wl, 0, 0, T=T)
    x, y = S.random_experts(wl, 0, 3, DEV), S.random_experts(wide, 0, 4, DEV)
    router, h_prev, H = B.make_router(li.W.to(DEV), None, None), li.h_prev.to(DEV), li.H.to(DEV)
    budget = S.make_budget_for(wl, T, max_swaps=0)          # nothing moves: the graph can be replayed
    step = lambda experts: loop.experts_step(loop.layer_step(0, router, h_prev, H, budget), H, experts)
    want = step(x).clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(x)
    step(y)                                                  # buffers of its own
    others = [torch.full((T * wl.k, wl.d), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(8)]     # takes what is free
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and all((o == 3.0).all() for o in others)
    assert loop.ctx.fb_device_status() == 0
    loop.close()
