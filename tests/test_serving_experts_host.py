"""ServingLoop.experts_step: what it refuses, which buffers it keeps and how its stream is ordered, with stand-ins for the
loop's parts and for torch's device calls: nothing is launched."""
import types

import pytest
import torch

from paper_2608_14205_b200 import experts as X
from paper_2608_14205_b200 import serving as S

T_MAX, D, K = 16, 32, 2


class Experts:
    """Images of which only the sizes are looked at."""

    def __init__(self, inter=16, e4m3=False, d=D, E=4, device="cpu"):
        self.d, self.E, self.inter, self.e4m3, self.dtype = d, E, inter, e4m3, torch.bfloat16
        self.images = torch.zeros(1, device=device)
        self.swapped = 0

    def apply_swaps(self, *a, stream=None):
        self.swapped += 1


class Buffers:
    def __init__(self, experts, tokens, k):
        self.size = (experts.inter, experts.e4m3, tokens, k)


@pytest.fixture
def loop(monkeypatch):
    """A loop of one layer; loop.ran lists the calls of run_experts as (buffers, H, T)."""
    ran = []
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(S.X, "ExpertBuffers", Buffers)
    monkeypatch.setattr(S.X, "run_experts", lambda ctx, experts, buf, H, T, *a: ran.append((buf, H, T)) or H)
    l = S.ServingLoop.__new__(S.ServingLoop)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)
    l.wl, l.T_max, l.device, l.dev = types.SimpleNamespace(d=D, E=4, k=K), T_MAX, 0, torch.device("cpu")
    l.ctx = types.SimpleNamespace(fb_layer_step=lambda *a: None)
    l.out = {name: i32(8) for name in ("counts", "swaps", "n_swaps", "load_before", "load_after", "ids", "w", "slot_offsets",
                                       "rank_offsets", "perm", "inv_perm", "rank_load")}
    l.placement, l._spare, l._q, l._x, l._buffers = {}, i32(4), None, None, {}
    l.ran = ran
    return l


def rows(T):
    return torch.zeros(T, D, dtype=torch.bfloat16)


@pytest.mark.parametrize("tokens", [1, 7, 9, T_MAX, T_MAX + 1])
def test_hidden_states_of_another_batch_are_refused(loop, tokens):
    x = Experts()
    r = loop.layer_step(0, None, rows(8), rows(8), None)
    with pytest.raises(AssertionError):
        loop.experts_step(r, rows(tokens), x)
    assert x.swapped == 0 and loop.ran == []
    loop.experts_step(r, rows(8), x)
    assert x.swapped == 1 and [t for _, _, t in loop.ran] == [8]


def test_a_step_that_a_later_one_has_overwritten_is_refused(loop):
    x = Experts()
    first = loop.layer_step(0, None, rows(8), rows(8), None)
    second = loop.layer_step(1, None, rows(8), rows(8), None)
    with pytest.raises(AssertionError):
        loop.experts_step(first, rows(8), x)
    assert x.swapped == 0 and loop.ran == []
    loop.experts_step(second, rows(8), x)
    assert x.swapped == 1


def test_buffers_stay_when_experts_of_another_size_are_used(loop):
    # work on them may be under way on any stream, or captured in a graph that will be replayed
    narrow, wide = Experts(16), Experts(64, e4m3=True)
    for x in (narrow, wide, narrow, Experts(16), wide):
        loop.experts_step(loop.layer_step(0, None, rows(8), rows(8), None), rows(8), x)
        assert loop._x is loop.ran[-1][0]
    a, b, c, d, e = (buf for buf, _, _ in loop.ran)
    assert a is c is d and b is e and a.size == (16, False, T_MAX, K) and b.size == (64, True, T_MAX, K)


class Stream:
    """Notes in `log` what waits for what."""

    def __init__(self, name, handle, log):
        self.name, self.cuda_stream, self.log = name, handle, log

    def wait_stream(self, other):
        self.log.append(f"{self.name} waits for {other.name}")


@pytest.mark.parametrize("given", ["none", "current", "side", "side by handle"])
@pytest.mark.parametrize("fails", [False, True], ids=["runs", "fails"])
def test_a_stream_begins_behind_the_current_one_which_goes_on_behind_it(loop, monkeypatch, given, fails):
    # layer_step writes index and plan on the current stream, the next one overwrites them there
    log = []
    current, side = Stream("current", 7, log), Stream("side", 9, log)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: current)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: {7: current, 9: side}[handle])
    x = Experts()
    x.apply_swaps = lambda *a, stream=None: log.append(("swaps", stream))

    def run(ctx, experts, buf, H, T, *a):
        log.append(("products", a[-1]))
        if fails:
            raise RuntimeError("refused")

    monkeypatch.setattr(S.X, "run_experts", run)
    stream = {"none": None, "current": current, "side": side, "side by handle": 9}[given]
    r = loop.layer_step(0, None, rows(8), rows(8), None)
    if fails:
        with pytest.raises(RuntimeError):
            loop.experts_step(r, rows(8), x, stream=stream)
    else:
        loop.experts_step(r, rows(8), x, stream=stream)
    work = [("swaps", stream), ("products", stream)]
    assert log == (["side waits for current", *work, "current waits for side"] if given.startswith("side") else work)


@pytest.mark.parametrize("other", [dict(d=16), dict(d=64), dict(E=3), dict(E=5), dict(device="meta")], ids=str)
def test_images_of_another_model_or_device_are_refused(loop, other):
    x = Experts(e4m3=True, **other)
    r = loop.layer_step(0, None, rows(8), rows(8), None)
    with pytest.raises(AssertionError):
        loop.experts_step(r, rows(8), x)
    assert x.swapped == 0 and loop.ran == []


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("d", [D - 16, D + 16])
def test_rows_of_another_length_are_refused(e4m3, d):
    x = X.SlotExperts.__new__(X.SlotExperts)
    x.d, x.e4m3, x.up_matrix, x.down_matrix = d, e4m3, types.SimpleNamespace(K=d), None
    made = []
    ctx = types.SimpleNamespace(**{name: lambda *a, stream=None, name=name: made.append(name) for name in ("fb_quantize_rows", "fb_expert_matmul", "fb_combine")})
    buf = types.SimpleNamespace(out=rows(8), x=rows(8), x_scale=rows(8), hidden=rows(16), hidden_scale=rows(16), rows=rows(16))
    with pytest.raises(AssertionError):
        X.run_experts(ctx, x, buf, rows(8), 8, K, None, None, None, None)
    assert made == []


@pytest.mark.parametrize("wrong", ["H float16", "H columns", "H strided", "addend rows", "addend float32", "addend strided"])
def test_what_is_refused_moves_no_weights(loop, wrong):
    # a refusal behind the swaps would leave them applied, and the call that follows would apply them again
    x = Experts()
    r = loop.layer_step(0, None, rows(8), rows(8), None)
    H, addend = rows(8), rows(8)
    strided = torch.zeros(8, 2 * D, dtype=torch.bfloat16)[:, :D]
    if wrong[0] == "H":
        H = {"H float16": H.half(), "H columns": rows(8)[:, :16].contiguous(), "H strided": strided}[wrong]
    else:
        addend = {"addend rows": rows(7), "addend float32": addend.float(), "addend strided": strided}[wrong]
    with pytest.raises(AssertionError):
        loop.experts_step(r, H, x, addend)
    assert x.swapped == 0 and loop.ran == []
    loop.experts_step(r, rows(8), x, rows(8))
    assert x.swapped == 1
