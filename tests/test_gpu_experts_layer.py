"""The experts' side of a layer behind the router: dispatch index, exchange of weights, products and combination together."""
import dataclasses

import pytest
import torch

from paper_2608_14205_b200 import binding as B
from paper_2608_14205_b200 import experts as X
from paper_2608_14205_b200 import inputs as I
from paper_2608_14205_b200 import serving as S

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda", 0)


def small(name, e4m3, d, inter, **kw):
    return dataclasses.replace(I.WORKLOADS[name], d=d, inter=inter, expert_e4m3=e4m3, expert_bytes=0, alpha_ns=0, fs_per_byte=0,
                               global_ns=2**64 - 1, rank_ns=2**64 - 1, link_ns=2**64 - 1, **kw)


def values(x: X.SlotExperts):
    """64-bit matrices of every slot."""
    def of(w, scale, halves):
        w = w.double()
        if scale is None:
            return w
        parts, at = [], 0
        for rows in halves:
            n = -(-rows // 128)
            s = scale[:, at: at + n].double().repeat_interleave(128, 1)[:, :rows].repeat_interleave(128, 2)[:, :, : w.shape[2]]
            parts.append(s)
            at += n
        return w * torch.cat(parts, 1)
    return of(x.gate_up, x.gate_up_scale, [x.inter] * 2), of(x.down, x.down_scale, [x.d])


def reference(wl, x, buf, H, ids, w, placement, addend):
    """(sum over the chosen experts + addend in 64 bits, bound on the library's error), for the rows that the products read:
    H, or what fb_quantize_rows made of it.  Every rounding is counted: 32-bit sums of n products n * 2^-23 * sum |products|;
    SwiGLU of erring sums 1.1 |u| dg + |silu(g)| du + 1.1 dg du, its own arithmetic 2^-19; the hidden row 2^-8 (bf16), or 2^-4
    and 2^-10 of its block's scale (e4m3); a row 2^-8; the weighted sum k + 1 more 32-bit roundings; the result 2^-8."""
    gu, down = values(x)
    T, d, inter, e4m3 = H.shape[0], wl.d, wl.inter, x.e4m3
    Hd = H.double()
    if e4m3:
        Hd = buf.x[:T].double() * buf.x_scale[:T].double().repeat_interleave(128, 1)[:, :d]
    out, err, size = (torch.zeros(T, d, dtype=torch.float64, device=DEV) for _ in range(3))
    step = 2.0 ** -23
    for e in range(wl.E):
        t, j = (ids == e).nonzero(as_tuple=True)
        if t.numel() == 0:
            continue
        slot = int(placement[e])
        g, u = (Hd[t] @ gu[slot].t()).chunk(2, 1)
        dg, du = (Hd[t].abs() @ gu[slot].abs().t() * ((d + d // 128 + 8) * step)).chunk(2, 1)
        silu = g * torch.sigmoid(g)
        h = silu * u
        dh = 1.1 * u.abs() * dg + silu.abs() * du + 1.1 * dg * du + h.abs() * 2.0 ** -19
        if e4m3:
            blocks = torch.nn.functional.pad(h.abs() + dh, (0, -inter % 128)).view(len(t), -1, 128).amax(2, keepdim=True)
            tiny = (blocks / 448 * 2.0 ** -10).expand(-1, -1, 128).reshape(len(t), -1)[:, :inter]
            dh = dh + (h.abs() + dh) * (2.0 ** -4 + 2.0 ** -20) + tiny
        else:
            dh = dh + (h.abs() + dh) * 2.0 ** -8
        y = h @ down[slot].t()
        absolute = (h.abs() + dh) @ down[slot].abs().t()
        dy = dh @ down[slot].abs().t() + absolute * ((inter + inter // 128 + 8) * step)
        dy = dy + (y.abs() + dy) * 2.0 ** -8
        weight = w[t, j].double()[:, None]
        out.index_add_(0, t, y * weight)
        err.index_add_(0, t, dy * weight)
        size.index_add_(0, t, (y.abs() + dy) * weight)
    out, size = out + addend.double(), size + addend.double().abs()
    err = err + size * ((wl.k + 1) * 2.0 ** -24)
    return out, err + (out.abs() + err) * 2.0 ** -8


@pytest.mark.parametrize("name,e4m3,d,inter,T", [("tiny", False, 256, 96, 300), ("tiny", True, 256, 128, 300), ("qwen3", False, 512, 160, 1000),
                                                 ("dsv3", True, 512, 144, 700), ("dsv3", True, 512, 144, 1), ("qwen3", True, 256, 128, 8200)])
def test_layer_with_moved_experts(name, e4m3, d, inter, T):
    wl = small(name, e4m3, d, inter)
    li = I.make_layer(wl, 0, 0, T=T)
    loop = S.ServingLoop(wl, T + 5)
    x = S.random_experts(wl, 0, 3, DEV)
    sb = li.select_bias.to(DEV) if li.select_bias is not None else None
    router = B.make_router(li.W.to(DEV), None, sb)
    H = li.H.to(DEV)
    r = loop.layer_step(0, router, li.h_prev.to(DEV), H, S.make_budget_for(wl, T))
    addend = torch.randn(T, d, device=DEV).bfloat16()
    before = x.images.clone()
    got = loop.experts_step(r, H, x, addend).clone()
    torch.cuda.synchronize()
    assert loop.ctx.fb_device_status() == 0
    if name != "tiny" and T > 1:                          # (two experts a rank: the plan may find nothing to swap)
        assert int(r["out"]["n_swaps"].item()) > 0
        assert not torch.equal(before, x.images), "weights were moved"
    # every expert's image sits in the slot of its new placement
    for e in range(wl.E):
        assert torch.equal(x.images[r["pi_new"][e]], before[r["pi_old"][e]])
    ids, w = r["out"]["ids"][: T * wl.k].view(T, wl.k), r["out"]["w"][: T * wl.k].view(T, wl.k)
    want, err = reference(wl, x, loop._x, H, ids, w, r["pi_new"], addend)
    assert ((got.double() - want).abs() <= err).all()
    # (the bound is a worst case; independent roundings come out far below it)
    rel = ((got.double() - want).square().sum() / want.square().sum()).sqrt().item()
    assert rel < (2.0 ** -4 if e4m3 else 2.0 ** -6)
    loop.close()


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_the_output_does_not_depend_on_the_placement(e4m3):
    # a row's sums have one order whatever its position: same bits before and after an exchange of weights
    wl = small("qwen3", e4m3, 512, 128)
    T = 1500
    li = I.make_layer(wl, 0, 0, T=T)
    H = li.H.to(DEV)
    router = B.make_router(li.W.to(DEV), None, None)
    outs = []
    for cap in (0, 6):
        loop = S.ServingLoop(dataclasses.replace(wl, max_swaps=6), T)
        x = S.random_experts(wl, 0, 5, DEV)
        r = loop.layer_step(0, router, li.h_prev.to(DEV), H, S.make_budget_for(wl, T, max_swaps=cap))
        outs.append(loop.experts_step(r, H, x).clone())
        torch.cuda.synchronize()
        assert (int(r["out"]["n_swaps"].item()) > 0) == (cap > 0)
        loop.close()
    assert torch.equal(outs[0], outs[1])


def test_a_rank_of_the_placement_by_itself():
    # expert-parallel: each rank's slots from its own rows, combined afterwards, give the layer's bits
    wl = small("tiny", False, 256, 96)
    T, k = 200, wl.k
    li = I.make_layer(wl, 0, 0, T=T)
    loop = S.ServingLoop(wl, T)
    x = S.random_experts(wl, 0, 7, DEV)
    H = li.H.to(DEV)
    r = loop.layer_step(0, B.make_router(li.W.to(DEV), None, None), li.h_prev.to(DEV), H, S.make_budget_for(wl, T))
    want = loop.experts_step(r, H, x).clone()
    o, ctx, m = r["out"], loop.ctx, wl.E // wl.R
    rank_offsets = o["rank_offsets"].tolist()
    rows = torch.zeros(T * k, wl.d, dtype=torch.bfloat16, device=DEV)
    for rank in range(wl.R):
        lo, hi = rank_offsets[rank], rank_offsets[rank + 1]
        if hi == lo:
            continue
        mine = slice(rank * m, rank * m + m)
        up = B.make_expert_matrix(x.gate_up[mine], None, B.FB_ACT_SWIGLU)
        down = B.make_expert_matrix(x.down[mine])
        offsets = o["slot_offsets"][rank * m: rank * m + m + 1]
        hidden = torch.empty(hi - lo, wl.inter, dtype=torch.bfloat16, device=DEV)
        y = torch.empty(hi - lo, wl.d, dtype=torch.bfloat16, device=DEV)
        ctx.fb_expert_matmul(up, H, None, offsets, o["perm"], hi - lo, hidden)
        ctx.fb_expert_matmul(down, hidden, None, offsets, None, hi - lo, y)
        rows[lo:hi] = y
    out = torch.empty(T, wl.d, dtype=torch.bfloat16, device=DEV)
    ctx.fb_combine(rows, o["w"], o["inv_perm"], T, wl.d, None, out)
    torch.cuda.synchronize()
    assert ctx.fb_device_status() == 0 and torch.equal(out, want)
    loop.close()


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_captured_chain_follows_new_tokens(e4m3):
    # route, quantise, up, down, combine in one graph; replayed on other hidden states, whose routing differs
    wl = small("qwen3", e4m3, 512, 128)
    T, k = 700, wl.k
    layers = [I.make_layer(wl, l, 0, T=T) for l in range(2)]
    ctx = B.Context(T, wl.d, wl.E, k, wl.R, wl.gate, wl.n_group, wl.topk_group, wl.renorm, wl.route_scale)
    x = S.random_experts(wl, 0, 9, DEV)
    buf = X.ExpertBuffers(x, T, k)
    router = B.make_router(layers[0].W.to(DEV), None, None)
    pi = layers[0].expert_to_slot.to(DEV)
    H = layers[0].H.to(DEV)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)
    ids, w, offsets, ranks, perm, inv, load = i32(T * k), torch.zeros(T * k, device=DEV), i32(wl.E + 1), i32(wl.R + 1), i32(T * k), i32(T * k), i32(wl.R)

    def chain():
        ctx.fb_route_dispatch(router, H, T, pi, ids, w, offsets, ranks, perm, inv, load)
        return X.run_experts(ctx, x, buf, H, T, k, w, offsets, perm, inv)

    chain()
    torch.cuda.synchronize()
    first_ids = ids.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = chain()
    H.copy_(layers[1].H.to(DEV))
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    got, got_ids = out.clone(), ids.clone()
    assert not torch.equal(got_ids, first_ids)
    out.zero_()
    chain()
    torch.cuda.synchronize()
    assert torch.equal(got_ids, ids) and torch.equal(got, out) and got.abs().sum() > 0
    assert ctx.fb_device_status() == 0
    ctx.close()


@pytest.mark.parametrize("name", ["qwen3", "dsv3"])
def test_serving_loop_with_experts_from_the_command_line(name, monkeypatch, capsys):
    import json
    monkeypatch.setitem(I.WORKLOADS, name, small(name, I.WORKLOADS[name].expert_e4m3, 512, 128))
    monkeypatch.setattr("sys.argv", ["serving", "--workload", name, "--steps", "2", "--layers", "2", "--tokens", "600", "--experts"])
    S.main()
    report = json.loads(capsys.readouterr().out)
    assert report["device_status"] == 0 and len(report["records"]) == 4
    assert all(0 < rec["out_rms"] < 100 for rec in report["records"])
