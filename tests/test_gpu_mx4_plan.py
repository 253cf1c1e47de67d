"""Layer and block plans whose expert weights are in microscaled 4 bits."""
import numpy as np
import pytest
import torch

import oracle.moe as om
import paper_2601_14327_amd as laep
from _gpu import case, dev, host
from oracle import mx4
from oracle.numerics import round_bf16

BF16, F32 = torch.bfloat16, torch.float32


def _weights(g, E, d, f):
    gu = torch.empty((E, 2 * f, d), device="cuda").normal_(0, d ** -0.5, generator=g).to(BF16)
    dn = torch.empty((E, d, f), device="cuda").normal_(0, f ** -0.5, generator=g).to(BF16)
    return laep.moe_mx4_quantize(gu), laep.moe_mx4_quantize(dn)


def _values(w):
    return laep.moe_mx4_dequantize(*w)


@pytest.mark.gpu
@pytest.mark.parametrize("act", [4, 16])
@pytest.mark.parametrize("T,d,E,k,f,beta", [(1, 128, 8, 2, 64, None), (33, 256, 8, 1, 192, None),
                                            (700, 192, 16, 4, 128, None), (400, 128, 16, 2, 64, 0.2)])
def test_layer(T, d, E, k, f, beta, act):
    case(f"mx4 layer plan T={T} d={d} E={E} k={k} f={f} prune={beta} act={act}")
    g = torch.Generator(device="cuda").manual_seed(T + d)
    x = torch.empty((T, d), device="cuda").normal_(generator=g).to(BF16)
    wr = torch.empty((E, d), device="cuda").normal_(0, 0.1, generator=g).to(BF16)
    gu, dn = _weights(g, E, d, f)
    plan = laep.MoELayerPlan(T, d, E, k, f, mx4_act=act)
    out = plan.forward(x, wr, gu, dn, prune_beta=beta)
    # the calls one by one
    y, _ = laep.moe_grouped_ffn_fwd_mx4(x, gu, dn, plan.offsets, row_src=plan.row_src, k=k,
                                        act_bits=act)
    assert torch.equal(out, laep.moe_combine(y, plan.topk_gate, plan.dest_row))
    # the 16-bit plan at the weights' values: with bf16 activations only float32 sums in
    # another order differ, then H's and y's and the output's rounding, three of 2^-8
    # relative to a row's largest value; MX4 activations lose up to a quarter of a value
    # twice, which over a row's sums is noise
    p16 = laep.MoELayerPlan(T, d, E, k, f)
    o16 = p16.forward(x, wr, _values(gu), _values(dn), prune_beta=beta)
    a, b = host(out), host(o16)
    rel = np.linalg.norm(a - b) / np.linalg.norm(b)
    assert rel <= (3 * 2.0 ** -8 if act == 16 else 0.3), rel
    # another pass over other tokens, then the first again: nothing is kept
    plan.forward(-x, wr, gu, dn, prune_beta=beta)
    assert torch.equal(plan.forward(x, wr, gu, dn, prune_beta=beta), torch.from_numpy(a).cuda().to(BF16))


@pytest.mark.gpu
def test_layer_against_the_oracle():
    case("mx4 layer plan against the oracle")
    T, d, E, k, f = 60, 128, 6, 2, 96 + 32
    rng = np.random.default_rng(2)
    x = round_bf16(rng.normal(size=(T, d)))
    wr = round_bf16(0.1 * rng.normal(size=(E, d)))
    gu, dn = (mx4.quantize(rng.normal(size=s) / np.sqrt(s[-1])) for s in ((E, 2 * f, d), (E, d, f)))
    plan = laep.MoELayerPlan(T, d, E, k, f, mx4_act=16)
    to = lambda q: laep.Mx4(torch.from_numpy(q[0]).cuda(), torch.from_numpy(q[1]).cuda())  # noqa: E731
    out = host(plan.forward(dev(x, BF16), dev(wr, BF16), to(gu), to(dn)))
    idx, gate = host(plan.topk_idx), host(plan.topk_gate)
    _, ref_gate = om.route(x, wr, k)[:2]
    assert np.abs(np.sort(gate, 1) - np.sort(ref_gate, 1)).max() <= 1e-5
    gv, dv = mx4.dequantize(*gu), mx4.dequantize(*dn)
    ref = np.zeros((T, d))
    for t in range(T):
        for j in range(k):
            h = round_bf16(mx4.swiglu(x[t] @ gv[idx[t, j]].T))
            ref[t] += gate[t, j] * round_bf16(h @ dv[idx[t, j]].T)
    # H, y and the output: three bf16 roundings
    assert np.linalg.norm(out - ref) <= 3 * 2.0 ** -8 * np.linalg.norm(ref)


@pytest.mark.gpu
@pytest.mark.parametrize("act", [4, 16])
def test_block(act):
    case(f"mx4 block plan act={act}")
    T, d, E, k, f = 130, 192, 8, 2, 128
    g = torch.Generator(device="cuda").manual_seed(4)
    x, res = (torch.empty((T, d), device="cuda").normal_(generator=g).to(BF16) for _ in range(2))
    wr = torch.empty((E, d), device="cuda").normal_(0, 0.1, generator=g).to(BF16)
    gamma = torch.empty(d, device="cuda").normal_(1, 0.1, generator=g)
    gu, dn = _weights(g, E, d, f)
    w = laep.BlockWeights(gamma, None, wr, gu, dn)
    block = laep.MoEBlockPlan(T, d, E, k, f, training=False, mx4_act=act)
    out, s = block.forward(x, w, residual=res)
    first = out.clone()
    yn, s2, _, _ = laep.moe_layer_norm(x, gamma, None, residual=res)
    plan = laep.MoELayerPlan(T, d, E, k, f, mx4_act=act)
    assert torch.equal(s, s2) and torch.equal(plan.forward(yn, wr, gu, dn), first)
    # a second block of the same model on shared scratch, and the first captured
    other = laep.MoEBlockPlan(T, d, E, k, f, training=False, mx4_act=act, scratch=block)
    o2, _ = other.forward(out, w, residual=s)
    assert torch.isfinite(o2).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, s = block.forward(x, w, residual=res)
    for _ in range(3):
        out.zero_()
        graph.replay()
        assert torch.equal(out, first)
        other.forward(out, w, residual=s)
        torch.cuda.synchronize()


@pytest.mark.gpu
def test_experts_removed():
    """Four of eight experts removed: their slots are gone, the map says where the others lie."""
    case("mx4 layer plan with an expert map")
    T, d, E, k, f = 200, 128, 8, 2, 64
    g = torch.Generator(device="cuda").manual_seed(8)
    x = torch.empty((T, d), device="cuda").normal_(generator=g).to(BF16)
    wr = torch.empty((E, d), device="cuda").normal_(0, 0.1, generator=g).to(BF16)
    gu, dn = _weights(g, E, d, f)
    alive = torch.tensor([1, 0, 1, 1, 0, 0, 1, 0], dtype=torch.uint8, device="cuda")
    emap, _ = laep.laep_compact_experts(alive)
    keep = alive.bool()
    few = [laep.Mx4(w.codes[keep].contiguous(), w.scale[keep].contiguous()) for w in (gu, dn)]
    a, b = (laep.MoELayerPlan(T, d, E, k, f, mx4_act=4) for _ in range(2))
    for p in (a, b):
        p.route_count(x, wr, alive=alive)
    assert torch.equal(a.experts_and_combine(x, gu, dn),
                       b.experts_and_combine(x, *few, expert_map=emap))


def test_plans_that_cannot_take_mx4_weights():
    with pytest.raises(ValueError, match="neither 4 nor 16"):
        laep.MoELayerPlan(4, 64, 4, 2, 64, mx4_act=8, device="cpu")
    for kw in (dict(backward=True), dict(save_act=True), dict(fused_dispatch=False),
               dict(dtype=F32)):
        with pytest.raises(ValueError, match="mx4_act needs"):
            laep.MoELayerPlan(4, 64, 4, 2, 64, mx4_act=16, device="cpu", **kw)
    with pytest.raises(ValueError, match="mx4_act needs"):
        laep.MoEBlockPlan(4, 64, 4, 2, 64, mx4_act=16, device="cpu")
    u8 = torch.uint8
    w = laep.Mx4(torch.zeros(4, 128, 32, dtype=u8), torch.zeros(4, 1, 128, 8, dtype=u8))
    t = torch.zeros(4, 64, 64, dtype=BF16)
    with pytest.raises(ValueError, match="only there"):
        laep.MoELayerPlan(4, 64, 4, 2, 64, device="cpu").experts_and_combine(t[0], w, t)
    with pytest.raises(ValueError, match="only there"):
        laep.MoELayerPlan(4, 64, 4, 2, 64, mx4_act=4, device="cpu").experts_and_combine(t[0], w, t)
    a = laep.MoELayerPlan(4, 64, 4, 2, 64, device="cpu")
    with pytest.raises(ValueError, match="same sizes and kind"):
        laep.MoELayerPlan(4, 64, 4, 2, 64, device="cpu", mx4_act=4, scratch=a)
