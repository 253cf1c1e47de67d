"""The block as one training step (MoEBlockPlan), its router's backward with the
balance loss and its expert backward at 8-bit checkpoints, against float64
autograd, the oracle and the calls they replace.

Tolerances.  Router products in float32: 1e-5 of the terms they sum (test_gpu_block's
reasons), bf16 dx one rounding.  The whole block passes through bf16 roundings of y,
act_save, H, y_perm, dY, dH, dA and dX, eight of 2^-9 each on one path, and the 8-bit
checkpoint's half a step of 1/128 of the block's largest value; rounding errors of
many rows add as noise, so a gradient's whole error, in the norm over the tensor,
stays below the worst single path: 8 * 2^-9 + 1/64 < 0.04."""
import os
import sys

import numpy as np
import pytest
import torch

import oracle.block as ob
import oracle.moe as om
import paper_2601_14327_amd as laep
from _gpu import case, dev, host

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def _rel(got, ref):
    got, ref = host(got), np.asarray(ref, np.float64)
    return np.linalg.norm(got - ref) / max(np.linalg.norm(ref), 1e-30)


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("T,d,E,k,S,dead", [(1, 64, 4, 1, 1, 0), (70, 72, 5, 2, 3, 0),
                                            (900, 128, 8, 2, 1, 2), (333, 200, 45, 8, 4, 0),
                                            (520, 64, 130, 4, 2, 30)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_router_backward_with_balance(T, d, E, k, S, dead, renorm, dtype):
    case(f"route_bwd_balance T={T} d={d} E={E} k={k} seqs={S} dead={dead} {renorm} {dtype}")
    rng = np.random.default_rng(T + E)
    dt = BF16 if dtype == "bf16" else F32
    x = dev(rng.standard_normal((T, d)).astype(np.float32), dt)
    w = dev((0.2 * rng.standard_normal((E, d))).astype(np.float32), dt)
    dg = dev(rng.standard_normal((T, k)).astype(np.float32), F32)
    dx0 = dev(rng.standard_normal((T, d)).astype(np.float32), dt)
    alive = None
    if dead:
        alive = np.ones(E, np.uint8)
        alive[rng.permutation(E)[:dead]] = 0
    off = None
    if S > 1:
        off = np.concatenate([[0], np.sort(rng.integers(0, T + 1, S - 1)), [T]]).astype(np.int32)
    at = None if alive is None else dev(alive, torch.uint8)
    ot = None if off is None else dev(off, torch.int32)
    idx, gate, logits = laep.moe_route(x, w, k, alive=at, renorm=renorm, want_logits=True)
    _, _, _, grad = laep.moe_balance_loss(logits, idx, coef=5.0, alive=at, seq_offsets=ot)
    dl_scale = dev(np.array([float(T)], np.float32), F32)
    dx, dw, db, dl = laep.moe_route_bwd_balance(
        dg, idx, gate, logits, x, w, grad, seq_offsets=ot, dloss=dl_scale, renorm=renorm,
        alive=at, dx=dx0.clone(), accumulate_dx=True, want_dlogits=True, want_dbias=True)
    gates_dl, _, _, _ = om.route_bwd(host(dg), host(idx), host(gate), host(x), host(w),
                                     logits=host(logits), alive=alive, renorm=renorm, dtype="f64")
    ref = gates_dl + ob.balance_loss_bwd(host(logits), host(grad), float(T), alive, off)
    scale = np.abs(ref).max()
    assert np.abs(host(dl) - ref).max() <= 1e-5 * scale
    hx, hw = host(x), np.where((alive if alive is not None else np.ones(E))[:, None], host(w), 0.0)
    terms = np.abs(host(dl)).T @ np.abs(hx)
    assert (np.abs(host(dw) - host(dl).T @ hx) <= 1e-5 * terms + 1e-30).all()
    assert (np.abs(host(db) - host(dl).sum(0)) <= 1e-5 * np.abs(host(dl)).sum(0) + 1e-30).all()
    rdx = host(dx0) + host(dl) @ hw
    tdx = np.abs(host(dx0)) + np.abs(host(dl)) @ np.abs(hw)
    unit = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
    assert (np.abs(host(dx) - rdx) <= unit * np.abs(rdx) + 1e-5 * tdx).all()
    # the halves of a training step, and without dlogits
    kw = dict(seq_offsets=ot, dloss=dl_scale, renorm=renorm, alive=at)
    a = laep.moe_route_bwd_balance(dg, idx, gate, logits, x, w, grad, data=False,
                                   want_dbias=True, **kw)
    b = laep.moe_route_bwd_balance(dg, idx, gate, logits, x, w, grad, weights=False,
                                   dx=dx0.clone(), accumulate_dx=True, **kw)
    assert torch.equal(a[1], dw) and torch.equal(a[2], db) and torch.equal(b[0], dx)


def test_router_backward_without_a_loss_is_the_plain_one():
    T, d, E, k = 300, 128, 16, 2
    case("route_bwd_balance with a zero gradient")
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((T, d), generator=g, device="cuda").to(BF16)
    w = (0.2 * torch.randn((E, d), generator=g, device="cuda")).to(BF16)
    dg = torch.randn((T, k), generator=g, device="cuda")
    zero = torch.zeros((1, E), device="cuda")
    idx, gate, logits = laep.moe_route(x, w, k, renorm=False, want_logits=True)
    got = laep.moe_route_bwd_balance(dg, idx, gate, logits, x, w, zero, renorm=False,
                                     want_dlogits=True)
    ref = laep.moe_route_bwd(dg, idx, gate, x, w, renorm=False, logits=logits, want_dlogits=True)
    assert torch.equal(got[3], ref[3])
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


@pytest.mark.parametrize("R_extra", [0, 37])
@pytest.mark.parametrize("dy_on_load", [False, True])
@pytest.mark.parametrize("T,d,E,k,f", [(40, 64, 4, 1, 64), (300, 128, 6, 2, 192),
                                       (700, 256, 9, 3, 320)])
def test_expert_backward_at_a_checkpoint(T, d, E, k, f, dy_on_load, R_extra):
    """Bit for bit the 16-bit call at the decoded pre-activations; rows past the
    experts' may hold anything."""
    case(f"ffn_bwd act8 T={T} d={d} E={E} k={k} f={f} dy on load {dy_on_load}")
    g = torch.Generator(device="cuda").manual_seed(T)
    r = lambda *s, std=1.0: (std * torch.randn(s, generator=g, device="cuda")).to(BF16)
    x, dout = r(T, d), r(T, d)
    wgu, wd, wr = r(E, 2 * f, d, std=0.1), r(E, d, f, std=0.1), r(E, d, std=0.1)
    alive = torch.ones(E, dtype=torch.uint8, device="cuda")
    if R_extra:
        alive[: E - k + 1] = 0         # fewer alive than slots: unrouted rows at the end
    idx, gate = laep.moe_route(x, wr, k, alive=alive)
    _, off, dest, src = laep.moe_expert_counts(idx, E, want_row_src=True)
    R = T * k
    n = int(off[-1])
    if n < R:
        src[n:] = 0
    y, act = laep.moe_grouped_ffn_fwd_gather(x, src, k, wgu, wd, off, save_act=True)
    act[n:] = 1.0
    if n + 1 < R:
        act[n + 1:] = float("nan")
    dy, _ = laep.moe_combine_bwd(dout, y, gate, dest)
    q, b = laep.moe_act8_save(act)
    dec = laep.moe_act8_load(q, b)
    kw = dict(dout=dout, topk_gate=gate)
    ref = laep.moe_grouped_ffn_bwd_gather(None if dy_on_load else dy, x, src, k, dec, wgu, wd,
                                          off, **kw)
    got = laep.moe_grouped_ffn_bwd_gather_act8(None if dy_on_load else dy, x, src, k, q, b, wgu,
                                               wd, off, **kw)
    assert torch.equal(got[0][:n], ref[0][:n])
    assert torch.equal(got[1], ref[1]) and torch.equal(got[2], ref[2])
    full = laep.moe_grouped_ffn_bwd_gather(None if dy_on_load else dy, x, src, k, act, wgu, wd,
                                           off, **kw)
    if n:
        for a, c in zip((got[0][:n], got[1], got[2]), (full[0][:n], full[1], full[2])):
            assert _rel(a, host(c)) <= 1 / 64


def _reference_block(x, res, w, k, coef, renorm, off, idx, gate_only=False):
    """float64 autograd of the block with the selection idx [T, k] given."""
    t = {n: v.double().requires_grad_(True) for n, v in
         dict(x=x, res=res, gamma=w.gamma, beta=w.beta, wr=w.w_router, wgu=w.w_gate_up,
              wd=w.w_down).items()}
    s = t["x"] + t["res"]
    y = torch.nn.functional.layer_norm(s, (s.shape[1],), t["gamma"], t["beta"], 1e-5)
    logits = y @ t["wr"].T
    p = torch.softmax(logits, 1)
    ids = idx.long()
    gate = torch.softmax(logits.gather(1, ids), 1) if renorm else p.gather(1, ids)
    out = torch.zeros_like(s)
    E, f = t["wr"].shape[0], t["wd"].shape[2]
    for e in range(E):
        tok, slot = (ids == e).nonzero(as_tuple=True)
        if tok.numel() == 0:
            continue
        a = y[tok] @ t["wgu"][e].T
        h = torch.nn.functional.silu(a[:, :f]) * a[:, f:]
        out = out.index_add(0, tok, gate[tok, slot, None] * (h @ t["wd"][e].T))
    loss = 0.0
    live = sum(b > a for a, b in zip(off, off[1:]))
    for a, b in zip(off, off[1:]):
        if b > a:
            n = torch.bincount(ids[a:b].ravel(), minlength=E).double()
            loss = loss + coef / live * (E * n / (k * (b - a)) * p[a:b].mean(0)).sum()
    return t, s, out, loss


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("act_bits", [8, 16])
@pytest.mark.parametrize("T,d,E,k,f,off", [(192, 128, 8, 2, 128, [0, 50, 50, 192]),
                                           (257, 64, 5, 1, 64, [0, 257]),
                                           (130, 256, 16, 4, 192, [0, 1, 130])])
def test_block_step_against_autograd(T, d, E, k, f, off, act_bits, renorm):
    case(f"block T={T} d={d} E={E} k={k} f={f} act_bits={act_bits} renorm={renorm}")
    g = torch.Generator().manual_seed(T + d)
    r = lambda *s, std=1.0, dt=BF16: (std * torch.randn(s, generator=g)).to("cuda").to(dt)
    x, res, dout = r(T, d), r(T, d), r(T, d)
    w = laep.BlockWeights(1 + r(d, std=0.1, dt=F32), r(d, std=0.1, dt=F32), r(E, d, std=0.3),
                          r(E, 2 * f, d, std=d ** -0.5), r(E, d, f, std=f ** -0.5))
    coef = 30.0        # large, so that the loss's gradient shows in the router's
    n_seq = len(off) - 1
    seq = torch.tensor(off, dtype=torch.int32, device="cuda") if n_seq > 1 else None
    plan = laep.MoEBlockPlan(T, d, E, k, f, n_seq=n_seq, coef=coef, act_bits=act_bits,
                             renorm=renorm)
    out, s = plan.forward(x, w, res, seq_offsets=seq)
    dx = plan.backward(dout, w, want_dbias=True)
    torch.cuda.synchronize()
    p = plan.layer
    cpu = laep.BlockWeights(*(v.cpu() for v in w))
    t, rs, rout, rloss = _reference_block(x.cpu(), res.cpu(), cpu, k, coef, renorm, off,
                                          p.topk_idx.cpu())
    ((rout + rs) * dout.cpu().double()).sum().add(rloss).backward()
    assert abs(float(plan.loss) - float(rloss.detach())) <= 0.01 * abs(float(rloss.detach()))
    assert _rel(out, rout.detach().numpy()) <= 0.04
    for name, got in (("x", dx), ("res", dx), ("gamma", plan.dgamma), ("beta", plan.dbeta),
                      ("wr", p.dw_router), ("wgu", p.dw_gate_up), ("wd", p.dw_down)):
        assert _rel(got, t[name].grad.numpy()) <= 0.04, name
    assert torch.equal(plan.seq_counts.sum(0).to(torch.int32), p.counts)


def test_blocks_share_scratch():
    T, d, E, k, f = 300, 128, 8, 2, 128
    case("two blocks on shared scratch")
    g = torch.Generator(device="cuda").manual_seed(2)
    r = lambda *s, std=1.0, dt=BF16: (std * torch.randn(s, generator=g, device="cuda")).to(dt)
    w = [laep.BlockWeights(1 + r(d, std=0.1, dt=F32), None, r(E, d, std=0.3),
                           r(E, 2 * f, d, std=0.1), r(E, d, f, std=0.1)) for _ in range(2)]
    x, dout = r(T, d), r(T, d)

    def step(blocks):
        h, stream = x, None
        for b, wb in zip(blocks, w):
            h, stream = b.forward(h, wb, stream)
        grad = dout
        for b, wb in zip(reversed(blocks), reversed(w)):
            grad = b.backward(grad, wb)
        return [h, stream, grad] + [v for b in blocks for v in
                                    (b.dgamma, b.loss, b.layer.dw_router, b.layer.dw_gate_up,
                                     b.layer.dw_down)]

    alone = [laep.MoEBlockPlan(T, d, E, k, f) for _ in range(2)]
    want = [v.clone() for v in step(alone)]
    first = laep.MoEBlockPlan(T, d, E, k, f)
    shared = [first, laep.MoEBlockPlan(T, d, E, k, f, scratch=first)]
    assert shared[1].layer.act_save is first.layer.act_save
    for _ in range(2):
        got = step(shared)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(ValueError, match="scratch"):
        laep.MoEBlockPlan(T, d, E, k, 2 * f, scratch=first)
    with pytest.raises(ValueError, match="scratch"):
        laep.MoEBlockPlan(T, d, E, k, f, n_seq=2, scratch=first)


def test_block_serves_single_tokens_and_pruned_experts():
    d, E, k, f = 256, 8, 2, 128
    case("block, serving form")
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s, std=1.0, dt=BF16: (std * torch.randn(s, generator=g, device="cuda")).to(dt)
    w = laep.BlockWeights(1 + r(d, std=0.1, dt=F32), r(d, std=0.1, dt=F32), r(E, d, std=0.3),
                          r(E, 2 * f, d, std=0.1), r(E, d, f, std=0.1))
    alive = torch.tensor([1, 0, 1, 1, 0, 1, 1, 1], dtype=torch.uint8, device="cuda")
    x, res = r(5, d), r(5, d)
    whole = laep.MoEBlockPlan(5, d, E, k, f)
    out, s = whole.forward(x, w, res, alive=alive)
    assert not whole.seq_counts[0][alive == 0].any()
    one = laep.MoEBlockPlan(1, d, E, k, f, training=False)
    for t in range(5):
        o, st = one.forward(x[t:t + 1].contiguous(), w, res[t:t + 1].contiguous(), alive=alive)
        assert torch.equal(st[0], s[t])
        assert _rel(o[0], host(out[t])) <= 2.0 ** -7


def test_plan_refuses_checkpoints_it_cannot_keep():
    with pytest.raises(ValueError, match="act_bits"):
        laep.MoELayerPlan(8, 64, 4, 2, 64, act_bits=8)
    with pytest.raises(ValueError, match="act_bits"):
        laep.MoELayerPlan(8, 64, 4, 2, 64, backward=True, act_bits=4)
    with pytest.raises(ValueError, match="act_bits"):
        laep.MoELayerPlan(8, 64, 4, 2, 64, backward=True, fused_dispatch=False, act_bits=8)


@pytest.mark.parametrize("act_bits", [8, 16])
def test_example_trains(act_bits):
    case(f"examples/train_block.py act_bits={act_bits}")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    sys.path.insert(0, os.path.join(root, "examples"))
    try:
        import train_block
    finally:
        sys.path.pop(0)
    history = train_block.train(steps=12, act_bits=act_bits)
    assert all(np.isfinite(v).all() for v in history)
    assert history[-1][0] < 0.9 * history[0][0]


def test_block_step_in_a_graph():
    """A captured training step replays to the eager bits, with eager work between."""
    T, d, E, k, f = 500, 128, 8, 2, 128
    case("block step, graph replays")
    g = torch.Generator(device="cuda").manual_seed(4)
    r = lambda *s, std=1.0, dt=BF16: (std * torch.randn(s, generator=g, device="cuda")).to(dt)
    w = laep.BlockWeights(1 + r(d, std=0.1, dt=F32), r(d, std=0.1, dt=F32), r(E, d, std=0.3),
                          r(E, 2 * f, d, std=0.1), r(E, d, f, std=0.1))
    off = torch.tensor([0, 100, 100, 500], dtype=torch.int32, device="cuda")
    plan = laep.MoEBlockPlan(T, d, E, k, f, n_seq=3)
    x, res, dout = r(T, d), r(T, d), r(T, d)

    def step():
        out, s = plan.forward(x, w, res, seq_offsets=off)
        dx = plan.backward(dout, w, want_dbias=True)
        p = plan.layer
        return [out, s, dx, plan.loss, plan.seq_counts, plan.dgamma, plan.dbeta, p.dw_router,
                p.dbias, p.dw_gate_up, p.dw_down]

    def inputs(seed):
        h = torch.Generator(device="cuda").manual_seed(seed)
        for t in (x, res, dout):
            t.copy_(torch.randn(t.shape, generator=h, device="cuda"))

    step()                       # streams and buffers exist before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for seed in (10, 11, 12):
        inputs(seed)
        want = [t.clone() for t in step()]
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
