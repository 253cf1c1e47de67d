"""Refusals of the calls around the experts (laep_block.h), on the host: an
invalid call returns its code before any HIP call."""
import ctypes
import math

import pytest
import torch

import paper_2601_14327_amd as laep
from test_abi import L, _err, _fake  # noqa: F401  (L: the library fixture)


def test_layer_norm_refusals(L):
    keep, p = _fake(2)
    q = p + 64

    def fwd(**kw):
        a = dict(dict(x=p, res=None, g=p, b=None, dt=1, T=4, d=8, eps=1e-5, s=None, y=q, m=p, r=p),
                 **kw)
        return L.moe_layer_norm(a["x"], a["res"], a["g"], a["b"], a["dt"], a["T"], a["d"],
                                a["eps"], a["s"], a["y"], a["m"], a["r"], None)

    assert fwd(dt=2) == 2 and "dtype" in _err(L)
    assert fwd(d=12) == 1 and "multiple of 8" in _err(L)
    assert fwd(d=0) == 1 and fwd(T=-1) == 1
    assert fwd(d=(1 << 28) + 8) == 2 and "2^28" in _err(L)
    assert fwd(eps=-1.0) == 1 and fwd(eps=math.nan) == 1 and "eps" in _err(L)
    assert fwd(s=q) == 1 and "residual" in _err(L)
    assert fwd(x=None) == 1 and fwd(g=None) == 1 and fwd(y=None) == 1
    assert fwd(x=p + 2) == 1 and "aligned" in _err(L)
    assert fwd(b=p + 4) == 1 and fwd(res=p + 8) == 1
    assert fwd(y=p) == 1 and "alias" in _err(L)
    assert fwd(res=p, x=q, y=p) == 1 and "alias" in _err(L)
    assert fwd(T=0, x=None, y=None) == 0        # no rows: valid, enqueues nothing

    need = L.moe_workspace_bytes(5, 4, 1, 1, 8, 0)
    assert need > 0

    def bwd(**kw):
        a = dict(dict(dy=p, s=p, g=p, m=p, r=p, dres=None, dt=1, T=4, d=8, dx=q, dg=p, db=p, ws=p,
                      n=need), **kw)
        return L.moe_layer_norm_bwd(a["dy"], a["s"], a["g"], a["m"], a["r"], a["dres"], a["dt"],
                                    a["T"], a["d"], a["dx"], a["dg"], a["db"], a["ws"], a["n"],
                                    None)

    assert bwd(dt=9) == 2 and bwd(d=4) == 1 and bwd(T=-3) == 1
    assert bwd(dg=None) == 1 and "dgamma" in _err(L)
    assert bwd(n=need - 1) == 3 and "workspace" in _err(L)
    assert bwd(ws=None) == 1 and bwd(ws=p + 4) == 1
    assert bwd(m=None) == 1 and bwd(dx=None) == 1 and bwd(dy=p + 2) == 1
    assert bwd(dx=p) == 1 and "alias" in _err(L)


def test_balance_refusals(L):
    keep, p = _fake()
    need = L.moe_workspace_bytes(6, 10, 3, 8, 0, 0)
    assert need > 0

    def fwd(**kw):
        a = dict(dict(l=p, i=p, al=None, off=p, T=10, E=8, k=2, S=3, coef=0.1, loss=p, c=p, pm=p,
                      gc=p, ws=p, n=need), **kw)
        return L.moe_balance_loss(a["l"], a["i"], a["al"], a["off"], a["T"], a["E"], a["k"],
                                  a["S"], a["coef"], a["loss"], a["c"], a["pm"], a["gc"], a["ws"],
                                  a["n"], None)

    assert fwd(E=257) == 1 and fwd(k=9) == 1 and fwd(T=-1) == 1
    assert fwd(T=1 << 30) == 1 and "int32" in _err(L)
    assert fwd(S=0) == 1 and fwd(S=(1 << 20) + 1) == 1 and "n_seq" in _err(L)
    assert fwd(off=None) == 1 and "seq_offsets" in _err(L)
    assert fwd(coef=math.inf) == 1 and fwd(coef=math.nan) == 1 and "coef" in _err(L)
    for name in ("l", "i", "loss", "c", "pm", "gc", "ws"):
        assert fwd(**{name: None}) == 1, name
    assert fwd(l=p + 4) == 1 and "aligned" in _err(L)
    assert fwd(n=need - 1) == 3

    def bwd(**kw):
        a = dict(dict(l=p, gc=p, al=None, off=None, dl=None, T=10, E=8, S=1, out=p, acc=0), **kw)
        return L.moe_balance_loss_bwd(a["l"], a["gc"], a["al"], a["off"], a["dl"], a["T"], a["E"],
                                      a["S"], a["out"], a["acc"], None)

    assert bwd(E=0) == 1 and bwd(T=-1) == 1 and bwd(S=2) == 1
    assert bwd(l=None) == 1 and bwd(gc=None) == 1 and bwd(out=None) == 1
    assert bwd(out=p + 4) == 1 and "aligned" in _err(L)
    assert bwd(T=0, l=None, out=None) == 0


def test_act8_refusals(L):
    keep, p = _fake(3)
    q = p + 64
    assert L.moe_act8_save(p, 3, 4, 64, p, p, None) == 2
    assert L.moe_act8_save(p, 1, 4, 48, p, p, None) == 1 and "32" in _err(L)
    assert L.moe_act8_save(p, 1, 4, 0, p, p, None) == 1
    assert L.moe_act8_save(p, 1, -1, 64, p, p, None) == 1
    assert L.moe_act8_save(p, 1, 1 << 31, 64, p, p, None) == 1
    assert L.moe_act8_save(None, 1, 4, 64, p, p, None) == 1
    assert L.moe_act8_save(p + 2, 1, 4, 64, p, p, None) == 1 and "aligned" in _err(L)
    assert L.moe_act8_save(None, 1, 0, 64, None, None, None) == 0
    assert L.moe_act8_load(p, p, 7, 4, 64, p, None) == 2
    assert L.moe_act8_load(p, p, 1, 4, 31, p, None) == 1
    assert L.moe_act8_load(p, None, 1, 4, 64, p, None) == 1
    assert L.moe_act8_load(p, p + 1, 1, 4, 64, p, None) == 1
    assert L.moe_swiglu_bwd_act8(p, p, p, 4, 4, 64, q, p, None) == 2
    assert L.moe_swiglu_bwd_act8(p, p, p, 1, 4, 48, q, p, None) == 1
    assert L.moe_swiglu_bwd_act8(p, p, None, 1, 4, 64, q, p, None) == 1
    assert L.moe_swiglu_bwd_act8(p, p, p, 1, 4, 64, p, q, None) == 1 and "alias" in _err(L)
    assert L.moe_swiglu_bwd_act8(p, p, q, 1, 4, 64, p, p, None) == 1 and "alias" in _err(L)
    assert L.moe_swiglu_bwd_act8(p, p, p + 2, 1, 4, 64, q, p, None) == 1


def test_workspaces_grow_with_every_size():
    """A workspace for the largest call serves every smaller one."""
    from paper_2601_14327_amd import LAEP_CALL_BALANCE, LAEP_CALL_LAYER_NORM_BWD, workspace_bytes

    n = [workspace_bytes(LAEP_CALL_LAYER_NORM_BWD, T, 1, 1, 1000) for T in range(0, 20000, 7)]
    assert n == sorted(n)
    n = [workspace_bytes(LAEP_CALL_LAYER_NORM_BWD, 5000, 1, 1, d) for d in range(8, 20000, 8)]
    assert n == sorted(n)
    n = [workspace_bytes(LAEP_CALL_BALANCE, T, 3, 64) for T in range(0, 400000, 61)]
    assert n == sorted(n)
    n = [workspace_bytes(LAEP_CALL_BALANCE, 1000, s, 64) for s in range(1, 3000)]
    assert n == sorted(n)
    n = [workspace_bytes(LAEP_CALL_BALANCE, 1000, 3, E) for E in range(1, 257)]
    assert n == sorted(n)


def test_binding_refuses_host_tensors_and_wrong_shapes():
    x = torch.zeros((4, 64))
    for call in (lambda: laep.moe_layer_norm(x, torch.ones(64)),
                 lambda: laep.moe_layer_norm_bwd(x, x, torch.ones(64), x[:, 0], x[:, 0]),
                 lambda: laep.moe_balance_loss(x, torch.zeros((4, 2), dtype=torch.int32)),
                 lambda: laep.moe_balance_loss_bwd(x, x[:1]),
                 lambda: laep.moe_act8_save(x),
                 lambda: laep.moe_act8_load(x, x),
                 lambda: laep.moe_swiglu_bwd_act8(x, x, x)):
        with pytest.raises(ValueError, match="device tensor"):
            call()


@pytest.mark.gpu
def test_binding_refuses_on_the_device():
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device="cuda")
    bf = torch.bfloat16
    x, g = z(4, 64, dt=bf), z(64)
    with pytest.raises(ValueError, match="gamma"):
        laep.moe_layer_norm(x, g.to(bf))
    with pytest.raises(ValueError, match="residual"):
        laep.moe_layer_norm(x, g, residual=z(4, 64))
    with pytest.raises(ValueError, match="contiguous"):
        laep.moe_layer_norm(z(4, 128, dt=bf)[:, :64], g)
    with pytest.raises(laep.LaepError):
        laep.moe_layer_norm(x, g, sum_out=z(4, 64, dt=bf))
    with pytest.raises(laep.LaepError):
        laep.moe_layer_norm(x.half(), g)
    with pytest.raises(laep.LaepError):
        laep.moe_layer_norm(z(4, 12, dt=bf), z(12))
    with pytest.raises(ValueError, match="mean"):
        laep.moe_layer_norm_bwd(x, x, g, z(3), z(4))
    with pytest.raises(laep.LaepError):
        laep.moe_layer_norm_bwd(x, x, g, z(4), z(4), ws=z(1))
    idx = z(4, 2, dt=torch.int32)
    with pytest.raises(ValueError, match="topk_idx"):
        laep.moe_balance_loss(z(4, 8), idx.long())
    with pytest.raises(ValueError, match="contiguous"):
        laep.moe_balance_loss(z(8, 4).t(), idx)
    with pytest.raises(ValueError, match="contiguous"):
        laep.moe_act8_save(z(64, 4, dt=bf).t())
    with pytest.raises(ValueError, match="contiguous"):
        laep.moe_swiglu_bwd_act8(z(4, 64, dt=torch.int8), z(4, 2, dt=torch.uint8),
                                 z(32, 4, dt=bf).t())
    with pytest.raises(ValueError, match="seq_offsets"):
        laep.moe_balance_loss(z(4, 8), idx, seq_offsets=z(3, dt=torch.int64))
    with pytest.raises(ValueError, match="grad_coef"):
        laep.moe_balance_loss_bwd(z(4, 8), z(2, 8))
    with pytest.raises(ValueError, match="accumulate"):
        laep.moe_balance_loss_bwd(z(4, 8), z(1, 8), accumulate=True)
    with pytest.raises(ValueError, match="dloss"):
        laep.moe_balance_loss_bwd(z(4, 8), z(1, 8), dloss=torch.ones(1))
    with pytest.raises(laep.LaepError):
        laep.moe_act8_save(z(4, 40, dt=bf))
    with pytest.raises(ValueError, match="scale"):
        laep.moe_act8_load(z(4, 64, dt=torch.int8), z(4, 1, dt=torch.uint8))
    with pytest.raises(laep.LaepError):
        laep.moe_act8_load(z(4, 64, dt=torch.int8), z(4, 2, dt=torch.uint8), torch.float16)
    with pytest.raises(ValueError, match="q must"):
        laep.moe_swiglu_bwd_act8(z(4, 64, dt=torch.int8), z(4, 2, dt=torch.uint8), x)


def test_router_backward_with_balance_refusals(L):
    keep, p = _fake()
    need = L.moe_workspace_bytes(4, 16, 2, 8, 64, 0)

    def call(**kw):
        a = dict(dict(dg=p, i=p, g=p, l=p, al=None, x=p, w=p, gc=p, off=None, S=1, dl=None, dt=1,
                      T=16, d=64, E=8, k=2, out=None, dw=p, db=None, dx=p, ws=p, n=need), **kw)
        return L.moe_route_bwd_balance(
            a["dg"], a["i"], a["g"], a["l"], a["al"], a["x"], a["w"], a["gc"], a["off"], a["S"],
            a["dl"], a["dt"], a["T"], a["d"], a["E"], a["k"], 1, a["out"], a["dw"], a["db"],
            a["dx"], 0, a["ws"], a["n"], None)

    assert call(dt=5) == 2 and call(k=9) == 1 and call(d=60) == 1 and call(T=-1) == 1
    assert call(S=2) == 1 and "seq_offsets" in _err(L)
    assert call(S=0, off=p) == 1
    assert call(dw=None, db=p) == 1 and "dbias" in _err(L)
    for name in ("dg", "i", "g", "l", "x", "w", "gc", "ws"):
        assert call(**{name: None}) == 1, name
    for name in ("l", "x", "w", "dx", "out", "ws"):
        assert call(**{name: p + 4}) == 1 and "aligned" in _err(L), name
    assert call(n=need - 1) == 3


def test_expert_backward_at_a_checkpoint_refusals(L):
    keep, p = _fake()

    def call(**kw):
        a = dict(dict(dy=p, dout=None, gate=None, x=p, rs=p, T=10, k=2, q=p, sc=p, dt=1, d=128,
                      f=128, R=20, dx=p, n=1 << 30), **kw)
        return L.moe_grouped_ffn_bwd_gather_act8(
            a["dy"], a["dout"], a["gate"], a["x"], a["rs"], a["T"], a["k"], a["q"], a["sc"], p, p,
            p, None, a["dt"], 8, a["d"], a["f"], a["R"], a["dx"], p, p, 0, p, a["n"], None)

    assert call(dt=0) == 2 and "LAEP_BF16" in _err(L)
    assert call(d=96) == 2 and call(R=21) == 1 and call(rs=None) == 1
    assert call(q=None) == 1 and call(sc=None) == 1 and call(dx=None) == 1
    assert call(q=p + 4) == 1 and call(sc=p + 4) == 1 and "aligned" in _err(L)
    assert call(dy=None) == 1 and "dout" in _err(L)
    assert call(n=64) == 3 and "moe_grouped_ffn_bwd_gather_act8" in _err(L)
    big = L.moe_grouped_ffn_bwd_gather_act8(None, p, p, p, p, 1 << 20, 1, p, p, p, p, p, None, 1, 8,
                                            1024, 128, 20, p, p, p, 0, p, 1 << 40, None)
    assert big == 2 and "2 GiB" in _err(L)
