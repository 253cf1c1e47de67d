"""Layer norm, balance loss and 8-bit checkpoints at sizes that take other paths than
the small ones: workgroups that walk several rows, rows wider than a workgroup's
registers in several passes, streamed loads, offsets past 2^31 elements, grids at
their limit.

Tolerances against the oracle are those of test_gpu_block.py (sums at most 200
roundings deep: a lane's rows, then its workgroup's, then 256 parts by 16).  Large calls
are compared bit for bit with small calls of the same rows: a row's result does not
depend on the others."""
import numpy as np
import pytest
import torch

import paper_2601_14327_amd as laep
from _gpu import case, dev, host
from test_gpu_block import (BF16, DT, F32, REL, _check_norm, _check_norm_bwd, _norm_inputs)

pytestmark = pytest.mark.gpu


# rows past what a grid of workgroups holds at a time, so that they walk: several rows
# side by side (8, 32, 128, 192 lanes a row), one row of one and of several vectors a lane
WALKS = [(40000, 64), (30000, 256), (8000, 1000), (4000, 1496), (1500, 5112), (1200, 9000),
         (1200, 12000)]


@pytest.mark.parametrize("T,d", WALKS + [(600, 16392)])
@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layer_norm_walks_rows(T, d, residual, dtype):
    case(f"layer norm, workgroups walk rows, T={T} d={d} {dtype} residual={residual}")
    x, res, dy, gamma, beta = _norm_inputs(T, d, dtype, 7 * T + d)
    if residual:
        out = laep.moe_layer_norm(x, gamma, beta, residual=res)
        _check_norm(x, res, gamma, beta, dtype, out)
        got = laep.moe_layer_norm_bwd(dy, out[1], gamma, out[2], out[3], dres=res)
        _check_norm_bwd(out[1], dy, gamma, out[2], out[3], res, dtype, got)
    else:
        out = laep.moe_layer_norm(x, gamma)
        _check_norm(x, None, gamma, None, dtype, out)
        got = laep.moe_layer_norm_bwd(dy, x, gamma, out[2], out[3], want_dbeta=False)
        _check_norm_bwd(x, dy, gamma, out[2], out[3], None, dtype, got)


def _slices(R, n=300):
    """The first, some middle and the last rows."""
    return [(0, n), (R // 2 - 7, R // 2 - 7 + n), (R - n, R)]


@pytest.mark.parametrize("dtype,R,f", [("bf16", 23040, 1024), ("f32", 13056, 1024),
                                       ("bf16", 1050000, 1024)])
def test_swiglu_bwd_act8_of_large_calls(dtype, R, f):
    """Past 224 MiB dH's loads stream; the last case's q passes 2^31 elements."""
    case(f"swiglu bwd act8, streamed, R={R} f={f} {dtype}")
    assert R * f * (2 + 4 * DT[dtype].itemsize) > 224 << 20
    g = torch.Generator(device="cuda").manual_seed(R)
    q = torch.randint(-127, 128, (R, 2 * f), dtype=torch.int8, device="cuda", generator=g)
    b = torch.randint(112, 123, (R, 2 * f // 32), dtype=torch.uint8, device="cuda", generator=g)
    dh = torch.randn((R, f), dtype=DT[dtype], device="cuda", generator=g)
    da, h = laep.moe_swiglu_bwd_act8(q, b, dh)
    for lo, hi in _slices(R):
        wa, wh = laep.moe_swiglu_bwd_act8(q[lo:hi], b[lo:hi], dh[lo:hi])
        assert torch.equal(da[lo:hi], wa) and torch.equal(h[lo:hi], wh)
    over, want = dh, h            # H in dH's place
    da2, h2 = laep.moe_swiglu_bwd_act8(q, b, over, h=over)
    assert h2 is over and torch.equal(h2, want) and torch.equal(da2, da)
    del q, b, dh, da, h, da2, h2, over, want
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_act8_past_the_grid(dtype):
    """More than 2^30 threads' values, so that the grid is walked a second time."""
    C = 8192
    R = (1 << 30) * (16 // DT[dtype].itemsize) // C + 70
    case(f"act8 past the grid, R={R} C={C} {dtype}")
    t = torch.zeros((R, C), dtype=DT[dtype], device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    for lo, hi in _slices(R, 100):
        t[lo:hi] = torch.randn((hi - lo, C), device="cuda", generator=g).to(t.dtype)
    q, b = laep.moe_act8_save(t)
    out = laep.moe_act8_load(q, b, t.dtype)
    seen = 0
    for lo, hi in _slices(R, 100):
        wq, wb = laep.moe_act8_save(t[lo:hi].contiguous())
        assert torch.equal(q[lo:hi], wq) and torch.equal(b[lo:hi], wb)
        assert torch.equal(out[lo:hi], laep.moe_act8_load(wq, wb, t.dtype))
        assert not q[seen:lo].any() and not out[seen:lo].any() and (b[seen:lo] == 1).all()
        seen = hi
    del t, q, b, out
    torch.cuda.empty_cache()


def test_swiglu_bwd_act8_past_the_grid():
    f = 8192
    R = (1 << 32) // f + 70                   # 2^30 threads of four float32 values, and more
    case(f"swiglu bwd act8 past the grid, R={R} f={f}")
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.zeros((R, 2 * f), dtype=torch.int8, device="cuda")
    b = torch.full((R, 2 * f // 32), 120, dtype=torch.uint8, device="cuda")
    dh = torch.zeros((R, f), device="cuda")
    for lo, hi in _slices(R, 100):
        q[lo:hi] = torch.randint(-127, 128, (hi - lo, 2 * f), device="cuda", generator=g)
        dh[lo:hi] = torch.randn((hi - lo, f), device="cuda", generator=g)
    want = [laep.moe_swiglu_bwd_act8(q[lo:hi], b[lo:hi], dh[lo:hi]) for lo, hi in _slices(R, 100)]
    da, h = laep.moe_swiglu_bwd_act8(q, b, dh, h=dh)
    seen = 0
    for (lo, hi), (wa, wh) in zip(_slices(R, 100), want):
        assert torch.equal(da[lo:hi], wa) and torch.equal(h[lo:hi], wh)
        assert not da[seen:lo].any() and not h[seen:lo].any()
        seen = hi
    del q, b, dh, da, h, want
    torch.cuda.empty_cache()


def test_layer_norm_past_2_to_the_31_elements():
    T, d = 1050000, 2048
    case(f"layer norm T={T} d={d}")
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((T, d), dtype=BF16, device="cuda", generator=g)
    res = torch.randn((T, d), dtype=BF16, device="cuda", generator=g)
    gamma = 1 + 0.1 * torch.randn(d, device="cuda", generator=g)
    beta = torch.randn(d, device="cuda", generator=g)
    y, s, mean, rstd = laep.moe_layer_norm(x, gamma, beta, residual=res)
    plain = laep.moe_layer_norm(x, gamma)
    for lo, hi in _slices(T):
        for whole, part in ((y, 0), (s, 1), (mean, 2), (rstd, 3)):
            want = laep.moe_layer_norm(x[lo:hi], gamma, beta, residual=res[lo:hi])[part]
            assert torch.equal(whole[lo:hi], want)
        assert torch.equal(plain[0][lo:hi], laep.moe_layer_norm(x[lo:hi], gamma)[0])
    # gradients that only a first and a last row carry: dgamma and dbeta are those rows'
    del y, plain
    dy = torch.zeros((T, d), dtype=BF16, device="cuda")
    dy[3] = torch.randn(d, device="cuda", generator=g)
    dy[T - 2] = torch.randn(d, device="cuda", generator=g)
    dx, dg, db = laep.moe_layer_norm_bwd(dy, s, gamma, mean, rstd, dres=res)
    pick = torch.tensor([3, T - 2], device="cuda")
    wx, wg, wb = laep.moe_layer_norm_bwd(dy[pick], s[pick], gamma, mean[pick], rstd[pick],
                                         dres=res[pick])
    assert torch.equal(dx[pick], wx) and torch.equal(dg, wg) and torch.equal(db, wb)
    dy[pick] = 0
    assert not dy.any()
    dx[pick] = res[pick]
    assert torch.equal(dx, res)               # the other rows pass dres on
    del x, res, s, dy, dx
    torch.cuda.empty_cache()


def test_balance_past_2_to_the_31_logits():
    T, E, k = 8500000, 256, 2
    # a lane sums up to T / 1024 / 4 = 2076 rows one after the other, a last pass 1024 parts
    tol = REL + 2.0 ** -24 * 3100
    case(f"balance loss T={T} E={E}")
    g = torch.Generator(device="cuda").manual_seed(6)
    logits = torch.randn((T, E), device="cuda", generator=g)
    logits[(1 << 31) // E:, :8] += 10.0       # rows past 2^31 elements show in the means
    idx = torch.randint(0, E, (T, k), dtype=torch.int32, device="cuda", generator=g)
    cuts = [0, 5, 4000000, 4000000, T]
    off = torch.tensor(cuts, dtype=torch.int32, device="cuda")
    loss, counts, prob, grad = laep.moe_balance_loss(logits, idx, seq_offsets=off)
    live = 3
    total = 0.0
    for s, (a, b) in enumerate(zip(cuts, cuts[1:])):
        want = torch.bincount(idx[a:b].reshape(-1), minlength=E) if b > a else \
            torch.zeros(E, device="cuda")
        assert torch.equal(counts[s].long(), want.long())
        ref = torch.zeros(E, dtype=torch.float64, device="cuda")
        for i in range(a, b, 500000):
            ref += torch.softmax(logits[i:min(i + 500000, b)].double(), 1).sum(0)
        ref /= max(b - a, 1)
        assert ((prob[s].double() - ref).abs() <= tol * ref).all()
        if b > a:
            f = E * want.double() / (k * (b - a))
            total += float((f * ref).sum()) / live
            coef = f / ((b - a) * live)
            assert ((grad[s].double() - coef).abs() <= REL * coef).all()
    assert abs(float(loss) - total) <= tol * total
    dl = laep.moe_balance_loss_bwd(logits, grad, seq_offsets=off)
    for a, b, s in ((0, 5, 0), (3999000, 4000000, 1), (4000000, 4000300, 3), (T - 300, T, 3)):
        want = laep.moe_balance_loss_bwd(logits[a:b], grad[s:s + 1])
        assert torch.equal(dl[a:b], want)
    del logits, idx, dl
    torch.cuda.empty_cache()
