"""Layer norm, balance loss and 8-bit activation checkpoints on the device
against the float64 oracle.

Tolerances (u = 2^-24).  A bf16 output is one rounding of a float32 value: half
an ulp, at most 2^-8 of the value.  Float32 parts: row statistics sum at most 200
roundings deep (a lane's share, then a tree), so 1e-5 (170 u) of the terms'
magnitude; probabilities carry the rounding of logit - max (|l| <= 20: 20 u) and
a few ulps of exp, also under 1e-5 of themselves; gradients 1e-5 of the terms they
sum.  Checkpoints are exact."""
import numpy as np
import pytest
import torch

import oracle.block as ob
import paper_2601_14327_amd as laep
from _gpu import case, dev, host

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
DT = {"bf16": BF16, "f32": F32}
REL = 1e-5


def _rounding(dtype):
    return 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23


def _check(name, got, ref, tol):
    got, ref = host(got), np.asarray(ref, np.float64)
    assert got.shape == ref.shape, name
    bad = ~(np.abs(got - ref) <= np.broadcast_to(tol, ref.shape))
    assert not bad.any(), (f"{name}: {int(bad.sum())} of {bad.size} off, first at "
                           f"{np.argwhere(bad)[0]}: {got[bad][0]} for {ref[bad][0]}")


# ---------------------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------------------
def _norm_inputs(T, d, dtype, seed, offset=0.0):
    rng = np.random.default_rng(seed)
    sc = np.exp(0.5 * rng.standard_normal(d))
    x = dev((rng.standard_normal((T, d)) * sc + offset).astype(np.float32), DT[dtype])
    res = dev(rng.standard_normal((T, d)).astype(np.float32), DT[dtype])
    dy = dev(rng.standard_normal((T, d)).astype(np.float32), DT[dtype])
    gamma = dev((1 + 0.2 * rng.standard_normal(d)).astype(np.float32), F32)
    beta = dev(rng.standard_normal(d).astype(np.float32), F32)
    return x, res, dy, gamma, beta


def _check_norm(x, res, gamma, beta, dtype, out, eps=1e-5):
    y, s, mean, rstd = out
    ry, rs, rm, rr = ob.layer_norm(host(x), host(gamma), None if beta is None else host(beta),
                                   None if res is None else host(res), eps, dtype)
    assert np.array_equal(host(s), rs)
    top = np.abs(rs).max(1)
    _check("mean", mean, rm, REL * top)
    # the centred values carry the mean's error, whole over their spread
    cond = REL + 8 * 2.0 ** -24 * top * rr
    _check("rstd", rstd, rr, rr * cond)
    g = np.abs(host(gamma)).max()
    scale = (np.abs(rs - rm[:, None]) * rr[:, None]).max(1) * g
    _check("y", y, ry, _rounding(dtype) * np.abs(ry) + (cond * (scale + g))[:, None])


def _check_norm_bwd(x, dy, gamma, mean, rstd, dres, dtype, out):
    dx, dgamma, dbeta = out
    rdx, rdg, rdb = ob.layer_norm_bwd(host(dy), host(x), host(gamma), host(mean), host(rstd),
                                      None if dres is None else host(dres))
    rs = host(rstd)[:, None]
    xh = np.abs((host(x) - host(mean)[:, None]) * rs)
    g = np.abs(host(dy) * host(gamma))
    # the terms of dx, and the roundings of s - mean inside xh
    terms = rs * (g + g.mean(1, keepdims=True) + xh * (g * xh).mean(1, keepdims=True))
    cond = REL + 8 * 2.0 ** -24 * (np.abs(host(x)).max(1) * host(rstd))[:, None]
    _check("dx", dx, rdx, _rounding(dtype) * np.abs(rdx) + cond * terms.max(1, keepdims=True))
    if dgamma is not None:
        _check("dgamma", dgamma, rdg, (cond * np.abs(host(dy)) * (xh + 1)).sum(0))
    if dbeta is not None:
        _check("dbeta", dbeta, rdb, REL * np.abs(host(dy)).sum(0))


NORM_SIZES = [(1, 8), (3, 16), (5, 72), (64, 128), (1, 2048), (257, 504), (65, 1000), (33, 2048),
              (130, 2056), (16, 2048), (17, 2048), (8, 4096), (17, 4096), (9, 4104), (5, 8192), (3, 16392), (1200, 256), (2500, 64)]


@pytest.mark.parametrize("T,d", NORM_SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layer_norm(T, d, dtype):
    case(f"layer norm T={T} d={d} {dtype}")
    x, res, dy, gamma, beta = _norm_inputs(T, d, dtype, 10 * T + d)
    _check_norm(x, res, gamma, beta, dtype, laep.moe_layer_norm(x, gamma, beta, residual=res))
    out = laep.moe_layer_norm(x, gamma)
    assert out[1] is x
    _check_norm(x, None, gamma, None, dtype, out)
    for dres, beta_too in ((res, True), (None, False)):
        got = laep.moe_layer_norm_bwd(dy, x, gamma, out[2], out[3], dres=dres,
                                      want_dbeta=beta_too)
        assert (got[2] is not None) == beta_too
        _check_norm_bwd(x, dy, gamma, out[2], out[3], dres, dtype, got)
    dx, dg, db = laep.moe_layer_norm_bwd(dy, x, gamma, out[2], out[3], weights=False)
    assert dg is None and db is None
    assert torch.equal(dx, got[0])


# widths of every number of waves a row may have, the last one partly filled; rows enough
# that a workgroup walks several
NORM_WIDTHS = [(1300, 776), (1300, 1224), (1300, 1496), (1300, 1544), (1300, 2504), (1300, 3000),
               (1300, 3528), (600, 5112), (600, 6000), (600, 7160), (300, 9000), (300, 12000),
               (300, 14000), (300, 15000), (1, 5112), (2, 14000)]


@pytest.mark.parametrize("T,d", NORM_WIDTHS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layer_norm_widths(T, d, dtype):
    case(f"layer norm T={T} d={d} {dtype}")
    x, res, dy, gamma, beta = _norm_inputs(T, d, dtype, 3 * T + d)
    out = laep.moe_layer_norm(x, gamma, beta, residual=res)
    _check_norm(x, res, gamma, beta, dtype, out)
    got = laep.moe_layer_norm_bwd(dy, out[1], gamma, out[2], out[3], dres=res)
    _check_norm_bwd(out[1], dy, gamma, out[2], out[3], res, dtype, got)
    # x and the residual's gradient written in place, by rows beside each other
    a, b = x.clone(), dy.clone()
    assert torch.equal(laep.moe_layer_norm(a, gamma, beta, residual=res, sum_out=a)[0], out[0])
    assert torch.equal(a, out[1])
    again = laep.moe_layer_norm_bwd(b, out[1], gamma, out[2], out[3], dres=res, dx=b)
    for p, q in zip(again, got):
        assert torch.equal(p, q)
    _check_norm(x, None, gamma, None, dtype, laep.moe_layer_norm(x, gamma))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [264, 2048, 8200, 16384])
def test_layer_norm_in_place(d, dtype):
    case(f"layer norm in place d={d} {dtype}")
    T = 37
    x, res, dy, gamma, beta = _norm_inputs(T, d, dtype, d)
    want = laep.moe_layer_norm(x, gamma, beta, residual=res)
    for target in ("x", "residual"):
        a, b = x.clone(), res.clone()
        got = laep.moe_layer_norm(a, gamma, beta, residual=b, sum_out=a if target == "x" else b)
        for p, q in zip(got, want):
            assert torch.equal(p, q)
    ref = laep.moe_layer_norm_bwd(dy, want[1], gamma, want[2], want[3], dres=res)
    for target in ("dy", "dres"):
        a, b = dy.clone(), res.clone()
        got = laep.moe_layer_norm_bwd(a, want[1], gamma, want[2], want[3], dres=b,
                                      dx=a if target == "dy" else b)
        for p, q in zip(got, ref):
            assert torch.equal(p, q)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layer_norm_common_offset_and_constant_rows(dtype):
    T, d = 20, 1032
    case(f"layer norm, rows with a large mean, {dtype}")
    x, _, dy, gamma, beta = _norm_inputs(T, d, dtype, 4, offset=300.0)
    x[3] = 2.5      # no spread: eps alone
    x[4] = 0.0
    out = laep.moe_layer_norm(x, gamma, beta, eps=1e-3)
    _check_norm(x, None, gamma, beta, dtype, out, eps=1e-3)
    assert torch.equal(out[0][3], beta.to(x.dtype)) and torch.equal(out[0][4], beta.to(x.dtype))
    _check_norm_bwd(x, dy, gamma, out[2], out[3], None, dtype,
                    laep.moe_layer_norm_bwd(dy, x, gamma, out[2], out[3]))


def test_layer_norm_keeps_bad_rows_to_themselves():
    T, d = 70, 520
    case("layer norm, an infinite and a NaN row")
    x, res, dy, gamma, beta = _norm_inputs(T, d, "bf16", 8)
    clean = laep.moe_layer_norm(x, gamma, beta)
    dclean = laep.moe_layer_norm_bwd(dy, x, gamma, clean[2], clean[3])[0]
    x[5, 7], x[66, 0] = float("inf"), float("nan")
    got = laep.moe_layer_norm(x, gamma, beta)
    dx = laep.moe_layer_norm_bwd(dy, x, gamma, got[2], got[3])[0]
    good = torch.ones(T, dtype=torch.bool, device="cuda")
    good[5] = good[66] = False
    assert torch.equal(got[0][good], clean[0][good]) and torch.equal(dx[good], dclean[good])
    assert got[0][5].isnan().all() and got[0][66].isnan().all()


def test_layer_norm_of_no_rows():
    case("layer norm T=0")
    x = torch.empty((0, 64), dtype=BF16, device="cuda")
    gamma = torch.ones(64, device="cuda")
    y, s, mean, rstd = laep.moe_layer_norm(x, gamma)
    assert y.shape == (0, 64) and mean.shape == (0,)
    dg, db = torch.full((64,), 5.0, device="cuda"), torch.full((64,), 5.0, device="cuda")
    dx, _, _ = laep.moe_layer_norm_bwd(x, x, gamma, mean, rstd, dgamma=dg, dbeta=db)
    assert dx.shape == (0, 64) and not dg.any() and not db.any()


# ---------------------------------------------------------------------------------------
# balance loss
# ---------------------------------------------------------------------------------------
def _balance_inputs(T, E, k, S, dead, seed):
    rng = np.random.default_rng(seed)
    logits = (1.5 * rng.standard_normal((T, E)) + rng.standard_normal(E)).astype(np.float32)
    alive = None
    if dead:
        alive = np.ones(E, np.uint8)
        alive[rng.permutation(E)[:dead]] = 0
    masked = logits if alive is None else np.where(alive, logits, -np.inf)
    idx = np.argsort(-masked, axis=1, kind="stable")[:, :k].astype(np.int32)
    if alive is not None:     # a dead expert's logit may hold anything
        for i, e in enumerate(np.nonzero(alive == 0)[0]):
            logits[:, e] = [np.nan, np.inf, -np.inf, np.finfo(np.float32).min][i % 4]
    off = None
    if S > 1:
        off = np.concatenate([[0], np.sort(rng.integers(0, T + 1, S - 1)), [T]]).astype(np.int32)
    return logits, idx, alive, off


def _check_balance(logits, idx, alive, off, coef, got, dloss=1.0):
    loss, counts, prob, grad = got
    rl, rc, rp, rg = ob.balance_loss(logits, idx, coef, alive, off)
    assert np.array_equal(host(counts), rc)
    _check("prob_mean", prob, rp, REL * rp)
    _check("grad_coef", grad, rg, REL * np.abs(rg))
    _check("loss", loss, [rl], REL * abs(rl))


def _check_balance_bwd(logits, alive, off, grad, got, dloss=1.0, add=0.0):
    ref = ob.balance_loss_bwd(logits, host(grad), dloss, alive, off) + add
    p = ob.alive_probs(logits, alive)
    bound = np.zeros_like(p)
    o = [0, len(logits)] if off is None else off
    for s in range(len(o) - 1):
        c = np.abs(host(grad)[s])
        q = p[o[s]:o[s + 1]]
        bound[o[s]:o[s + 1]] = q * (c + (q * c).sum(1, keepdims=True))
    _check("dlogits", got, ref, REL * abs(dloss) * bound + 2.0 ** -23 * np.abs(ref))


BALANCE = [(1, 1, 1, 1, 0), (1, 64, 8, 1, 0), (3, 2, 1, 1, 0), (8, 64, 8, 1, 0), (8, 64, 8, 5, 0),
           (63, 5, 2, 1, 0), (64, 8, 2, 3, 2), (65, 45, 8, 4, 0), (200, 33, 4, 1, 8),
           (129, 256, 8, 7, 64), (1000, 16, 2, 1, 0), (777, 100, 3, 40, 25), (513, 128, 8, 2, 0),
           (300, 255, 4, 1, 1), (128, 256, 4, 4, 0), (129, 256, 4, 4, 0),
           (512, 64, 8, 2, 8), (513, 64, 8, 2, 8), (8192, 4, 1, 3, 0), (2100, 64, 8, 1, 0), (5000, 7, 2, 33, 0), (4099, 64, 2, 600, 5)]


@pytest.mark.parametrize("T,E,k,S,dead", BALANCE)
def test_balance_loss(T, E, k, S, dead):
    case(f"balance loss T={T} E={E} k={k} sequences={S} dead={dead}")
    logits, idx, alive, off = _balance_inputs(T, E, k, S, dead, T + E)
    lt, it = dev(logits, F32), dev(idx, torch.int32)
    kw = dict(alive=None if alive is None else dev(alive, torch.uint8),
              seq_offsets=None if off is None else dev(off, torch.int32))
    got = laep.moe_balance_loss(lt, it, coef=0.02, **kw)
    _check_balance(logits, idx, alive, off, 0.02, got)
    again = laep.moe_balance_loss(lt, it, coef=0.02, **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    dl = laep.moe_balance_loss_bwd(lt, got[3], **kw)
    _check_balance_bwd(logits, alive, off, got[3], dl)
    if alive is not None:
        assert not dl[:, dev(1 - alive, torch.bool)].any()
    base = np.random.default_rng(0).standard_normal((T, E)).astype(np.float32)
    acc = laep.moe_balance_loss_bwd(lt, got[3], dloss=dev(np.array([-3.0], np.float32), F32),
                                    dlogits=dev(base, F32), accumulate=True, **kw)
    _check_balance_bwd(logits, alive, off, got[3], acc, -3.0, base.astype(np.float64))


# far more sequences than tokens, nearly all empty, and tokens of none before, between
# and after them
@pytest.mark.parametrize("T,E,S", [(1, 8, 300), (4, 64, 2000), (7, 45, 3), (300, 64, 5000)])
@pytest.mark.parametrize("gaps", [False, True])
def test_balance_empty_sequences(T, E, S, gaps):
    case(f"balance loss T={T} E={E} sequences={S} gaps={gaps}")
    logits, idx, _, off = _balance_inputs(T, E, 2, S, 0, T + S)
    if gaps:   # the first and the last token outside
        off = np.clip(off, min(1, T - 1), max(T - 1, 1)).astype(np.int32)
    lt, it, ot = dev(logits, F32), dev(idx, torch.int32), dev(off, torch.int32)
    got = laep.moe_balance_loss(lt, it, coef=0.02, seq_offsets=ot)
    _check_balance(logits, idx, None, off, 0.02, got)
    dl = laep.moe_balance_loss_bwd(lt, got[3], seq_offsets=ot)
    _check_balance_bwd(logits, None, off, got[3], dl)
    assert not dl[:off[0]].any() and not dl[off[-1]:].any()


@pytest.mark.parametrize("E", [3, 45, 64, 253])
def test_balance_gradient_in_place(E):
    T, k = 1500, 1
    case(f"balance gradient over the logits E={E}")
    logits, idx, _, off = _balance_inputs(T, E, k, 3, 0, E)
    lt, ot = dev(logits, F32), dev(off, torch.int32)
    grad = laep.moe_balance_loss(lt, dev(idx, torch.int32), seq_offsets=ot)[3]
    want = laep.moe_balance_loss_bwd(lt, grad, seq_offsets=ot)
    got = laep.moe_balance_loss_bwd(lt, grad, seq_offsets=ot, dlogits=lt)
    assert got is lt and torch.equal(got, want)


def test_balance_counts_match_the_layer():
    T, E, k = 1000, 64, 8
    case("balance loss, counts of a routed batch")
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((T, 256), generator=g, device="cuda").to(BF16)
    wr = (0.1 * torch.randn((E, 256), generator=g, device="cuda")).to(BF16)
    idx, _, logits = laep.moe_route(x, wr, k, want_logits=True)
    counts = laep.moe_balance_loss(logits, idx)[1]
    assert torch.equal(counts[0], laep.moe_expert_counts(idx, E)[0])


def test_balance_gradient_against_differences():
    T, E, k = 90, 12, 2
    case("balance loss, differences")
    logits, idx, alive, off = _balance_inputs(T, E, k, 4, 0, 5)
    ot = dev(off, torch.int32)
    coef = 64.0
    _, _, _, grad = laep.moe_balance_loss(dev(logits, F32), dev(idx, torch.int32), coef=coef,
                                          seq_offsets=ot)
    dl = host(laep.moe_balance_loss_bwd(dev(logits, F32), grad, seq_offsets=ot))
    step = 2.0 ** -5
    rng = np.random.default_rng(1)
    for _ in range(12):
        way = rng.standard_normal((T, E)).astype(np.float32)
        lo, hi = (host(laep.moe_balance_loss(dev(logits + s * way, F32), dev(idx, torch.int32),
                                             coef=coef, seq_offsets=ot)[0])[0]
                  for s in (-step, step))
        # loss ~ coef: float32 differences hold 1e-5 coef / step, truncation step^2 of the
        # third derivative (below coef |way|^3 ~ 30 coef)
        assert abs((hi - lo) / (2 * step) - (dl * way).sum()) <= \
            coef * (1e-5 / step + 30 * step ** 2 / 6)


def test_balance_rows_without_logits_and_tokens_of_no_sequence():
    T, E, k = 70, 40, 2
    case("balance loss, rows of -inf, unrouted slots, tokens of no sequence")
    logits, idx, _, _ = _balance_inputs(T, E, k, 1, 0, 9)
    logits[[0, 33, 69]] = -np.inf
    idx[[0, 33, 69]] = -1
    logits[7, :20] = -np.inf
    off = np.array([3, 3, 30, 60], np.int32)      # 0..2 and 60..69 belong to no sequence
    got = laep.moe_balance_loss(dev(logits, F32), dev(idx, torch.int32), coef=1.0,
                                seq_offsets=dev(off, torch.int32))
    _check_balance(logits, idx, None, off, 1.0, got)
    dl = laep.moe_balance_loss_bwd(dev(logits, F32), got[3], seq_offsets=dev(off, torch.int32))
    _check_balance_bwd(logits, None, off, got[3], dl)
    assert not dl[:3].any() and not dl[60:].any() and not dl[33].any()


def test_balance_nan_stays_in_its_sequence():
    T, E, k = 300, 64, 2
    case("balance loss, a NaN logit")
    logits, idx, _, off = _balance_inputs(T, E, k, 3, 0, 11)
    off = np.array([0, 100, 200, 300], np.int32)
    kw = dict(seq_offsets=dev(off, torch.int32))
    clean = laep.moe_balance_loss(dev(logits, F32), dev(idx, torch.int32), **kw)
    dclean = laep.moe_balance_loss_bwd(dev(logits, F32), clean[3], **kw)
    logits[150, 3] = np.nan
    got = laep.moe_balance_loss(dev(logits, F32), dev(idx, torch.int32), **kw)
    dl = laep.moe_balance_loss_bwd(dev(logits, F32), got[3], **kw)
    assert got[0].isnan().all() and got[2][1].isnan().all()
    assert torch.equal(got[2][[0, 2]], clean[2][[0, 2]]) and torch.equal(got[1], clean[1])
    keep = torch.arange(T, device="cuda") != 150
    assert torch.equal(dl[keep], dclean[keep]) and dl[150].isnan().all()


def test_balance_of_no_tokens_and_all_dead():
    case("balance loss T=0, and no alive expert")
    for off in (None, torch.zeros(4, dtype=torch.int32, device="cuda")):
        out = laep.moe_balance_loss(torch.empty((0, 8), device="cuda"),
                                    torch.empty((0, 2), dtype=torch.int32, device="cuda"),
                                    seq_offsets=off)
        assert all(not t.any() for t in out)
    logits = torch.randn((10, 8), device="cuda")
    dead = torch.zeros(8, dtype=torch.uint8, device="cuda")
    out = laep.moe_balance_loss(logits, torch.full((10, 2), -1, dtype=torch.int32, device="cuda"),
                                alive=dead)
    assert all(not t.any() for t in out)
    assert not laep.moe_balance_loss_bwd(logits, out[3], alive=dead).any()


def test_balance_on_another_stream():
    T, E, k = 5000, 64, 8
    case("balance loss and layer norm on a side stream")
    logits, idx, alive, off = _balance_inputs(T, E, k, 5, 0, 2)
    lt, it, ot = dev(logits, F32), dev(idx, torch.int32), dev(off, torch.int32)
    want = laep.moe_balance_loss(lt, it, seq_offsets=ot)
    x, res, dy, gamma, beta = _norm_inputs(500, 1024, "bf16", 1)
    wantn = laep.moe_layer_norm(x, gamma, beta, residual=res)
    wantb = laep.moe_layer_norm_bwd(dy, x, gamma, wantn[2], wantn[3])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = laep.moe_balance_loss(lt, it, seq_offsets=ot)
        gotn = laep.moe_layer_norm(x, gamma, beta, residual=res)
        gotb = laep.moe_layer_norm_bwd(dy, x, gamma, gotn[2], gotn[3])
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip((*want, *wantn, *wantb), (*got, *gotn, *gotb)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T,E,S", [(131072, 64, 1), (140000, 8, 3)])
def test_balance_long_batches(T, E, S):
    """Chunks at and past the limit of their number."""
    k = 2
    case(f"balance loss T={T} E={E}")
    logits, idx, alive, off = _balance_inputs(T, E, k, S, 0, 1)
    got = laep.moe_balance_loss(dev(logits, F32), dev(idx, torch.int32), coef=0.5,
                                seq_offsets=None if off is None else dev(off, torch.int32))
    p = ob.alive_probs(logits)
    o = [0, T] if off is None else off
    for s in range(len(o) - 1):
        a, b = o[s], o[s + 1]
        if a == b:
            continue
        assert np.array_equal(host(got[1])[s], np.bincount(idx[a:b].ravel(), minlength=E))
        ref = p[a:b].mean(0)
        assert (np.abs(host(got[2])[s] - ref) <= REL * ref).all()


# ---------------------------------------------------------------------------------------
# 8-bit checkpoints
# ---------------------------------------------------------------------------------------
def _act(R, C, dtype, seed):
    rng = np.random.default_rng(seed)
    sc = np.exp(3 * rng.standard_normal((R, C // 32))).repeat(32, 1)
    t = dev((rng.standard_normal((R, C)) * sc).astype(np.float32), DT[dtype])
    t[0, :32] = 0.0
    return t


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,C", [(1, 32), (1, 64), (3, 96), (7, 160), (65, 2048), (257, 4128),
                                 (1000, 736), (2, 16384)])
def test_act8_round_trip(R, C, dtype):
    case(f"act8 R={R} C={C} {dtype}")
    t = _act(R, C, dtype, R + C)
    q, b = laep.moe_act8_save(t)
    rq, rb = ob.act8_save(host(t))
    assert np.array_equal(host(b), rb) and np.array_equal(host(q), rq)
    ref = ob.act8_load(rq, rb)
    for dt in (BF16, F32):
        assert np.array_equal(host(laep.moe_act8_load(q, b, dt)), ref)   # exact in either


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_act8_special_values(dtype):
    case(f"act8 special values {dtype}")
    t = _act(40, 96, dtype, 3)
    big = float(torch.finfo(DT[dtype]).max)
    for r, v in enumerate([float("inf"), -float("inf"), float("nan"), big, -big, 2.0 ** -126,
                           2.0 ** -130, 2.0 ** -119, 127.5, 255.0, 1.0, -0.0]):
        t[r, 32 + r] = v
    t[12, 32:64] = 2.0 ** -130      # subnormal blocks
    t[13, 32:64] = 2.0 ** -121
    q, b = laep.moe_act8_save(t)
    rq, rb = ob.act8_save(host(t))
    assert np.array_equal(host(b), rb) and np.array_equal(host(q), rq)
    out, ref = host(laep.moe_act8_load(q, b, DT[dtype])), ob.act8_load(rq, rb)
    assert np.array_equal(out, ref, equal_nan=True)
    assert np.isnan(out[:3, 32:64]).all() and np.isfinite(out[3:]).all()
    assert np.isfinite(out[:3, :32]).all() and np.isfinite(out[:3, 64:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,f", [(1, 32), (5, 64), (129, 96), (64, 1024), (333, 2048), (2, 4128)])
def test_swiglu_bwd_act8(R, f, dtype):
    case(f"swiglu bwd act8 R={R} f={f} {dtype}")
    rng = np.random.default_rng(R + f)
    t = dev((3 * rng.standard_normal((R, 2 * f))).astype(np.float32), DT[dtype])
    dh = dev(rng.standard_normal((R, f)).astype(np.float32), DT[dtype])
    q, b = laep.moe_act8_save(t)
    da, h = laep.moe_swiglu_bwd_act8(q, b, dh)
    rda, rh = ob.swiglu_bwd_act8(host(q), host(b), host(dh))
    a = np.abs(ob.act8_load(host(q), host(b)))
    ag, au, d = a[:, :f], a[:, f:], np.abs(host(dh))
    terms = np.concatenate([d * au * (1 + ag), d * ag], 1)
    _check("da", da, rda, _rounding(dtype) * np.abs(rda) + REL * terms)
    _check("h", h, rh, _rounding(dtype) * np.abs(rh) + REL * ag * au)
    over = dh.clone()
    da2, h2 = laep.moe_swiglu_bwd_act8(q, b, over, h=over)     # H in dH's place
    assert h2 is over and torch.equal(da, da2) and torch.equal(h, h2)


def test_act8_past_32_bit_offsets():
    R, C = 1050000, 2048                      # 2.15 G elements
    case(f"act8 R={R} C={C}")
    t = torch.zeros((R, C), dtype=BF16, device="cuda")
    t[0], t[R - 1], t[R // 2 + 7] = 1.5, -3.0, 0.75
    t[R - 1, 5] = 100.0
    q, b = laep.moe_act8_save(t)
    out = laep.moe_act8_load(q, b)
    assert torch.equal(out[0], t[0]) and torch.equal(out[R // 2 + 7], t[R // 2 + 7])
    assert torch.equal(out[R - 1, 32:], t[R - 1, 32:]) and float(out[R - 1, 5]) == 100.0
    assert not out[1:1000].any() and not out[R - 1000:R - 1].any()
    del t, q, b, out
    torch.cuda.empty_cache()
