"""Experts in microscaled 4 bits against the float64 oracle.

Quantisation is exact: codes and scales are compared bit for bit.  Products: every
product of two MX4 values, and of an MX4 and a bf16 value, is exact in float32 (at most 2
+ 8 significant bits), so a sum of K of them errs by at most K roundings of partial sums
below S = sum |x w|: K 2^-24 S, and the output's rounding by half a step.
"""
import numpy as np
import pytest
import torch

import paper_2601_14327_amd as laep
from _gpu import case, dev, host
from oracle import mx4
from oracle.numerics import round_bf16, sigmoid, silu

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}     # half a step, relative


def _round(a, dtype):
    return round_bf16(a) if dtype == "bf16" else np.asarray(a, np.float32).astype(np.float64)


# ---- quantisation --------------------------------------------------------------------
def _special(g, shape, dtype):
    """Values over the whole range of exponents, with zeros, ties, and blocks that hold
    infinities and NaNs."""
    x = g.normal(size=shape) * np.ldexp(1.0, g.integers(-120, 120, size=shape[:-1] + (1,)))
    flat = x.reshape(-1, 32)
    n = flat.shape[0]
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.96875, -0.25, -5.0])
    for i in range(n):
        kind = g.integers(0, 12)
        if kind == 0:
            flat[i] = 0.0
        elif kind == 1:
            flat[i] = g.choice(ties, 32) * np.ldexp(1.0, int(g.integers(-120, 120)))
        elif kind == 2:
            flat[i, g.integers(0, 32)] = g.choice([np.inf, -np.inf, np.nan])
        elif kind == 3:                                  # below the normal numbers
            flat[i] = g.normal(size=32) * 2.0 ** -128
        elif kind == 4:                                  # the largest
            flat[i] = g.choice([1.9921875, -1.5, 1.0], 32) * 2.0 ** 127
        elif kind == 5:
            flat[i] = 0.0
            flat[i, 31] = -2.0 ** -133
    return _round(x, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1, 32), (3, 64), (17, 256), (33, 288), (2, 5, 1056),
                                   (16, 992), (3, 2, 31, 512), (1000, 96)])
def test_quantize_is_the_definition(shape, dtype):
    case(f"mx4 quantize {shape} {dtype}")
    x = _special(np.random.default_rng(len(shape) * 1000 + shape[-1]), shape, dtype)
    codes, scale = laep.moe_mx4_quantize(dev(x, DT[dtype]))
    rc, rs = mx4.quantize(x)
    assert np.array_equal(host(scale), rs)
    assert np.array_equal(host(codes), rc)
    want = mx4.dequantize(rc, rs)
    for out in ("bf16", "f32"):
        got = host(laep.moe_mx4_dequantize(codes, scale, DT[out]))
        assert np.array_equal(got, want, equal_nan=True)


def test_dequantize_every_code_at_every_scale():
    case("mx4 dequantize all codes and scales")
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))[:, :].copy()      # 512 columns
    scale = np.repeat(np.arange(256, dtype=np.uint8)[None, :, None], 2, 0).repeat(8, 2).copy()
    want = mx4.dequantize(codes, scale)
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)  # b 253, 254
    for out in ("bf16", "f32"):
        got = host(laep.moe_mx4_dequantize(torch.from_numpy(codes).cuda(),
                                           torch.from_numpy(scale).cuda(), DT[out]))
        assert np.array_equal(got, want, equal_nan=True)


def test_no_rows_and_given_buffers():
    case("mx4 quantize, no rows; given buffers")
    e = laep.moe_mx4_quantize(torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"))
    assert e.codes.shape == (0, 32) and e.scale.shape == (1, 0, 8)
    assert laep.moe_mx4_dequantize(*e).shape == (0, 64)
    x = torch.randn((7, 320), device="cuda")
    codes = torch.full((7, 160), 0xAA, dtype=torch.uint8, device="cuda")
    scale = torch.full((2, 7, 8), 0xFF, dtype=torch.uint8, device="cuda")
    q = laep.moe_mx4_quantize(x, codes=codes, scale=scale)
    assert q.codes is codes and q.scale is scale and (scale[1, :, 2:] == 0).all()
    out = torch.empty_like(x)
    assert laep.moe_mx4_dequantize(*q, torch.float32, out=out) is out
    assert np.array_equal(host(out), mx4.dequantize(*mx4.quantize(host(x))))


def test_quantize_past_2_to_the_31_elements():
    """Rows beyond 2^31 elements equal a small call's of the same rows."""
    case("mx4 quantize of 2^31 + elements")
    R, C = 2_100_000, 1056
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty((R, C), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    codes, scale = laep.moe_mx4_quantize(x)
    for lo, hi in ((0, 40), (R // 2, R // 2 + 40), (R - 40, R)):
        q = laep.moe_mx4_quantize(x[lo:hi].contiguous())
        assert torch.equal(codes[lo:hi], q.codes) and torch.equal(scale[:, lo:hi], q.scale)
        y = laep.moe_mx4_dequantize(codes[lo:hi].contiguous(), scale[:, lo:hi].contiguous())
    out = laep.moe_mx4_dequantize(codes, scale, out=x)
    assert torch.equal(out[R - 40:], y)


# ---- routing ----------------------------------------------------------------------------
def _routing(g, T, k, E, dead=0, skew=0.7):
    """(row_src [T k], offsets [E + 1], expert_map [E] or None), experts' loads uneven."""
    logits = g.normal(size=(T, E)) + g.normal(size=E) * skew
    gone = g.permutation(E)[:dead]
    logits[:, gone] = -np.inf
    idx = np.argsort(-logits, axis=1, kind="stable")[:, :k].reshape(-1)
    row_src = np.argsort(idx, kind="stable").astype(np.int32)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(idx, minlength=E))]).astype(np.int32)
    emap = None
    if dead:
        alive = np.ones(E, bool)
        alive[gone] = False
        emap = np.where(alive, np.cumsum(alive) - 1, -1).astype(np.int32)
        # (slots in another order than the experts)
        emap = np.where(emap >= 0, alive.sum() - 1 - emap, -1).astype(np.int32)
    return row_src, offsets, emap


def _i32(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _mx4(q):
    return laep.Mx4(torch.from_numpy(q[0]).cuda(), torch.from_numpy(q[1]).cuda())


def _bound(mag, ref, K, dtype):
    return K * 2.0 ** -24 * mag + HALF[dtype] * (np.abs(ref) + K * 2.0 ** -24 * mag) + 1e-38


SIZES = [   # T, k, E, dead, N, K
    (1, 1, 1, 0, 64, 64), (1, 1, 1, 0, 192, 128), (3, 1, 2, 0, 64, 320), (33, 1, 1, 0, 128, 256),
    (8, 1, 1, 0, 256, 2048), (1, 8, 16, 0, 320, 448), (16, 4, 8, 2, 192, 576),
    (70, 2, 5, 1, 448, 192), (200, 2, 3, 0, 320, 960), (129, 1, 1, 0, 128, 1088),
    (513, 1, 1, 0, 576, 512), (700, 4, 12, 3, 256, 1216), (1100, 2, 4, 0, 1088, 768),
    (64, 2, 128, 0, 64, 704), (40, 8, 256, 100, 128, 64), (3000, 2, 7, 1, 640, 320),
    # past 256 rows an expert and 576 columns: the 256 x 256 tiles
    (700, 1, 2, 0, 64, 576), (1400, 2, 5, 1, 704, 640), (2100, 1, 1, 0, 320, 1216),
    (1500, 4, 9, 3, 256, 1024), (9000, 1, 30, 2, 576, 832)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", [4, 16])
@pytest.mark.parametrize("T,k,E,dead,N,K", SIZES)
def test_grouped_product(T, k, E, dead, N, K, act, dtype):
    case(f"mx4 product T={T} k={k} E={E} dead={dead} N={N} K={K} act={act} {dtype}")
    g = np.random.default_rng(T * 7 + N + K)
    row_src, offsets, emap = _routing(g, T, k, E, dead)
    x = round_bf16(g.normal(size=(T, K)) * np.exp(g.normal(size=(T, 1))))
    qw = mx4.quantize(g.normal(size=(E - dead, N, K)) * 0.05)
    qx = mx4.quantize(x)
    xv = mx4.dequantize(*qx) if act == 4 else x
    ref, mag = mx4.grouped_product(xv[row_src // k], mx4.dequantize(*qw), offsets, emap)
    out = laep.moe_mx4_grouped_product(_mx4(qx) if act == 4 else dev(x, torch.bfloat16), _mx4(qw),
                                       _i32(offsets), row_src=_i32(row_src), k=k,
                                       expert_map=_i32(emap), dtype=DT[dtype])
    err = np.abs(host(out) - ref)
    assert (err <= _bound(mag, ref, K, dtype)).all(), (err / _bound(mag, ref, K, dtype)).max()
    # the rows already in the experts' order give the same bits
    rows = xv[row_src // k]
    own = _mx4(mx4.quantize(rows)) if act == 4 else dev(rows, torch.bfloat16)
    again = laep.moe_mx4_grouped_product(own, _mx4(qw), _i32(offsets), expert_map=_i32(emap),
                                         dtype=DT[dtype])
    assert torch.equal(again, out)


@pytest.mark.parametrize("act", [4, 16])
@pytest.mark.parametrize("T,N,K", [(5, 192, 320), (300, 128, 320), (2000, 256, 448),
                                   (2000, 320, 704)])
def test_rows_left_as_they_were_and_nans_confined(T, N, K, act):
    """Rows of experts without a slot, and behind the last expert, keep what they held; a
    row with a NaN, and an expert whose weights hold one, spoil nothing else."""
    case(f"mx4 product: rows left, NaNs, T={T} act={act}")
    g = np.random.default_rng(T)
    E, k = 6, 1
    row_src, offsets, _ = _routing(g, T, k, E, skew=0.0)
    offsets = np.minimum(offsets, T - 2).astype(np.int32)       # two rows behind the last
    emap = np.array([2, -1, 0, 1, -1, 3], np.int32)
    x = round_bf16(g.normal(size=(T, K)))
    bad_row = int(row_src[offsets[2]]) if offsets[3] > offsets[2] else 0
    x[bad_row, 33] = np.nan
    w = g.normal(size=(4, N, K)) * 0.05
    w[1, 7, 40] = np.inf
    qw, qx = mx4.quantize(w), mx4.quantize(x)
    ref, mag = mx4.grouped_product((mx4.dequantize(*qx) if act == 4 else x)[row_src],
                                   mx4.dequantize(*qw), offsets, emap)
    out = torch.full((T, N), 7.0, dtype=torch.float32, device="cuda")
    laep.moe_mx4_grouped_product(_mx4(qx) if act == 4 else dev(x, torch.bfloat16), _mx4(qw),
                                 _i32(offsets), row_src=_i32(row_src), k=k, expert_map=_i32(emap),
                                 dtype=torch.float32, out=out)
    got = host(out)
    left = np.zeros(T, bool)
    left[offsets[-1]:] = True
    for e in (1, 4):
        left[offsets[e]:offsets[e + 1]] = True
    assert (got[left] == 7.0).all()
    live = got[~left]
    r, m = ref[~left], mag[~left]
    assert np.array_equal(np.isnan(live), np.isnan(r))
    ok = ~np.isnan(r)
    assert (np.abs(live - r)[ok] <= _bound(m, r, K, "f32")[ok]).all()


# ---- the FFN ------------------------------------------------------------------------------
def _ffn_inputs(seed, T, k, E, dead, d, f):
    g = np.random.default_rng(seed)
    row_src, offsets, emap = _routing(g, T, k, E, dead)
    x = round_bf16(g.normal(size=(T, d)))
    gu = mx4.quantize(g.normal(size=(E - dead, 2 * f, d)) / np.sqrt(d))
    dn = mx4.quantize(g.normal(size=(E - dead, d, f)) / np.sqrt(f))
    return x, row_src, offsets, emap, gu, dn


def _ffn_check(y, x, row_src, offsets, emap, gu, dn, k, act, act_save=None):
    """Against the oracle, allowing for H whatever A's float32 sums can do to its rounding:
    where H and the same H moved by its error round alike, nothing."""
    d, f = x.shape[1], dn[0].shape[-1] * 2
    xv = mx4.dequantize(*mx4.quantize(x)) if act == 4 else x
    A, mag = mx4.grouped_product(xv[row_src // k], mx4.dequantize(*gu), offsets, emap)
    eA = d * 2.0 ** -24 * mag
    if act_save is not None:
        err = np.abs(host(act_save) - A)
        assert (err <= _bound(mag, A, d, "bf16")).all()
    a, u, ea, eu = A[:, :f], A[:, f:], eA[:, :f], eA[:, f:]
    h = silu(a) * u
    # |silu'| <= 1.1; sigmoid by hardware exp2 and reciprocal: relative (|a| + 4) 2^-23
    eh = (1.1 * ea * (np.abs(u) + eu) + np.abs(silu(a)) * eu + np.abs(h) * (np.abs(a) + 4) * 2.0 ** -23
          + np.abs(h) * 2.0 ** -22)
    if act == 16:
        hq, lo, hi = round_bf16(h), round_bf16(h - eh), round_bf16(h + eh)
        eq = np.maximum(np.abs(hi - hq), np.abs(hq - lo))
    else:
        def rounded(v, b):
            q = np.ldexp(v, 127 - b)
            c = mx4.nearest_code(q)
            return np.ldexp(np.where(c & 8, -1.0, 1.0) * mx4.STEPS[c & 7], b - 127)

        hb, eb = h.reshape(-1, f // 32, 32), eh.reshape(-1, f // 32, 32)
        amax, far = np.abs(hb).max(-1), eb.max(-1)
        b, blo, bhi = (mx4.exponent_of(v)[..., None] for v in
                       (amax, np.maximum(amax - far, 0), amax + far))
        hq = rounded(hb, b)
        eq = np.maximum(np.abs(rounded(hb + eb, b) - hq), np.abs(hq - rounded(hb - eb, b)))
        # the block's scale itself may go either way: one of its larger steps
        eq = np.where(blo != bhi, np.ldexp(2.0, np.maximum(b, bhi) - 127), eq)
        hq, eq = hq.reshape(h.shape), eq.reshape(h.shape)
    wd = mx4.dequantize(*dn)
    ref, m2 = mx4.grouped_product(hq, wd, offsets, emap)
    _, slack = mx4.grouped_product(eq, wd, offsets, emap)
    tol = _bound(m2 + slack, ref, f, "bf16") + slack * (1 + 2.0 ** -8)
    got = host(y)
    live = ~np.isnan(ref)
    assert (np.abs(got - ref)[live] <= tol[live]).all(), np.nanmax((np.abs(got - ref) / tol)[live])
    # and far closer than the worst case as a whole
    rel = np.linalg.norm((got - ref)[live]) / max(np.linalg.norm(ref[live]), 1e-30)
    return rel


FFN_SIZES = [   # T, k, E, dead, d, f
    (1, 1, 1, 0, 64, 64), (1, 8, 16, 0, 256, 192), (3, 2, 4, 1, 320, 64), (16, 4, 12, 3, 512, 320),
    (40, 2, 3, 0, 192, 448), (200, 2, 4, 1, 448, 256), (600, 4, 6, 0, 256, 576),
    (1500, 1, 3, 1, 320, 192), (1000, 8, 16, 0, 128, 128), (9, 3, 200, 50, 64, 128),
    # the 256 x 256 tiles
    (600, 2, 3, 0, 576, 640), (1200, 1, 4, 1, 704, 576), (900, 2, 4, 0, 1024, 832)]


@pytest.mark.parametrize("act", [4, 16])
@pytest.mark.parametrize("T,k,E,dead,d,f", FFN_SIZES)
def test_grouped_ffn(T, k, E, dead, d, f, act):
    case(f"mx4 ffn T={T} k={k} E={E} dead={dead} d={d} f={f} act={act}")
    x, row_src, offsets, emap, gu, dn = _ffn_inputs(T + d + f, T, k, E, dead, d, f)
    kw = dict(row_src=_i32(row_src), k=k, act_bits=act, expert_map=_i32(emap))
    args = (dev(x, torch.bfloat16), _mx4(gu), _mx4(dn), _i32(offsets))
    y, a = laep.moe_grouped_ffn_fwd_mx4(*args, save_act=act == 16, **kw)
    _ffn_check(y, x, row_src, offsets, emap, gu, dn, k, act, a)
    # a workspace that held NaNs, and none of the pre-activations: the same bits
    ws = torch.full((laep.workspace_bytes(laep.LAEP_CALL_MX4_FFN, T, k, E, d, f),), 0xFF,
                    dtype=torch.uint8, device="cuda")
    y2, none = laep.moe_grouped_ffn_fwd_mx4(*args, ws=ws, **kw)
    assert none is None and torch.equal(y, y2)
    # rows already in the experts' order
    y3, _ = laep.moe_grouped_ffn_fwd_mx4(dev(x[row_src // k], torch.bfloat16), *args[1:],
                                         act_bits=act, expert_map=_i32(emap))
    assert torch.equal(y, y3)


@pytest.mark.parametrize("act", [4, 16])
def test_no_tokens(act):
    case(f"mx4 ffn of no tokens, act={act}")
    _, _, _, _, gu, dn = _ffn_inputs(0, 1, 1, 4, 0, 64, 64)
    off = torch.zeros(5, dtype=torch.int32, device="cuda")
    src = torch.zeros(0, dtype=torch.int32, device="cuda")
    x = torch.zeros((0, 64), dtype=torch.bfloat16, device="cuda")
    y, _ = laep.moe_grouped_ffn_fwd_mx4(x, _mx4(gu), _mx4(dn), off, row_src=src, act_bits=act)
    assert y.shape == (0, 64)
    # tokens, but none of them routed
    y = torch.full((4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    laep.moe_grouped_ffn_fwd_mx4(torch.ones((4, 64), dtype=torch.bfloat16, device="cuda"),
                                 _mx4(gu), _mx4(dn), off, act_bits=act, y_perm=y)
    assert (y == 3.0).all()


def test_quantisation_aware_gradients():
    """The gradients at the MX4 weights' values and the kept pre-activations: those of the
    16-bit layer at the same values, and differences of the oracle."""
    case("mx4 ffn gradients")
    T, k, E, d, f = 48, 2, 4, 128, 192
    x, row_src, offsets, _, gu, dn = _ffn_inputs(77, T, k, E, 0, d, f)
    xt, src, off = dev(x, torch.bfloat16), _i32(row_src), _i32(offsets)
    y, a = laep.moe_grouped_ffn_fwd_mx4(xt, _mx4(gu), _mx4(dn), off, row_src=src, k=k,
                                        save_act=True)
    wg, wd = laep.moe_mx4_dequantize(*_mx4(gu)), laep.moe_mx4_dequantize(*_mx4(dn))
    y16, a16 = laep.moe_grouped_ffn_fwd_gather(xt, src, k, wg, wd, off, save_act=True)
    g = np.random.default_rng(5)
    dyv = round_bf16(g.normal(size=(T * k, d)))
    dy = dev(dyv, torch.bfloat16)
    dx, dgu, ddn = laep.moe_grouped_ffn_bwd_gather(dy, xt, src, k, a, wg, wd, off)
    # float64: loss = sum dy y; gradients by the chain rule over float64 arrays
    wgv, wdv = mx4.dequantize(*gu), mx4.dequantize(*dn)

    def loss(wgv, wdv, rows):
        A, _ = mx4.grouped_product(rows, wgv, offsets)
        Y, _ = mx4.grouped_product(mx4.swiglu(A), wdv, offsets)
        return (dyv * Y).sum()

    rows = x[row_src // k]
    for arr, grad, which in ((wgv, host(dgu), 0), (wdv, host(ddn), 1), (rows, host(dx), 2)):
        scale = np.abs(grad).max()
        for _ in range(12):
            at = tuple(g.integers(0, n) for n in arr.shape)
            eps = 1e-4
            v = []
            for sgn in (1, -1):
                p = arr.copy()
                p[at] += sgn * eps
                v.append(loss(*((p, wdv, rows) if which == 0 else (wgv, p, rows) if which == 1
                                else (wgv, wdv, p))))
            # dA, H, A and dX are bf16: four roundings of 2^-8 on sums of many terms
            assert abs((v[0] - v[1]) / (2 * eps) - grad[at]) <= 4 * 2.0 ** -8 * scale


# ---- streams and graphs --------------------------------------------------------------------
@pytest.mark.parametrize("act", [4, 16])
@pytest.mark.parametrize("T,d,f", [(2, 256, 192), (700, 256, 192), (700, 576, 640)])
def test_captured_and_on_another_stream(T, d, f, act):
    case(f"mx4 ffn in a graph, T={T} d={d} f={f} act={act}")
    k, E = 2, 4
    sets = [_ffn_inputs(s, T, k, E, 0, d, f) for s in (1, 2)]
    gu, dn = _mx4(sets[0][4]), _mx4(sets[0][5])
    ws = torch.empty(laep.workspace_bytes(laep.LAEP_CALL_MX4_FFN, T, k, E, d, f),
                     dtype=torch.uint8, device="cuda")
    xs = [dev(s[0], torch.bfloat16) for s in sets]
    srcs, offs = [_i32(s[1]) for s in sets], [_i32(s[2]) for s in sets]
    eager = [laep.moe_grouped_ffn_fwd_mx4(x, gu, dn, o, row_src=r, k=k, act_bits=act, ws=ws)[0]
             for x, r, o in zip(xs, srcs, offs)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = laep.moe_grouped_ffn_fwd_mx4(xs[0], gu, dn, offs[0], row_src=srcs[0], k=k,
                                             act_bits=act, ws=ws)[0]
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other, eager[0])
    # two graphs share the workspace; replayed in turn, with eager work between
    x, src, off = xs[0].clone(), srcs[0].clone(), offs[0].clone()
    ys = [torch.empty_like(eager[0]) for _ in range(2)]
    graphs = []
    for y in ys:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            laep.moe_grouped_ffn_fwd_mx4(x, gu, dn, off, row_src=src, k=k, act_bits=act, ws=ws,
                                         y_perm=y)
        graphs.append(graph)
    for i in range(6):
        w = i % 2 ^ i // 3
        x.copy_(xs[w]), src.copy_(srcs[w]), off.copy_(offs[w])
        ys[i % 2].zero_()
        graphs[i % 2].replay()
        assert torch.equal(ys[i % 2], eager[w])
        laep.moe_grouped_ffn_fwd_mx4(xs[1 - w], gu, dn, offs[1 - w], row_src=srcs[1 - w], k=k,
                                     act_bits=act, ws=ws)
        torch.cuda.synchronize()
