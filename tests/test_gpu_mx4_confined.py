"""The products and the FFN at MX4 weights in every tile: a NaN spoils its own rows or
columns and nothing else.

A call with NaNs planted is compared with the same call without them, bit for bit, where
none may reach: the clean call's values are held to the oracle in test_gpu_mx4_tiles.py.
The bad rows are an expert's first, one in the middle and its last, so that they share
tiles with good rows, the last, ragged one among them; bad weights lie in the first and the
last column of a slot; an expert has no slot, and rows lie behind the last expert."""
import numpy as np
import pytest
import torch

import paper_2601_14327_amd as laep
from _gpu import case
from test_gpu_mx4 import DT, _ffn_check, _ffn_inputs, _i32, _mx4, _routing

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16

PRODUCTS = [   # rows and columns of the tiles; T, k, E, N, K
    ((32, 64), 90, 1, 4, 128, 576), ((64, 128), 1500, 2, 16, 1088, 704),
    ((128, 128), 2100, 3, 3, 1088, 192), ((128, 256), 4100, 2, 19, 2112, 1024),
    ((256, 256), 17000, 1, 4, 3584, 640)]
LEFT = 5       # rows behind the last expert's


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda").to(BF16)


def _layout(seed, T, k, E):
    """row_src and offsets of T k routed rows, the last LEFT of no expert; a map with
    expert 1 without a slot, the others' slots in another order."""
    row_src, offsets, _ = _routing(np.random.default_rng(seed), T, k, E, skew=0.5)
    offsets = np.minimum(offsets, T * k - LEFT)
    emap = np.array([E - 2 - (e - (e > 1)) for e in range(E)], np.int32)
    emap[1] = -1
    return row_src, offsets, emap


def _of_expert(offsets, e):
    rows = np.zeros(offsets[-1] + LEFT, bool)
    rows[offsets[e]:offsets[e + 1]] = True
    return rows


def _fullest(offsets, but):
    n = np.diff(offsets).copy()
    n[but] = 0
    return int(np.argmax(n))


def _bad_tokens(row_src, k, offsets, e):
    """Tokens of an expert's first, middle and last row; every routed row of them."""
    a, b = offsets[e], offsets[e + 1]
    tokens = np.unique(row_src[[a, (a + b) // 2, b - 1]] // k)
    return tokens, np.isin(row_src // k, tokens)


def _poisoned(w, slot, rows, block):
    """w with a block of the given rows of a slot not finite."""
    codes, scale = w.codes.clone(), w.scale.clone()
    scale[slot, block // 8, rows, block % 8] = 255
    return laep.Mx4(codes, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", [4, 16])
@pytest.mark.parametrize("tile,T,k,E,N,K", PRODUCTS)
def test_product(tile, T, k, E, N, K, act, dtype):
    case(f"mx4 product, NaNs confined, tile={tile} T={T} k={k} E={E} N={N} K={K} act={act} {dtype}")
    assert laep.laep_mx4_product_tile(T * k, E, N, K, act) == tile
    g = torch.Generator(device="cuda").manual_seed(T + N)
    row_src, offsets, emap = _layout(T, T, k, E)
    x, w = _normal(g, T, K), laep.moe_mx4_quantize(_normal(g, E - 1, N, K) * 0.05)
    kw = dict(expert_map=_i32(emap), dtype=DT[dtype])

    def run(x, w, ordered=False):
        out = torch.full((T * k, N), 7.0, dtype=DT[dtype], device="cuda")
        if ordered:
            x = x[torch.from_numpy(row_src // k).cuda()]
        a = laep.moe_mx4_quantize(x) if act == 4 else x
        how = {} if ordered else dict(row_src=_i32(row_src), k=k)
        laep.moe_mx4_grouped_product(a, w, _i32(offsets), out=out, **how, **kw)
        return out

    clean = run(x, w)
    assert torch.isfinite(clean).all()
    left = _of_expert(offsets, 1)
    left[offsets[-1]:] = True
    assert (clean[torch.from_numpy(left).cuda()] == 7.0).all()
    # rows
    e = _fullest(offsets, 1)
    tokens, rows = _bad_tokens(row_src, k, offsets, e)
    x2 = x.clone()
    x2[tokens[0], 33] = float("nan")
    x2[tokens[1:], K - 1] = float("nan")
    bad = torch.from_numpy(rows & ~left).cuda()
    for ordered in (False, True):
        got = run(x2, w, ordered)
        assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], clean[~bad])
    # weights: a block of the first and the last column's rows
    cols = torch.tensor([0, N - 1], device="cuda")
    got = run(x, _poisoned(w, int(emap[e]), cols, K // 32 - 1))
    nan = torch.zeros_like(got, dtype=torch.bool)
    nan[offsets[e]:offsets[e + 1], cols] = True
    assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], clean[~nan])


FFNS = [   # the two products' tiles; T, k, E, d, f
    ((32, 64), (32, 64), 90, 1, 4, 192, 320), ((64, 128), (64, 128), 1500, 2, 2, 576, 448),
    ((128, 128), (64, 128), 3200, 2, 2, 320, 704),
    ((128, 256), (128, 256), 1000, 8, 20, 1088, 1024),
    ((256, 256), (128, 256), 16500, 2, 2, 576, 1024)]


@pytest.mark.parametrize("act", [4, 16])
@pytest.mark.parametrize("gate_up,down,T,k,E,d,f", FFNS)
def test_ffn(gate_up, down, T, k, E, d, f, act):
    case(f"mx4 ffn, NaNs confined, tiles={gate_up}, {down} T={T} k={k} E={E} d={d} f={f} act={act}")
    assert laep.laep_mx4_ffn_tile(T * k, E, d, f, act) == gate_up
    assert laep.laep_mx4_ffn_tile(T * k, E, d, f, act, down=True) == down
    g = torch.Generator(device="cuda").manual_seed(T + d)
    row_src, offsets, _ = _routing(np.random.default_rng(T), T, k, E, skew=0.5)
    offsets = np.minimum(offsets, T * k - LEFT)
    x = _normal(g, T, d)
    gu = laep.moe_mx4_quantize(_normal(g, E, 2 * f, d) * d ** -0.5)
    dn = laep.moe_mx4_quantize(_normal(g, E, d, f) * f ** -0.5)

    def run(x, gu, dn):
        y = torch.full((T * k, d), 7.0, dtype=BF16, device="cuda")
        laep.moe_grouped_ffn_fwd_mx4(x, gu, dn, _i32(offsets), row_src=_i32(row_src), k=k,
                                     act_bits=act, y_perm=y)
        return y

    def holds(got, nan):
        assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], clean[~nan])

    clean = run(x, gu, dn)
    assert torch.isfinite(clean).all() and (clean[offsets[-1]:] == 7.0).all()
    none = torch.zeros_like(clean, dtype=torch.bool)
    e = _fullest(offsets, [])
    tokens, rows = _bad_tokens(row_src, k, offsets, e)
    rows[offsets[-1]:] = False
    x2 = x.clone()
    x2[tokens, d - 1] = float("nan")
    nan = none.clone()
    nan[torch.from_numpy(rows).cuda()] = True
    holds(run(x2, gu, dn), nan)
    # a gate and an up row: H has a NaN in each of the expert's rows
    nan = none.clone()
    nan[offsets[e]:offsets[e + 1]] = True
    for row in (0, 2 * f - 1):
        holds(run(x, _poisoned(gu, e, row, d // 32 - 1), dn), nan)
    nan = none.clone()
    nan[offsets[e]:offsets[e + 1], d - 1] = True
    holds(run(x, gu, _poisoned(dn, e, d - 1, f // 32 - 1)), nan)


@pytest.mark.parametrize("act", [4, 16])
@pytest.mark.parametrize("tiles,T,k,E,dead,d,f", [
    (((32, 64), (32, 64)), 200, 2, 4, 1, 448, 256),
    (((64, 128), (64, 128)), 1500, 2, 2, 0, 576, 448),
    (((128, 256), (128, 256)), 1000, 8, 20, 0, 1088, 1024)])
def test_ffn_is_close_as_a_whole(tiles, T, k, E, dead, d, f, act):
    """Far below the worst case of every element.  y's rounding is at most 2^-8 of a value.
    An H that rounds the other way lies within its float32 error of a border: the error, a
    random walk of d steps of 2^-24, is below 1e-5 of the value, so at most 1e-4 of the
    values do, each by at most half of itself (the largest step of 4-bit values), sqrt(1e-4)
    / 2 as a whole: in all 2^-8 + 0.005 < 0.01."""
    case(f"mx4 ffn as a whole tiles={tiles} T={T} k={k} E={E} d={d} f={f} act={act}")
    assert tuple(laep.laep_mx4_ffn_tile(T * k, E, d, f, act, down=b) for b in (0, 1)) == tiles
    x, row_src, offsets, emap, gu, dn = _ffn_inputs(T + d + f, T, k, E, dead, d, f)
    y, _ = laep.moe_grouped_ffn_fwd_mx4(torch.from_numpy(x).cuda().to(BF16), _mx4(gu), _mx4(dn),
                                        _i32(offsets), row_src=_i32(row_src), k=k, act_bits=act,
                                        expert_map=_i32(emap))
    assert _ffn_check(y, x, row_src, offsets, emap, gu, dn, k, act) < 0.01
