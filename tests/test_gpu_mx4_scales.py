"""The products at MX4 weights at scales near the ends of float32's range."""
import numpy as np
import pytest
import torch

import paper_2601_14327_amd as laep
from _gpu import case, dev, host
from oracle import mx4
from oracle.numerics import round_bf16
from test_gpu_mx4 import DT, _bound, _i32, _mx4, _routing

pytestmark = pytest.mark.gpu


def _operand(g, shape, exponents):
    """Random codes, the scale of each row one of the given biased exponents."""
    rows = shape[:-1]
    codes = g.integers(0, 256, size=rows + (shape[-1] // 2,)).astype(np.uint8)
    b = np.zeros(shape[:-2] + (-(-shape[-1] // 256), shape[-2], 8), np.uint8)
    row_b = g.choice(exponents, size=rows).astype(np.uint8)
    for c in range(shape[-1] // 32):
        b[..., c // 8, :, c % 8] = row_b
    return codes, b


@pytest.mark.parametrize("tile,T,E,N,K", [((32, 64), 60, 2, 128, 576), ((64, 128), 1000, 1, 2048, 576),
                                          ((128, 256), 8100, 20, 2048, 576)])
@pytest.mark.parametrize("x_b,w_b", [((127, 180, 240), (0, 1, 2)),    # weights below 2^-125
                                     ((0, 1, 2), (127, 180, 230)),    # activations
                                     ((200, 220, 230), (20, 40, 60))])
@pytest.mark.parametrize("act", [4, 16])
def test_scales_at_the_ends(tile, T, E, N, K, x_b, w_b, act):
    """Products of very small and very large values, their sums in the middle: as exact as
    any.  A sum or product below float32's normal numbers may be 0: 2^-126 each."""
    case(f"mx4 product tile={tile} T={T} E={E} N={N} K={K} act={act} scales {x_b} {w_b}")
    assert laep.laep_mx4_product_tile(T, E, N, K, act) == tile
    g = np.random.default_rng(T + x_b[0])
    row_src, offsets, _ = _routing(g, T, 1, E)
    qx, qw = _operand(g, (T, K), x_b), _operand(g, (E, N, K), w_b)
    xv = mx4.dequantize(*qx)
    assert np.array_equal(round_bf16(xv), xv)
    ref, mag = mx4.grouped_product(xv[row_src], mx4.dequantize(*qw), offsets)
    assert np.abs(ref).max() < 2.0 ** 125
    out = laep.moe_mx4_grouped_product(_mx4(qx) if act == 4 else dev(xv, torch.bfloat16), _mx4(qw),
                                       _i32(offsets), row_src=_i32(row_src), dtype=DT["f32"])
    err = np.abs(host(out) - ref)
    tol = _bound(mag, ref, K, "f32") + K * 2.0 ** -126
    assert (err <= tol).all(), (err / tol).max()
