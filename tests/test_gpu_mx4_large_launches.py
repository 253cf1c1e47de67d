"""Products at MX4 weights of more workgroups than one grid dimension holds."""
import numpy as np
import pytest
import torch

import paper_2601_14327_amd as laep
from _gpu import case, dev, host
from oracle import mx4
from oracle.numerics import round_bf16
from test_gpu_mx4 import _bound, _i32, _mx4

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act,tile,R,N", [(4, (32, 64), 256, 1 << 22), (16, (32, 64), 256, 1 << 22),
                                          (4, (64, 128), 1800, 1 << 23)])
def test_more_workgroups_than_one_grid_dimension_holds(act, tile, R, N):
    """Past 2^24 workgroups of 256 threads: every row of every column is written."""
    case(f"mx4 product of many tiles act={act} tile={tile} R={R} N={N}")
    E, K = 256, 64
    assert laep.laep_mx4_product_tile(R, E, N, K, act) == tile
    assert (R // tile[0] + E) * (N // tile[1]) > 1 << 24
    g = np.random.default_rng(R + act)
    offsets = np.sort(g.choice(R - 1, E - 1, replace=False) + 1)
    offsets = np.concatenate([[0], offsets, [R]]).astype(np.int32)
    x = round_bf16(g.normal(size=(R, K)))
    qx = mx4.quantize(x)
    w = laep.Mx4(torch.randint(0, 256, (1, N, K // 2), dtype=torch.uint8, device="cuda"),
                 torch.zeros((1, 1, N, 8), dtype=torch.uint8, device="cuda"))
    w.scale[..., :2] = torch.randint(120, 128, (1, 1, N, 2), dtype=torch.uint8, device="cuda")
    out = torch.full((R, N), float("nan"), dtype=torch.bfloat16, device="cuda")
    laep.moe_mx4_grouped_product(_mx4(qx) if act == 4 else dev(x, torch.bfloat16), w, _i32(offsets),
                                 expert_map=_i32(np.zeros(E, np.int32)), out=out)
    xv = mx4.dequantize(*qx) if act == 4 else x
    for n in (0, N // 2, N - 64):
        wv = mx4.dequantize(host(w.codes[0, n:n + 64]), host(w.scale[0, :, n:n + 64]))
        ref, mag = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
        assert (np.abs(host(out[:, n:n + 64]) - ref) <= _bound(mag, ref, K, "bf16")).all()
    for rows in out.split(64):
        assert torch.isfinite(rows).all()
    del out, w
    torch.cuda.empty_cache()
