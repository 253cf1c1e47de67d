"""Calls of more workgroups than one grid dimension holds (2^32 threads): every output is
written."""
import pytest
import torch

import paper_2601_14327_amd as laep
from _gpu import case

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _last_rows(T, d):
    """Zeros, 1 to 3 in the last three rows."""
    x = torch.zeros((T, d), dtype=BF16, device="cuda")
    x[-3:] = torch.arange(1.0, 4.0, device="cuda")[:, None].to(BF16)
    return x


def _nan(*shape, dtype=BF16):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def test_rows_of_2_to_the_28_tokens():
    """Dispatch and both sums over a token's rows, one row each: copies."""
    T, d = (1 << 28) + 70, 8
    case(f"permute, combine, permute backward T={T} d={d}")
    x, dest = _last_rows(T, d), torch.arange(T, dtype=torch.int32, device="cuda")
    out = _nan(T, d)
    laep.moe_permute(x, dest, 1, out=out)
    assert torch.equal(out, x)
    out.fill_(float("nan"))
    laep.moe_permute_bwd(x, dest, T, 1, out=out)
    assert torch.equal(out, x)
    out.fill_(float("nan"))
    laep.moe_combine(x, torch.ones((T, 1), device="cuda"), dest, out=out)
    assert torch.equal(out, x)
    del x, dest, out
    torch.cuda.empty_cache()


def test_combine_backward_of_2_to_the_24_tokens():
    T, d = (1 << 24) + 70, 8
    case(f"combine backward T={T} d={d}")
    x, dest = _last_rows(T, d), torch.arange(T, dtype=torch.int32, device="cuda")
    gate, dy, dgate = torch.full((T, 1), 2.0, device="cuda"), _nan(T, d), \
        _nan(T, 1, dtype=torch.float32)
    laep.moe_combine_bwd(x, x, gate, dest, dy_perm=dy, dgate=dgate)
    assert torch.equal(dy, 2 * x)
    assert dgate[-3:, 0].tolist() == [8.0, 32.0, 72.0] and not dgate[:-3].any()


@pytest.mark.parametrize("renorm", [True, False])
def test_router_backward_data_of_2_to_the_26_tokens(renorm):
    T, E, k, d = (1 << 26) + 70, 2, 1, 8
    case(f"router backward, data T={T} E={E} d={d} renorm={renorm}")
    idx = torch.zeros((T, k), dtype=torch.int32, device="cuda")
    gate, dg = torch.ones((T, k), device="cuda"), torch.zeros((T, k), device="cuda")
    gate[-3:], dg[-3:] = 0.5, 4.0
    x, wr = torch.zeros((T, d), dtype=BF16, device="cuda"), _nan(E, d)
    wr[0], wr[1] = 1.0, 3.0
    dx = _nan(T, d)
    logits = None if renorm else torch.zeros((T, E), device="cuda")
    off = torch.tensor([0, T, T], dtype=torch.int32, device="cuda")
    src = torch.arange(T, dtype=torch.int32, device="cuda")
    laep.moe_route_bwd(dg, idx, gate, x, wr, renorm=renorm, logits=logits, offsets=off, row_src=src,
                       dx=dx, weights=False)
    # s = g dg = 2; renorm: dl = g (dg - s) = 1 at expert 0; full: p (q - s) = 1 and -1
    assert (dx[-3:] == (1.0 if renorm else -2.0)).all() and not dx[:-3].any()


def test_routing_of_2_to_the_28_tokens():
    T, E, k, d = (1 << 28) + 70, 2, 1, 8
    case(f"routing and counts T={T} E={E} d={d}")
    x, wr = _last_rows(T, d), torch.zeros((E, d), dtype=BF16, device="cuda")
    wr[1] = 1.0
    idx = torch.full((T, k), -7, dtype=torch.int32, device="cuda")
    gate = _nan(T, k, dtype=torch.float32)
    src = torch.full((T,), -7, dtype=torch.int32, device="cuda")
    dest = torch.full((T,), -7, dtype=torch.int32, device="cuda")
    _, _, counts, offsets, _, _, _ = laep.moe_route_count(
        x, wr, k, want_row_src=True, topk_idx=idx, topk_gate=gate, dest_row=dest, row_src=src)
    assert idx[-3:, 0].tolist() == [1, 1, 1] and not idx[:-3].any() and (gate == 1.0).all()
    assert counts.tolist() == [T - 3, 3] and offsets.tolist() == [0, T - 3, T]
    rows = torch.arange(T, dtype=torch.int32, device="cuda")
    assert torch.equal(src, rows) and torch.equal(dest, rows)
    del x, idx, gate, src, dest, rows
    torch.cuda.empty_cache()


def test_ffn_of_2_to_the_24_tiles():
    """One row an expert, all 256 of one matrix of 2^22 hidden columns."""
    R, E, d, f = 256, 256, 64, 1 << 22
    case(f"ffn R={R} E={E} d={d} f={f}")
    assert laep.laep_ffn_fwd_row_tile(R, E, d, f) == 32
    assert (R // 32 + E) * (f // 64) > 1 << 24
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((R, d), generator=g, device="cuda").to(BF16)
    gu = torch.randn((1, 2 * f, d), generator=g, device="cuda", dtype=BF16) * 0.125
    dn = torch.zeros((1, d, f), device="cuda", dtype=BF16)
    dn[0, :, -64:] = torch.eye(64, device="cuda").to(BF16)      # y: the last columns of H
    off = torch.arange(E + 1, dtype=torch.int32, device="cuda")
    emap = torch.zeros(E, dtype=torch.int32, device="cuda")
    act = _nan(R, 2 * f)
    ws = torch.full((laep.workspace_bytes(laep.LAEP_CALL_FFN_FWD, R, 1, E, d, f),), 0xFF,
                    dtype=torch.uint8, device="cuda")
    y, _ = laep.moe_grouped_ffn_fwd(x, gu, dn, off, expert_map=emap, act_save=act, ws=ws)
    for rows in act.split(16):
        assert torch.isfinite(rows).all()
    xv, gv, uv = (v.double().cpu() for v in (x, gu[0, f - 64:f], gu[0, 2 * f - 64:]))
    a, u = xv @ gv.T, xv @ uv.T
    h = a * torch.sigmoid(a) * u
    # A rounded, then H and y: half a step each of values of their own size
    assert ((act[:, f - 64:f].double().cpu() - a).abs() <= 2.0 ** -8 * a.abs() + 1e-4).all()
    assert ((y.double().cpu() - h).abs() <= 3 * 2.0 ** -8 * h.abs() + 1e-4).all()
    del act, gu, dn, ws
    torch.cuda.empty_cache()
