"""Buffers given to the calls around the experts: the binding refuses what the kernels
could not use (host tensors, strided views, other types and shapes) before the C call."""
import pytest
import torch

import paper_2601_14327_amd as laep
from paper_2601_14327_amd import api

BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def z(*s, dt=F32):
    return torch.zeros(s, dtype=dt, device="cuda")


def test_a_host_workspace_is_refused():
    with pytest.raises(ValueError, match="ws must be a device tensor"):
        api._given_ws(torch.zeros(1 << 20, dtype=U8), torch.device("cpu"),
                      laep.LAEP_CALL_BALANCE, 4, 1, 8)


def _calls_with_workspace(ws):
    """Each call that takes a workspace, at a size that needs at most 1 MB."""
    x, g = z(4, 64, dt=BF16), z(64)
    idx, gate = z(4, 2, dt=I32), z(4, 2)
    wr, lg = z(8, 64, dt=BF16), z(4, 8)
    yield lambda: laep.moe_layer_norm_bwd(x, x.clone(), g, z(4), z(4), ws=ws)
    yield lambda: laep.moe_balance_loss(lg, idx, ws=ws)
    yield lambda: laep.moe_route_bwd_balance(z(4, 2), idx, gate, lg, x, wr, z(1, 8), ws=ws)
    xt, off = z(4, 64, dt=BF16), torch.tensor([0, 4], dtype=I32, device="cuda")
    src = torch.arange(4, dtype=I32, device="cuda")
    yield lambda: laep.moe_grouped_ffn_bwd_gather_act8(
        z(4, 64, dt=BF16), xt, src, 1, z(4, 128, dt=torch.int8), z(4, 4, dt=U8),
        z(1, 128, 64, dt=BF16), z(1, 64, 64, dt=BF16), off, ws=ws)


@pytest.mark.gpu
def test_host_and_strided_workspaces_are_refused():
    for call in _calls_with_workspace(torch.zeros(1 << 22, dtype=U8)):
        with pytest.raises(ValueError, match="ws must be a device tensor"):
            call()
    for call in _calls_with_workspace(z(1 << 20, 4, dt=U8)[:, 0]):
        with pytest.raises(ValueError, match="ws must be contiguous"):
            call()
    for call in _calls_with_workspace(z(16, dt=U8)):      # too small: the C call's
        with pytest.raises(laep.LaepError, match="workspace"):
            call()
    for call in _calls_with_workspace(z(1 << 20)):        # of any type
        call()
    torch.cuda.synchronize()


def _route_bwd_args(T=4, d=64, E=8, k=2):
    return dict(dgate=z(T, k), topk_idx=z(T, k, dt=I32), topk_gate=z(T, k), logits=z(T, E),
                x=z(T, d, dt=BF16), w_router=z(E, d, dt=BF16), grad_coef=z(1, E))


@pytest.mark.gpu
@pytest.mark.parametrize("name,bad", [
    ("dgate", lambda: z(4, 3)), ("dgate", lambda: z(4, 2, dt=BF16)),
    ("topk_gate", lambda: z(3, 2)), ("topk_idx", lambda: z(4, 2, dt=torch.int64)),
    ("x", lambda: z(3, 64, dt=BF16)), ("x", lambda: z(4, 32, dt=BF16)),
    ("w_router", lambda: z(8, 64)),
    ("dx", lambda: z(4, 64)), ("dx", lambda: z(3, 64, dt=BF16)),
    ("dx", lambda: z(4, 128, dt=BF16)[:, :64]),
    ("dx", lambda: torch.zeros((4, 64), dtype=BF16)),
    ("dbias", lambda: z(7)), ("dbias", lambda: z(8, dt=BF16)),
    ("dbias", lambda: torch.zeros(8))])
def test_router_backward_with_balance_refuses_other_buffers(name, bad):
    args = _route_bwd_args()
    args[name] = bad()
    with pytest.raises(ValueError, match=f"^{name} must"):
        laep.moe_route_bwd_balance(**args)


@pytest.mark.gpu
def test_router_backward_with_balance_takes_its_own_buffers():
    args = _route_bwd_args()
    dx, db = z(4, 64, dt=BF16) + 1, z(8) + 1
    got = laep.moe_route_bwd_balance(**args, dx=dx, dbias=db)   # a given dbias is computed
    assert got[0] is dx and got[2] is db and not dx.any() and not db.any()
