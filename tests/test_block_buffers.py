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


def _expert_bwd_args(T=4, d=64, E=2, k=1, f=64):
    R = T * k
    return dict(dy_perm=z(R, d, dt=BF16), x=z(T, d, dt=BF16),
                row_src=torch.arange(R, dtype=I32, device="cuda"), k=k,
                act_q=z(R, 2 * f, dt=torch.int8), act_scale=z(R, 2 * f // 32, dt=U8) + 120,
                w_gate_up=z(E, 2 * f, d, dt=BF16), w_down=z(E, d, f, dt=BF16),
                offsets=torch.tensor([0, 1, R], dtype=I32, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("name,bad", [
    ("dy_perm", lambda: z(4, 64)), ("dy_perm", lambda: z(3, 64, dt=BF16)),
    ("row_src", lambda: z(4, dt=torch.int64)), ("offsets", lambda: z(3, dt=torch.int64)),
    ("w_gate_up", lambda: z(2, 128, 64)), ("w_gate_up", lambda: z(2, 64, 64, dt=BF16)),
    ("w_gate_up", lambda: z(1, 128, 64, dt=BF16)), ("w_down", lambda: z(2, 64, 64)),
    ("w_down", lambda: z(2, 128, 64, dt=BF16)),
    ("expert_map", lambda: z(3, dt=I32)), ("expert_map", lambda: z(2, dt=torch.int64)),
    ("dx_perm", lambda: z(4, 64)), ("dx_perm", lambda: z(4, 128, dt=BF16)[:, :64]),
    ("dx_perm", lambda: torch.zeros((4, 64), dtype=BF16)),
    ("dw_gate_up", lambda: z(2, 128, 64, dt=BF16)), ("dw_gate_up", lambda: z(2, 64, 64)),
    ("dw_down", lambda: z(1, 64, 64)), ("dw_down", lambda: torch.zeros((2, 64, 64)))])
def test_expert_backward_at_a_checkpoint_refuses_other_buffers(name, bad):
    args = _expert_bwd_args()
    args[name] = bad()
    with pytest.raises(ValueError, match=f"^{name} must"):
        laep.moe_grouped_ffn_bwd_gather_act8(**args)


@pytest.mark.gpu
@pytest.mark.parametrize("name,bad", [
    ("dout", lambda: z(4, 64)), ("dout", lambda: z(3, 64, dt=BF16)),
    ("topk_gate", lambda: z(4, 1, dt=BF16)), ("topk_gate", lambda: z(4, 2))])
def test_expert_backward_at_a_checkpoint_refuses_other_gradients(name, bad):
    args = _expert_bwd_args()
    args.update(dy_perm=None, dout=z(4, 64, dt=BF16), topk_gate=z(4, 1))
    args[name] = bad()
    with pytest.raises(ValueError, match=f"^{name} must"):
        laep.moe_grouped_ffn_bwd_gather_act8(**args)


@pytest.mark.gpu
def test_expert_backward_at_a_checkpoint_takes_its_own_buffers():
    args = _expert_bwd_args()
    own = dict(dx_perm=z(4, 64, dt=BF16) + 1, dw_gate_up=z(2, 128, 64) + 1,
               dw_down=z(2, 64, 64) + 1)
    got = laep.moe_grouped_ffn_bwd_gather_act8(**args, **own)
    assert all(a is b and not a.any() for a, b in zip(got, own.values()))


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [lambda: z(3, 8), lambda: z(4, 8, dt=BF16), lambda: z(8, 4).t(),
                                 lambda: z(4, 7), lambda: torch.zeros((4, 8))])
def test_routing_refuses_other_logits(bad):
    x, wr = z(4, 64, dt=BF16), z(8, 64, dt=BF16)
    with pytest.raises(ValueError, match="^logits must"):
        laep.moe_route_count(x, wr, 2, logits=bad())
    with pytest.raises(ValueError, match="^logits must"):
        laep.moe_route_count(x, wr, 2, want_logits=True, logits=bad())


@pytest.mark.gpu
def test_routing_writes_given_logits():
    x, wr = z(4, 64, dt=BF16), z(8, 64, dt=BF16)
    logits = z(4, 8) + 1
    assert laep.moe_route_count(x, wr, 2, logits=logits)[6] is logits and not logits.any()


def _block():
    T, d, E, k, f = 8, 64, 4, 2, 64
    plan = laep.MoEBlockPlan(T, d, E, k, f)
    w = dict(gamma=z(d) + 1, beta=None, w_router=z(E, d, dt=BF16),
             w_gate_up=z(E, 2 * f, d, dt=BF16), w_down=z(E, d, f, dt=BF16))
    return plan, w, z(T, d, dt=BF16)


@pytest.mark.gpu
@pytest.mark.parametrize("name,bad", [
    ("w_router", lambda: z(4, 32, dt=BF16)), ("w_router", lambda: z(3, 64, dt=BF16)),
    ("w_router", lambda: z(4, 64)), ("w_gate_up", lambda: z(4, 64, 64, dt=BF16)),
    ("w_gate_up", lambda: z(3, 128, 64, dt=BF16)), ("w_gate_up", lambda: z(4, 128, 64)),
    ("w_down", lambda: z(4, 64, 32, dt=BF16)), ("w_down", lambda: z(4, 64, 64))])
def test_block_refuses_weights_of_other_sizes(name, bad):
    plan, w, x = _block()
    plan.forward(x, laep.BlockWeights(**w))
    wrong = laep.BlockWeights(**dict(w, **{name: bad()}))
    for call in (lambda: plan.forward(x, wrong), lambda: plan.backward(x, wrong)):
        with pytest.raises(ValueError, match=f"^{name} must"):
            call()


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [lambda: z(7, 64, dt=BF16), lambda: z(8, 64),
                                 lambda: z(8, 128, dt=BF16)[:, ::2],
                                 lambda: torch.zeros((8, 64), dtype=BF16)])
def test_block_refuses_other_gradients(bad):
    plan, w, x = _block()
    plan.forward(x, laep.BlockWeights(**w))
    with pytest.raises(ValueError, match="^dout must"):
        plan.backward(bad(), laep.BlockWeights(**w))
