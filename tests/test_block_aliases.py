"""Buffers that the calls around the experts may not share (laep_block.h) are refused
on the host, before any HIP call."""
import pytest

from test_abi import L, _err, _fake  # noqa: F401  (L: the library fixture)

T, E = 16, 8
ROWS = T * E * 4      # bytes of the logits


def _balance_bwd(L, logits, out, accumulate):
    keep, p = _fake()
    return L.moe_balance_loss_bwd(p + logits, p, None, None, None, T, E, 1, p + out, accumulate,
                                  None)


@pytest.mark.parametrize("at", [0, 16, ROWS - 16, -16, 16 - ROWS])
def test_balance_gradient_is_not_added_over_the_logits(L, at):
    assert _balance_bwd(L, 1024, 1024 + at, 1) == 1 and "dlogits" in _err(L)


@pytest.mark.parametrize("at", [16, ROWS - 16, -16, 16 - ROWS])
def test_balance_gradient_may_not_overlap_a_part_of_the_logits(L, at):
    assert _balance_bwd(L, 1024, 1024 + at, 0) == 1 and "dlogits" in _err(L)


@pytest.mark.parametrize("renorm", [0, 1])
@pytest.mark.parametrize("at", [0, 16, ROWS - 16, -16, 16 - ROWS])
def test_router_backward_does_not_write_dlogits_over_the_logits(L, at, renorm):
    keep, p = _fake()
    need = L.moe_workspace_bytes(4, T, 2, E, 64, 0)
    assert L.moe_route_bwd_balance(p, p, p, p + 1024, None, p, p, p, None, 1, None, 1, T, 64, E, 2,
                                   renorm, p + 1024 + at, p, None, p, 0, p, need, None) == 1
    assert "dlogits" in _err(L)
