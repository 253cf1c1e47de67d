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
