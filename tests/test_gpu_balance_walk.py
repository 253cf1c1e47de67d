"""Balance loss: empty sequences are skipped together, wherever they lie."""
import numpy as np
import pytest
import torch

import paper_2601_14327_amd as laep
from _gpu import case, dev
from test_gpu_block import F32, _balance_inputs, _check_balance, _check_balance_bwd

pytestmark = pytest.mark.gpu


def _many_empty(T, first, n_seq, where):
    """Offsets of n_seq sequences, nearly all empty at one place; tokens before
    `first` belong to none."""
    off = np.full(n_seq + 1, first, np.int32)
    if where == "first":
        off[-1] = T
    elif where == "middle":
        off[n_seq // 2:] = (first + T) // 2
        off[-1] = T
    else:
        off[1:] = T
    return off


@pytest.mark.parametrize("where", ["first", "middle", "last"])
def test_empty_sequences_after_tokens_of_none(where):
    T, E, k, n_seq = 300, 8, 2, 3000
    case(f"balance loss, tokens of no sequence before {n_seq} empty ones, {where}")
    logits, idx, _, _ = _balance_inputs(T, E, k, 1, 0, 3)
    off = _many_empty(T, 101, n_seq, where)
    lt, it, ot = dev(logits, F32), dev(idx, torch.int32), dev(off, torch.int32)
    got = laep.moe_balance_loss(lt, it, seq_offsets=ot)
    _check_balance(logits, idx, None, off, 1.0, got)
    dl = laep.moe_balance_loss_bwd(lt, got[3], seq_offsets=ot)
    _check_balance_bwd(logits, None, off, got[3], dl)
    assert not dl[:101].any()


@pytest.mark.parametrize("first", [0, 100, 101])
@pytest.mark.parametrize("where", ["first", "middle", "last"])
def test_empty_sequences_are_skipped_together(where, first):
    """The gradient of 300 tokens beside 200000 empty sequences: a search each would
    take more than 0.1 us each, 20 ms; together they take a few searches (10 us)."""
    T, E, n_seq = 300, 8, 200000
    case(f"balance gradient, {n_seq} empty sequences, {where}, first token {first}")
    logits = torch.randn((T, E), device="cuda")
    grad = torch.zeros((n_seq, E), device="cuda")
    ot = dev(_many_empty(T, first, n_seq, where), torch.int32)
    out = torch.empty_like(logits)
    took = []
    for _ in range(4):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        laep.moe_balance_loss_bwd(logits, grad, seq_offsets=ot, dlogits=out)
        b.record()
        torch.cuda.synchronize()
        took.append(a.elapsed_time(b))
    assert min(took) < 5.0, f"{min(took)} ms"
