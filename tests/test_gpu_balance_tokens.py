"""Balance loss of as many tokens as an int32 counts."""
import pytest
import torch

import paper_2601_14327_amd as laep
from _gpu import case

pytestmark = pytest.mark.gpu

T = (1 << 31) - 1


def test_gradient_of_tokens_of_no_sequence():
    """Tokens outside every sequence get zeros up to the last one, and nothing else is
    written."""
    E, pad = 2, 512
    case(f"balance gradient T={T} E={E}, nearly all tokens of no sequence")
    logits = torch.zeros((T, E), device="cuda")
    grad = torch.tensor([[1.0, 0.0]], device="cuda")
    off = torch.tensor([5, 9], dtype=torch.int32, device="cuda")
    whole = torch.full(((T + 2 * pad) * E,), 7.0, device="cuda")
    out = whole[pad * E:(pad + T) * E].view(T, E)
    laep.moe_balance_loss_bwd(logits, grad, seq_offsets=off, dlogits=out)
    torch.cuda.synchronize()
    assert (whole[:pad * E] == 7.0).all() and (whole[(pad + T) * E:] == 7.0).all()
    assert out[5:9].tolist() == [[0.25, -0.25]] * 4       # p (c - sum p c), p = 1/2
    out[5:9] = 0.0
    step = 1 << 28
    assert not any(bool(out[i:i + step].any()) for i in range(0, T, step))
    del logits, whole, out
    torch.cuda.empty_cache()


def test_loss_of_one_sequence():
    E, k = 2, 1
    case(f"balance loss T={T} E={E}")
    logits = torch.zeros((T, E), device="cuda")
    idx = torch.zeros((T, k), dtype=torch.int32, device="cuda")
    loss, counts, prob, grad = laep.moe_balance_loss(logits, idx, coef=0.5)
    assert counts.tolist() == [[T, 0]]
    # sums of halves: exact up to 2^24 of them, then at most 1024 + 4 roundings
    assert (prob - 0.5).abs().max() <= 1100 * 2.0 ** -24
    assert abs(float(loss) - 0.5) <= 0.5 * 1200 * 2.0 ** -24
    assert abs(float(grad[0, 0]) * T - 1.0) <= 1e-6 and not grad[0, 1].any()
    del logits, idx
    torch.cuda.empty_cache()
