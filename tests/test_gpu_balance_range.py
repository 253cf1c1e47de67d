"""Balance loss at the ends of the float32 range: rows masked with a finite value,
logits whose product with log2 e overflows, large logits with a common offset.

Tolerances as in test_gpu_block.py: the differences to a row's maximum are exact or
at most 20 here, or so large that the probability is 0 in 64 bits as well."""
import numpy as np
import pytest
import torch

import oracle.block as ob
import paper_2601_14327_amd as laep
from _gpu import case, dev
from test_gpu_block import F32, _check_balance, _check_balance_bwd

pytestmark = pytest.mark.gpu

LOW, TOP = np.finfo(np.float32).min, np.finfo(np.float32).max


def _extreme_rows(logits, rng):
    """Rewrites every other row to one of the kinds below; returns the masked rows."""
    T, E = logits.shape
    masked = []
    for i, t in enumerate(range(0, T, 2)):
        row, kind = logits[t], i % 12
        some = rng.random(E) < 0.5
        some[rng.integers(E)] = True
        if kind == 0:
            row[:] = LOW                       # a padded token
        elif kind == 1:
            row[:] = -1e30
        elif kind == 2:
            row[:] = -1e10
        elif kind == 3:
            row[:] = 1e10
        elif kind == 4:
            row[:] = TOP
        elif kind == 5:
            row[some] = LOW                    # some experts masked by a value
        elif kind == 6:
            row[rng.integers(E)] = 2.5e38      # one maximum whose log2 e fold overflows
        elif kind == 7:
            row[:] = -2.5e38
        elif kind == 8:
            row[:] = np.where(some, TOP, LOW)  # a difference that overflows
        elif kind == 9:
            row[:] = np.where(some, LOW, -np.inf)
        elif kind == 10:
            row[:] = np.float32(3e6) + np.rint(row)    # a common offset, exact differences
        else:
            row[:] = np.float32(-3e6) + np.rint(row)
        if kind in (0, 1, 2, 7):
            masked.append(t)
    return masked


@pytest.mark.parametrize("T,E,k,off,dead", [
    (1, 8, 2, None, 0), (24, 2, 1, None, 0), (48, 45, 4, [0, 10, 10, 48], 0),
    (130, 256, 8, None, 40), (64, 8, 2, [0, 1, 30, 64], 3), (3000, 64, 8, None, 0),
    (5001, 45, 4, [0, 7, 2500, 5001], 5), (2100, 13, 2, [0, 1000, 1000, 1001, 2100], 0),
    (4100, 256, 4, [0, 4100], 64), (700, 130, 2, [5, 300, 690], 0)])
def test_balance_at_the_ends_of_the_range(T, E, k, off, dead):
    case(f"balance loss, extreme logits T={T} E={E} k={k} off={off} dead={dead}")
    rng = np.random.default_rng(T + E)
    logits = rng.standard_normal((T, E)).astype(np.float32)
    masked = _extreme_rows(logits, rng)
    alive = None
    if dead:
        alive = np.ones(E, np.uint8)
        alive[rng.permutation(E)[:dead]] = 0
        masked_logits = np.where(alive, logits, -np.inf)
    else:
        masked_logits = logits
    idx = np.argsort(-masked_logits, axis=1, kind="stable")[:, :k].astype(np.int32)
    o = None if off is None else np.array(off, np.int32)
    kw = dict(alive=None if alive is None else dev(alive, torch.uint8),
              seq_offsets=None if o is None else dev(o, torch.int32))
    got = laep.moe_balance_loss(dev(logits, F32), dev(idx, torch.int32), coef=0.5, **kw)
    _check_balance(logits, idx, alive, o, 0.5, got)
    dl = laep.moe_balance_loss_bwd(dev(logits, F32), got[3], **kw)
    _check_balance_bwd(logits, alive, o, got[3], dl)
    # a uniform row of the alive experts, as its definition says
    p = ob.alive_probs(logits, alive)
    n = E - dead
    for t in masked:
        assert np.allclose(p[t][p[t] > 0], 1 / n) and (p[t] > 0).sum() == n


@pytest.mark.parametrize("T", [40, 4000])
def test_one_masked_token_leaves_the_others_alone(T):
    """A padded token's row, all finfo.min, is uniform: the loss stays finite and the
    other tokens' gradients keep their bits."""
    E, k = 64, 8
    case(f"balance loss, a padded token in T={T}")
    rng = np.random.default_rng(T)
    logits = rng.standard_normal((T, E)).astype(np.float32)
    logits[T // 2] = LOW
    idx = np.argsort(-logits, axis=1, kind="stable")[:, :k].astype(np.int32)
    got = laep.moe_balance_loss(dev(logits, F32), dev(idx, torch.int32))
    _check_balance(logits, idx, None, None, 1.0, got)
    dl = laep.moe_balance_loss_bwd(dev(logits, F32), got[3])
    _check_balance_bwd(logits, None, None, got[3], dl)
    other = logits.copy()
    other[T // 2] = 0.0
    want = laep.moe_balance_loss_bwd(dev(other, F32), got[3])
    assert torch.equal(dl, want)      # a row of equal logits, whatever their value
