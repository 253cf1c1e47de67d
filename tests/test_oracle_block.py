"""Pins of oracle.block: torch autograd through independent float64 forwards,
central differences, closed forms and hand-worked checkpoints."""
import numpy as np
import pytest
import torch

import oracle.block as ob


def _differences(fn, x, step=1e-5):
    """Central differences of a scalar function at every element of x."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        v = x[i]
        x[i] = v + step
        hi = fn()
        x[i] = v - step
        lo = fn()
        x[i] = v
        g[i] = (hi - lo) / (2 * step)
    return g


@pytest.mark.parametrize("with_dres", [False, True])
def test_layer_norm_gradients(with_dres):
    rng = np.random.default_rng(1)
    T, d = 5, 16
    x, dy = rng.standard_normal((T, d)) * 2 + 1, rng.standard_normal((T, d))
    gamma, beta = 1 + 0.3 * rng.standard_normal(d), rng.standard_normal(d)
    w = rng.standard_normal((T, d)) if with_dres else np.zeros((T, d))
    y, s, mean, rstd = ob.layer_norm(x, gamma, beta)
    xt = torch.tensor(x, requires_grad=True)
    gt, bt = torch.tensor(gamma, requires_grad=True), torch.tensor(beta, requires_grad=True)
    yt = torch.nn.functional.layer_norm(xt, (d,), gt, bt, 1e-5)
    np.testing.assert_allclose(y, yt.detach().numpy(), rtol=0, atol=1e-12)
    ((yt * torch.tensor(dy)).sum() + (xt * torch.tensor(w)).sum()).backward()
    dx, dgamma, dbeta = ob.layer_norm_bwd(dy, s, gamma, mean, rstd, w if with_dres else None)
    for a, b in ((dx, xt), (dgamma, gt), (dbeta, bt)):
        np.testing.assert_allclose(a, b.grad.numpy(), rtol=0, atol=1e-11)
    # truncation of the differences: step^2 times a third derivative, and 1e-16 / step
    num = _differences(lambda: float((ob.layer_norm(x, gamma, beta)[0] * dy).sum()
                                     + (x * w).sum()), x)
    np.testing.assert_allclose(dx, num, rtol=0, atol=1e-7)


def test_layer_norm_residual_and_constant_rows():
    x = np.full((2, 8), 3.0)
    y, s, mean, rstd = ob.layer_norm(x, np.ones(8), np.arange(8.0), residual=x, eps=1e-2)
    np.testing.assert_array_equal(s, 6.0)
    np.testing.assert_array_equal(y, np.tile(np.arange(8.0), (2, 1)))
    np.testing.assert_allclose(rstd, 10.0)


@pytest.mark.parametrize("seqs", [None, [0, 0, 7, 7, 12, 12]])
@pytest.mark.parametrize("dead", [0, 3])
def test_balance_loss_gradients(seqs, dead):
    rng = np.random.default_rng(3 + dead)
    T, E, k, coef = 12, 7, 2, 0.3
    logits = rng.standard_normal((T, E))
    alive = np.ones(E, np.uint8)
    alive[:dead] = 0
    idx = np.argsort(-np.where(alive, logits, -np.inf), axis=1)[:, :k].astype(np.int32)
    loss, counts, prob, grad = ob.balance_loss(logits, idx, coef, alive, seqs)
    off = [0, T] if seqs is None else seqs
    lt = torch.tensor(logits, requires_grad=True)
    p = torch.softmax(lt.masked_fill(torch.tensor(alive) == 0, float("-inf")), 1)
    want, full = 0.0, [(a, b) for a, b in zip(off, off[1:]) if b > a]
    for a, b in full:
        n = np.bincount(idx[a:b].ravel(), minlength=E)
        frac = torch.tensor((E - dead) * n / (k * (b - a)))
        want = want + coef * (frac * p[a:b].mean(0)).sum() / len(full)
    assert abs(float(want.detach()) - loss) < 1e-13
    assert counts.sum() == T * k
    want.backward()
    dl = ob.balance_loss_bwd(logits, grad, 1.0, alive, seqs)
    np.testing.assert_allclose(dl, lt.grad.numpy(), rtol=0, atol=1e-14)
    num = _differences(lambda: ob.balance_loss(logits, idx, coef, alive, seqs)[0], logits)
    np.testing.assert_allclose(dl, num, rtol=0, atol=1e-9)
    np.testing.assert_allclose(dl.sum(1), 0, atol=1e-15)   # a softmax's Jacobian
    np.testing.assert_allclose(2.5 * dl, ob.balance_loss_bwd(logits, grad, 2.5, alive, seqs))


def test_even_loads_give_the_coefficient():
    E, k = 8, 2
    idx = np.array([[(t * k + j) % E for j in range(k)] for t in range(16)], np.int32)
    rng = np.random.default_rng(0)
    loss, counts, _, _ = ob.balance_loss(rng.standard_normal((16, E)), idx, 0.01)
    assert abs(loss - 0.01) < 1e-15 and (counts == 4).all()
    # all load and all probability on one expert: E times that
    logits = np.full((4, E), -np.inf)
    logits[:, 5] = 0.0
    loss, _, prob, _ = ob.balance_loss(logits, np.full((4, 1), 5, np.int32), 0.01)
    assert abs(loss - 0.08) < 1e-15 and prob[0, 5] == 1.0


def test_rows_without_an_alive_logit_and_unrouted_slots():
    logits = np.array([[-np.inf, -np.inf], [0.0, 0.0]])
    loss, counts, prob, grad = ob.balance_loss(logits, np.array([[-1], [1]], np.int32), 1.0)
    np.testing.assert_array_equal(prob, [[0.25, 0.25]])
    np.testing.assert_array_equal(counts, [[0, 1]])
    assert not ob.balance_loss_bwd(logits, grad)[0].any()


def test_act8_by_hand():
    v = np.zeros((1, 96))
    v[0, 0], v[0, 1], v[0, 2], v[0, 3] = 1.0, -0.5, 1 / 128, 3 / 128   # steps of 1/64
    v[0, 32], v[0, 33] = 255 / 128, -127 / 64                          # 127.5 steps: the last one
    v[0, 64] = np.inf
    q, b = ob.act8_save(v)
    np.testing.assert_array_equal(b, [[121, 121, 255]])
    assert q[0, :4].tolist() == [64, -32, 0, 2]     # ties to even
    assert q[0, 32:34].tolist() == [127, -127] and not q[0, 64:].any()
    out = ob.act8_load(q, b)
    assert out[0, 0] == 1.0 and out[0, 1] == -0.5 and np.isnan(out[0, 64:]).all()


def test_act8_error_bound_and_tiny_values():
    rng = np.random.default_rng(5)
    v = rng.standard_normal((64, 256)) * np.exp(rng.uniform(-60, 60, (64, 256 // 32))).repeat(32, 1)
    v = v.astype(np.float32).astype(np.float64)
    q, b = ob.act8_save(v)
    err = np.abs(ob.act8_load(q, b) - v).reshape(64, -1, 32)
    step = np.ldexp(1.0, b.astype(int) - 127)
    top = np.abs(v).reshape(64, -1, 32).max(2)
    assert (top / step >= 64).all() and (top / step < 128).all()
    assert (err.max(2) <= np.where(top / step > 127.5, 1.0, 0.5) * step).all()
    q, b = ob.act8_save(np.full((1, 32), 2.0 ** -140))     # below the smallest scale
    assert b[0, 0] == 1 and not q.any()


def test_swiglu_backward_at_a_checkpoint():
    rng = np.random.default_rng(7)
    q, b = ob.act8_save(rng.standard_normal((6, 128)))
    dh = rng.standard_normal((6, 64))
    at = torch.tensor(ob.act8_load(q, b), requires_grad=True)
    h = torch.nn.functional.silu(at[:, :64]) * at[:, 64:]
    (h * torch.tensor(dh)).sum().backward()
    da, hh = ob.swiglu_bwd_act8(q, b, dh)
    np.testing.assert_allclose(hh, h.detach().numpy(), rtol=0, atol=1e-14)
    np.testing.assert_allclose(da, at.grad.numpy(), rtol=0, atol=1e-14)
