"""Oracle of what a pre-norm MoE block computes around the layer (float64
NumPy): layer norm, the router's balance loss, 8-bit activation checkpoints.

Test infrastructure only; see the package docstring.

Only the paper's comparison systems train with a balance loss, and its block's
norm is not spelled out; the readings used here:

* layer norm over the columns of s = round(x + residual), the variance the mean
  of the centred squares, statistics unrounded;
* balance loss per sequence s of n_s tokens: coef * sum_e f[s, e] P[s, e] with
  f[s, e] = N_alive counts[s, e] / (k n_s) and P the mean probability (softmax
  over the alive experts), averaged over the non-empty sequences; evenly loaded
  experts give coef.  The counts carry no gradient;
* 8-bit checkpoints: 32 columns share a power-of-two scale by the exponent of
  their largest magnitude, values round to the nearest of 127 steps.
"""
from __future__ import annotations

import numpy as np

from .numerics import rounder, sigmoid

F64 = np.float64
ACT8_BLOCK = 32


# --------------------------------------------------------------------------
# Layer norm
# --------------------------------------------------------------------------
def layer_norm(x, gamma, beta=None, residual=None, eps=1e-5, dtype="f64"):
    """Returns (y, s, mean, rstd); y is unrounded, s as stored in dtype."""
    s = np.asarray(x, F64)
    if residual is not None:
        s = rounder(dtype)(s + np.asarray(residual, F64))
    mean = s.mean(axis=1)
    cen = s - mean[:, None]
    rstd = 1.0 / np.sqrt((cen ** 2).mean(axis=1) + eps)
    y = cen * rstd[:, None] * np.asarray(gamma, F64)
    if beta is not None:
        y = y + np.asarray(beta, F64)
    return y, s, mean, rstd


def layer_norm_bwd(dy, s, gamma, mean, rstd, dres=None):
    """Returns (dx, dgamma, dbeta), unrounded."""
    dy, s = np.asarray(dy, F64), np.asarray(s, F64)
    rs = np.asarray(rstd, F64)[:, None]
    xh = (s - np.asarray(mean, F64)[:, None]) * rs
    g = dy * np.asarray(gamma, F64)
    dx = rs * (g - g.mean(axis=1, keepdims=True) - xh * (g * xh).mean(axis=1, keepdims=True))
    if dres is not None:
        dx = dx + np.asarray(dres, F64)
    return dx, (dy * xh).sum(axis=0), dy.sum(axis=0)


# --------------------------------------------------------------------------
# Balance loss
# --------------------------------------------------------------------------
def alive_probs(logits, alive=None):
    """Softmax over the alive experts; dead ones, and tokens whose alive logits
    are all -inf, get 0."""
    l = np.asarray(logits, F64)
    a = np.ones(l.shape[1], bool) if alive is None else np.asarray(alive).astype(bool)
    p = np.zeros_like(l)
    sub = l[:, a]
    if sub.size:
        m = sub.max(axis=1, keepdims=True)
        ex = np.exp(sub - np.where(np.isneginf(m), 0.0, m))
        z = ex.sum(axis=1, keepdims=True)
        p[:, a] = ex / np.where(z == 0.0, 1.0, z)
    return p


def balance_loss(logits, topk_idx, coef, alive=None, seq_offsets=None):
    """Returns (loss, counts [S, E], prob_mean [S, E], grad_coef [S, E])."""
    T, E = logits.shape
    k = topk_idx.shape[1]
    off = [0, T] if seq_offsets is None else [int(o) for o in seq_offsets]
    S = len(off) - 1
    n_alive = E if alive is None else int(np.asarray(alive).astype(bool).sum())
    p = alive_probs(logits, alive)
    counts = np.zeros((S, E), np.int64)
    prob = np.zeros((S, E))
    frac = np.zeros((S, E))
    grad = np.zeros((S, E))
    live = sum(off[s + 1] > off[s] for s in range(S))
    loss = 0.0
    for s in range(S):
        a, b = off[s], off[s + 1]
        if a == b:
            continue
        for e in np.asarray(topk_idx)[a:b].ravel():
            if 0 <= e < E:
                counts[s, e] += 1
        prob[s] = p[a:b].sum(axis=0) / (b - a)
        frac[s] = n_alive * counts[s] / (k * (b - a))
        loss += coef * float((frac[s] * prob[s]).sum()) / live
        grad[s] = coef * frac[s] / ((b - a) * live)
    return loss, counts, prob, grad


def balance_loss_bwd(logits, grad_coef, dloss=1.0, alive=None, seq_offsets=None):
    """dlogits [T, E], unrounded."""
    T, E = logits.shape
    off = [0, T] if seq_offsets is None else [int(o) for o in seq_offsets]
    p = alive_probs(logits, alive)
    dl = np.zeros((T, E))
    for s in range(len(off) - 1):
        a, b = off[s], off[s + 1]
        c = np.asarray(grad_coef, F64)[s]
        dl[a:b] = dloss * p[a:b] * (c - (p[a:b] * c).sum(axis=1, keepdims=True))
    return dl


# --------------------------------------------------------------------------
# 8-bit activation checkpoints
# --------------------------------------------------------------------------
def act8_save(act):
    """act [R, C] (values of the storage type).  Returns (q [R, C] int8,
    scale [R, C / 32] uint8)."""
    a = np.asarray(act, F64)
    R, C = a.shape
    v = a.reshape(R, C // ACT8_BLOCK, ACT8_BLOCK)
    bad = ~np.isfinite(v).all(axis=2)
    v = np.where(bad[..., None], 0.0, v)
    amax = np.abs(v).max(axis=2)
    _, e = np.frexp(amax)                  # amax = m 2^e, 1/2 <= m < 1
    biased = np.where(amax == 0.0, 0, np.maximum(e - 1 + 127, 0))
    b = np.maximum(biased - 6, 1)
    q = np.rint(np.ldexp(v, (127 - b)[..., None]))
    q = np.clip(q, -127, 127)
    b = np.where(bad, 255, b)
    return q.reshape(R, C).astype(np.int8), b.astype(np.uint8)


def act8_load(q, scale):
    R, C = q.shape
    v = np.asarray(q, F64).reshape(R, C // ACT8_BLOCK, ACT8_BLOCK)
    b = np.asarray(scale).astype(np.int64)[..., None]
    out = np.where(b == 255, np.nan, np.ldexp(v, b - 127))
    return out.reshape(R, C)


def swiglu_bwd_act8(q, scale, dh):
    """Returns (dA [R, 2f], H [R, f]), unrounded, at the decoded pre-activations."""
    dh = np.asarray(dh, F64)
    f = dh.shape[1]
    a = act8_load(q, scale)
    ag, au = a[:, :f], a[:, f:]
    s = sigmoid(ag)
    return (np.concatenate([dh * au * s * (1.0 + ag * (1.0 - s)), dh * ag * s], axis=1),
            ag * s * au)
