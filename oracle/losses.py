"""Plain CPU oracle of the training losses, in fp64.

TEST INFRASTRUCTURE ONLY, like the rest of this package.

* cross entropy of a vocabulary head: z = H W^T + b, lse = log sum exp z,
  loss = lse - z[target]; rows whose target lies outside [0, V), and rows
  without a logit above -inf, take no part;
* its gradients for row weights g: D = g (softmax(z) - onehot(target)),
  dH = D W, dW = D^T H, db = sum D;
* balance loss of a router: p = softmax(H W^T + b), counts c of the routed
  slots (S in n rows), L = E / (S n) sum_e c_e sum_t p_te, and its gradients
  with the counts held constant.
"""
from __future__ import annotations

import numpy as np


def _softmax(z):
    m = z.max(axis=1, keepdims=True)
    e = np.exp(z - np.where(np.isneginf(m), 0.0, m))
    s = e.sum(axis=1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        lse = np.where(np.isneginf(m), 0.0, m) + np.log(s)
        return e / np.where(s == 0.0, 1.0, s), lse[:, 0]


def logits(W, H, b=None):
    z = np.asarray(H, np.float64) @ np.asarray(W, np.float64).T
    return z if b is None else z + np.asarray(b, np.float64)


def head_loss(W, H, target, b=None):
    """(loss [Q], lse [Q])."""
    z = logits(W, H, b)
    _, lse = _softmax(z)
    y = np.asarray(target, np.int64)
    live = (y >= 0) & (y < z.shape[1]) & ~np.isneginf(lse)
    zy = z[np.arange(len(y)), np.where((y >= 0) & (y < z.shape[1]), y, 0)]
    with np.errstate(invalid="ignore"):
        return np.where(live, lse - zy, 0.0), lse


def head_loss_d(W, H, target, g, b=None):
    """(D [Q, V], softmax [Q, V], rows that take part [Q])."""
    z = logits(W, H, b)
    p, lse = _softmax(z)
    y = np.asarray(target, np.int64)
    live = (y >= 0) & (y < z.shape[1]) & ~np.isneginf(lse)
    D = p.copy()
    D[np.nonzero(live)[0], y[live]] -= 1.0
    return np.where(live[:, None], D * np.asarray(g, np.float64)[:, None], 0.0), p, live


def head_loss_grad(W, H, target, g, b=None):
    """(dH, dW, db)."""
    D, _, live = head_loss_d(W, H, target, g, b)
    H = np.where(live[:, None], np.asarray(H, np.float64), 0.0)
    return D @ np.asarray(W, np.float64), D.T @ H, D.sum(axis=0)


def balance_loss(W, H, target, b=None):
    """(loss, counts [E + 1], prob_sum [E], prob [Q, E])."""
    E = np.asarray(W).shape[0]
    p, _ = _softmax(logits(W, H, b))
    t = np.asarray(target, np.int64)
    ok = (t >= 0) & (t < E)
    live = ok.any(axis=1)
    c = np.bincount(t[ok], minlength=E)[:E]
    n, S = int(live.sum()), int(c.sum())
    ps = p[live].sum(axis=0) if n else np.zeros(E)
    loss = E * float(c @ ps) / (float(S) * n) if n else 0.0
    return loss, np.append(c, n).astype(np.int64), ps, p


def balance_grad(W, H, target, dloss, b=None, counts=None):
    """(dH, dW, db, dz); `counts` [E + 1]: in place of this batch's own."""
    E = np.asarray(W).shape[0]
    _, own, _, p = balance_loss(W, H, target, b)
    cn = own if counts is None else np.asarray(counts, np.int64)
    c, n = cn[:E].astype(np.float64), int(cn[E])
    t = np.asarray(target, np.int64)
    live = ((t >= 0) & (t < E)).any(axis=1)
    k = dloss * E / (c.sum() * n) if n else 0.0
    dz = k * p * (c[None, :] - (p @ c)[:, None])
    dz = np.where(live[:, None], dz, 0.0)
    Hl = np.where(live[:, None], np.asarray(H, np.float64), 0.0)
    return dz @ np.asarray(W, np.float64), dz.T @ Hl, dz.sum(axis=0), dz
