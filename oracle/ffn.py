"""Plain CPU oracle of the expert feed-forward block and of 8-bit checkpoints,
in fp64.

TEST INFRASTRUCTURE ONLY, like the rest of this package.

* rows x sorted by expert between offsets: u = x Wu^T, g = x Wg^T, a = silu(g) u
  (without Wg: relu(u)), y = a Wd^T; rows of no expert give zeros;
* its gradients for dy, from u and g: da = dy Wd, s = sigmoid(g), du = da g s,
  dg = da u s (1 + g (1 - s)) (relu: du = da [u > 0]), dx = du Wu + dg Wg,
  dWu = du^T x, dWg = dg^T x, dWd = dy^T a;
* checkpoints: blocks of 32 values of a row in steps 2^(e - 6), 2^e <= max |v|
  < 2^(e + 1), e >= -127; scale byte e + 127, 255 for a block with NaN or
  infinity; codes are the nearest whole numbers (ties to even) in -127 .. 127.
"""
from __future__ import annotations

import numpy as np

BLOCK = 32


def groups(offsets, n):
    """(first, end) of each expert's rows, borders held to [0, n]."""
    o = np.clip(np.asarray(offsets, np.int64), 0, n)
    return [(int(a), max(int(a), int(b))) for a, b in zip(o, o[1:])]


def _sigmoid(g):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-g))


def pre(w, x, offsets):
    """Pre-activations [n, F] of the rows (zeros for rows of no expert)."""
    out = np.zeros((x.shape[0], w.shape[1]))
    for e, (a, b) in enumerate(groups(offsets, x.shape[0])):
        out[a:b] = x[a:b] @ w[e].T
    return out


def act(u, g):
    return np.maximum(u, 0.0) if g is None else _sigmoid(g) * g * u


def forward(wu, wg, wd, x, offsets):
    """(y, u, g)."""
    u = pre(wu, x, offsets)
    g = None if wg is None else pre(wg, x, offsets)
    return pre(wd, act(u, g), offsets), u, g


def dact(da, u, g):
    """(du, dg)."""
    if g is None:
        return np.where(u > 0, da, 0.0), None
    s = _sigmoid(g)
    return da * g * s, da * u * s * (1.0 + g * (1.0 - s))


def backward(wu, wg, wd, x, dy, u, g, offsets):
    """(dx, dwu, dwg, dwd)."""
    n = x.shape[0]
    dx = np.zeros_like(x)
    dw = [None if w is None else np.zeros_like(w) for w in (wu, wg, wd)]
    for e, (a, b) in enumerate(groups(offsets, n)):
        if a == b:
            continue
        ge = None if g is None else g[a:b]
        du, dg = dact(dy[a:b] @ wd[e], u[a:b], ge)
        dx[a:b] = du @ wu[e]
        dw[0][e] = du.T @ x[a:b]
        dw[2][e] = dy[a:b].T @ act(u[a:b], ge)
        if dg is not None:
            dx[a:b] += dg @ wg[e]
            dw[1][e] = dg.T @ x[a:b]
    return (dx, *dw)


def pack(x):
    """(codes int8 [n, c], scale uint8 [n, blocks])."""
    x = np.asarray(x, np.float64)
    n, c = x.shape
    v = np.zeros((n, -(-c // BLOCK) * BLOCK))
    v[:, :c] = x
    v = v.reshape(n, -1, BLOCK)
    top = np.abs(v).max(axis=2)
    bad = ~np.isfinite(top)
    e = np.frexp(np.where(bad, 1.0, top))[1] - 1
    e = np.where(top == 0, -127, np.maximum(e, -127))
    q = np.clip(np.rint(np.ldexp(np.where(bad[:, :, None], 0.0, v), (6 - e)[:, :, None])), -127, 127)
    scale = np.where(bad, 255, e + 127).astype(np.uint8)
    return q.reshape(n, -1)[:, :c].astype(np.int8), scale


def unpack(codes, scale):
    e = np.repeat(scale.astype(np.int64) - 133, BLOCK, axis=1)[:, :codes.shape[1]]
    return np.where(e == 122, np.nan, np.ldexp(codes.astype(np.float64), e))
