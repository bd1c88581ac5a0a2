"""64-bit reference of the row operators, with the elementwise bounds that fp32 sums must meet.

Every function returns (value, bound): the value from the definition, row by row and group by group
in numpy float64, and what a sum of the same products in fp32, of whatever order, may be off by.
A sum of K products rounds each product and each addition once, 2^-24 of a partial sum each; the
bound takes 2^-23 (K + 4) of the sum of magnitudes, which also covers an instruction that
truncates. A bf16 output adds 2^-8 of the value (half a unit in the last place is 2^-9)."""
from __future__ import annotations

import numpy as np

U_SUM = 2.0 ** -23


def members(ids, G):
    """Rows of each group, ascending."""
    return [np.flatnonzero(ids == g) for g in range(G)]


def order(ids, G):
    key = np.where((ids < 0) | (ids >= G), G, ids)
    return np.concatenate([[0], np.cumsum(np.bincount(key, minlength=G + 1)[:G])]), np.argsort(
        key, kind="stable")


def _out(dtype):
    return 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23


def _bound(terms, magnitude, value, dtype):
    return U_SUM * (terms + 4) * magnitude + _out(dtype) * np.abs(value) + 1e-37


def grouped(x, w, ids, dtype):
    y, mag = np.zeros((x.shape[0], w.shape[2])), np.zeros((x.shape[0], w.shape[2]))
    for g, rows in enumerate(members(ids, w.shape[0])):
        y[rows] = x[rows] @ w[g]
        mag[rows] = np.abs(x[rows]) @ np.abs(w[g])
    return y, _bound(x.shape[1], mag, y, dtype)


def grouped_grad(x, w, dy, ids, dtype):
    dx, dxm = np.zeros_like(x), np.zeros_like(x)
    dw, dwb = np.zeros_like(w), np.zeros_like(w)
    for g, rows in enumerate(members(ids, w.shape[0])):
        dx[rows] = dy[rows] @ w[g].T
        dxm[rows] = np.abs(dy[rows]) @ np.abs(w[g]).T
        dw[g] = x[rows].T @ dy[rows]
        dwb[g] = _bound(len(rows), np.abs(x[rows]).T @ np.abs(dy[rows]), dw[g], dtype)
    return (dx, _bound(w.shape[2], dxm, dx, dtype)), (dw, dwb)


def adapter(x, w, a, b, scale, ids, dtype):
    """The product between, a^T x, is rounded once more: 2^-23, or 2^-16 for its two bf16 parts."""
    n_in, r = a.shape[1:]
    y, mag = x @ w, np.abs(x) @ np.abs(w)
    mid = 2.0 ** -16 if dtype == "bf16" else 0.0
    low = np.zeros_like(y)
    for g, rows in enumerate(members(ids, a.shape[0])):
        y[rows] += scale[g] * ((x[rows] @ a[g]) @ b[g])
        low[rows] = abs(scale[g]) * ((np.abs(x[rows]) @ np.abs(a[g])) @ np.abs(b[g]))
    return y, _bound(2 * n_in + 2 * r, mag + low, y, dtype) + mid * low


def adapter_grad(x, w, a, b, dy, scale, ids, dtype):
    n_in, r = a.shape[1:]
    n_out = w.shape[1]
    mid = 2.0 ** -16 if dtype == "bf16" else 0.0
    dx, dxm = dy @ w.T, np.abs(dy) @ np.abs(w).T
    low = np.zeros_like(dx)
    da, dab, db, dbb = (np.zeros_like(t) for t in (a, a, b, b))
    for g, rows in enumerate(members(ids, a.shape[0])):
        s, xg, dg = scale[g], x[rows], dy[rows]
        u, um = s * (dg @ b[g].T), abs(s) * (np.abs(dg) @ np.abs(b[g]).T)
        h, hm = s * (xg @ a[g]), abs(s) * (np.abs(xg) @ np.abs(a[g]))
        dx[rows] += u @ a[g].T
        low[rows] = um @ np.abs(a[g]).T
        da[g], m = xg.T @ u, np.abs(xg).T @ um
        dab[g] = _bound(len(rows) + n_out, m, da[g], dtype) + mid * m
        db[g], m = h.T @ dg, hm.T @ np.abs(dg)
        dbb[g] = _bound(len(rows) + n_in, m, db[g], dtype) + mid * m
    return ((dx, _bound(2 * n_out + 2 * r, dxm + low, dx, dtype) + mid * low), (da, dab), (db, dbb))


# ---------------------------------------------------------------- AdamW, in single fp32 operations

F = np.float32
BLOCK = 256


def decode(codes, scales, signed):
    s = np.repeat(scales, BLOCK)[:codes.size].astype(F)
    if signed:
        t = codes.astype(F) * F(1 / 127)
        return t * np.abs(t) * s
    t = codes.astype(F) * F(1 / 255)
    t = t * t
    return t * t * s


def _blocks(x):
    return np.concatenate([x, np.zeros(-x.size % BLOCK, F)]).reshape(-1, BLOCK)


def encode(m, v):
    """(m codes, v codes, m scales, v scales)"""
    ms, vs = np.abs(_blocks(m)).max(1), _blocks(v).max(1)
    with np.errstate(all="ignore"):
        rep = lambda s: np.repeat(s, BLOCK)[:m.size]
        rm = np.where(rep(ms) > 0, np.abs(m) / rep(ms), F(0))
        rv = np.where(rep(vs) > 0, v / rep(vs), F(0))
    qm = np.rint(np.sqrt(rm) * F(127))
    qv = np.rint(np.sqrt(np.sqrt(rv)) * F(255))
    qv = np.where(v > 0, np.maximum(qv, 1), qv)
    return np.where(m < 0, -qm, qm).astype(np.int8), qv.astype(np.uint8), ms, vs


def adamw(p, g, m, v, step, lr, beta1, beta2, eps, weight_decay, grad_scale=1.0):
    """One step on fp32 moments: (p, m, v), every operation rounded to fp32."""
    c1, c2 = 1 - beta1 ** step, 1 - beta2 ** step
    g = g.astype(F) * F(grad_scale)
    m = m * F(beta1) + g * F(1 - beta1)
    v = v * F(beta2) + g * g * F(1 - beta2)
    den = np.sqrt(v * F(1 / c2)) + F(eps)
    return p * F(1 - lr * weight_decay) - m * F(lr / c1) / den, m, v
