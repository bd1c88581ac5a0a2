"""64-bit references of routing, layers and joining, with elementwise bounds of what fp32 and the roundings of the
types may be off by. Every function returns (value, bound) pairs, or what it says.

U = 2^-24 is fp32's rounding; a bf16 one is off by 2^-8 of the value at most. An exponential of an argument a has the
argument rounded: relative 2 |a| U, and a few U of its own."""
from __future__ import annotations

import math

import numpy as np
from scipy.special import erfc

from tests import rows_ref

U = 2.0 ** -24
TINY = 1e-37


def out(dtype):
    return 2.0 ** -8 if dtype == "bf16" else U


# ---------------------------------------------------------------- activations

def logistic(z):
    return np.where(z >= 0, 1 / (1 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))))


def cdf(z):
    return 0.5 * erfc(-z / math.sqrt(2))


def density(z):
    return np.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)


# What the normal distribution's tail P(-|z|) of bf16 results may be off by: it is 2^q, q a polynomial in |z|, whose
# relative error up to 8 is at most 2^-14.9 and which stays below 2^-50 past it (test_layers_ref.py evaluates it); fp32
# rounds q, below 53 up to there, in seven steps of at most 53 U each: times log 2, 260 U, 2^-15.9. gelu takes the tail
# times |z|, its slope once.
def tail(z, dtype):
    if dtype != "bf16":
        return 0.0
    return np.where(np.abs(z) > 8, 2.0 ** -49, (2.0 ** -14.9 + 260 * U) * cdf(-np.abs(z)))


def act(z, name, dtype="f32"):
    """(value, bound of evaluating it in fp32, largest slope)"""
    if name == "silu":
        v = z * logistic(z)
        return v, U * (2 * np.abs(z) + 10) * np.abs(v), 1.1
    if name == "gelu":
        v = z * cdf(z)
        return v, U * (2 * z * z + 16) * np.abs(v) + np.abs(z) * tail(z, dtype), 1.13
    if name == "relu":
        return np.maximum(z, 0), 0 * z, 1.0
    return z, 0 * z, 1.0


def slope(z, name, dtype="f32"):
    """(value, bound)"""
    if name == "silu":
        f = logistic(z)
        return f * (1 + z * (1 - f)), U * (4 * np.abs(z) + 24) * (f + np.abs(z) * f * (1 - f))
    if name == "gelu":
        return (cdf(z) + z * density(z),
                U * (2 * z * z + 24) * (cdf(z) + np.abs(z) * density(z)) + tail(z, dtype))
    if name == "relu":
        return (z > 0).astype(float), 0 * z
    return np.ones_like(z), 0 * z


# ---------------------------------------------------------------- layers

def layer(x, w, bias, residual, ids, name, per_row, dtype):
    """(y, z), each (value, bound)"""
    n, N = ids.size, w.shape[2]
    z, mag = np.zeros((n, N)), np.zeros((n, N))
    for g, rows in enumerate(rows_ref.members(ids, w.shape[0])):
        z[rows] = x[rows // per_row] @ w[g]
        mag[rows] = np.abs(x[rows // per_row]) @ np.abs(w[g])
        if bias is not None:
            z[rows] += bias[g]
            mag[rows] += np.abs(bias[g])
    zb = rows_ref.U_SUM * (x.shape[1] + 5) * mag
    y, yb, most = act(z, name, dtype)
    yb = yb + most * zb
    if residual is not None:
        y = y + residual
        yb = yb + U * np.abs(y)
    return (y, yb + out(dtype) * np.abs(y) + TINY), (z, zb + out(dtype) * np.abs(z) + TINY)


def layer_grad(x, w, z, dy, ids, name, per_row, dtype):
    """(dx, dw, dbias), each (value, bound)"""
    G, K, N = w.shape
    s, sb = slope(z, name, dtype)
    dz = dy * s
    dzb = np.abs(dy) * sb + U * np.abs(dz)
    if dtype == "bf16" and name != "none":
        dzb = dzb + out(dtype) * (np.abs(dz) + dzb)
    n = ids.size
    dx, dxb = np.zeros((n, K)), np.zeros((n, K))
    dw, dwb, db, dbb = np.zeros(w.shape), np.zeros(w.shape), np.zeros((G, N)), np.zeros((G, N))
    for g, rows in enumerate(rows_ref.members(ids, G)):
        d, b, xs = dz[rows], dzb[rows], x[rows // per_row]
        terms = rows_ref.U_SUM * (len(rows) + 4)
        dx[rows] = d @ w[g].T
        dxb[rows] = (b + rows_ref.U_SUM * (N + 4) * np.abs(d)) @ np.abs(w[g]).T
        dw[g] = xs.T @ d
        dwb[g] = np.abs(xs).T @ (b + terms * np.abs(d)) + out(dtype) * np.abs(dw[g])
        db[g] = d.sum(0)
        dbb[g] = (b + terms * np.abs(d)).sum(0) + out(dtype) * np.abs(db[g])
    of = lambda a: a.reshape(n // per_row, per_row, K).sum(1)
    v = of(dx)
    bound = of(dxb + rows_ref.U_SUM * per_row * np.abs(dx)) + out(dtype) * np.abs(v)
    return (v, bound + TINY), (dw, dwb + TINY), (db, dbb + TINY)


# ---------------------------------------------------------------- joining

def mix(y, weights, residual, k, dtype):
    n, N = y.shape[0] // k, y.shape[1]
    t = y.reshape(n, k, N) * (1.0 if weights is None else weights[:, :, None])
    v, mag = t.sum(1), np.abs(t).sum(1)
    if residual is not None:
        v, mag = v + residual, mag + np.abs(residual)
    return v, rows_ref.U_SUM * (k + 2) * mag + out(dtype) * np.abs(v) + TINY


def mix_grad(dout, weights, y, k, dtype):
    n, N = dout.shape
    w = np.ones((n, k)) if weights is None else weights
    dy = (w[:, :, None] * dout[:, None, :]).reshape(n * k, N)
    t = y.reshape(n, k, N) * dout[:, None, :]
    return ((dy, (U + out(dtype)) * np.abs(dy) + TINY),
            (t.sum(2), rows_ref.U_SUM * (N + 2) * np.abs(t).sum(2) + TINY))


# ---------------------------------------------------------------- routing

def scores(logits, score):
    gone = ~(logits > -np.inf)
    if score == "softmax":
        with np.errstate(invalid="ignore"):
            top = np.where(gone, -np.inf, logits).max(1, keepdims=True)
            e = np.where(gone, 0.0, np.exp(np.where(gone, 0.0, logits) - np.where(np.isfinite(top), top, 0.0)))
        total = e.sum(1, keepdims=True)
        return e / np.where(total > 0, total, 1.0)
    return np.where(gone, 0.0, logistic(np.where(gone, 0.0, logits)))


def route(logits, k, bias, score, blocks, keep, renorm, scale):
    """(ids, (weights, bound))"""
    n, E = logits.shape
    s = scores(logits, score)
    plain = bias is None and (blocks == 1 or keep == blocks)
    key = logits.copy() if plain else s + (0.0 if bias is None else bias)
    key[~(logits > -np.inf)] = -np.inf
    if keep < blocks:
        for i in range(n):
            rows = np.sort(key[i].reshape(blocks, -1), 1)[:, ::-1]
            total = rows[:, 0] + (np.where(np.isinf(rows[:, 1]), 0.0, rows[:, 1]) if rows.shape[1] > 1 else 0.0)
            best = np.argsort(-total, kind="stable")[:keep]
            for b in set(range(blocks)) - set(best.tolist()):
                key[i].reshape(blocks, -1)[b] = -np.inf
    ids = np.argsort(-key, axis=1, kind="stable")[:, :k].astype(np.int32)
    there = np.take_along_axis(key, ids, 1) > -np.inf
    w = np.where(there, np.take_along_axis(s, ids, 1), 0.0)
    if renorm:
        total = w.sum(1, keepdims=True)
        w = w / np.where(total > 0, total, 1.0)
    w = w * scale
    finite = np.where(np.isfinite(logits), logits, 0.0)
    span = finite.max(1, keepdims=True) - finite.min(1, keepdims=True) + np.abs(finite).max(1, keepdims=True)
    return np.where(there, ids, -1), (w, U * (6 * span + E + 24) * np.abs(w) + TINY)


def route_grad(logits, ids, u, score, renorm, scale, dtype):
    """(value, bound)"""
    n, E = logits.shape
    s = scores(logits, score)
    there = (ids >= 0) & (ids < E)
    at = np.where(there, ids, 0)
    there &= np.take_along_axis(logits, at, 1) > -np.inf
    p = np.where(there, np.take_along_axis(s, at, 1), 0.0)
    u = np.where(there, u, 0.0)
    total = p.sum(1, keepdims=True) if renorm else np.ones((n, 1))
    p = p / np.where(total > 0, total, 1.0)
    mean = (u * p).sum(1, keepdims=True) if renorm or score == "softmax" else np.zeros((n, 1))
    mag = (np.abs(u) * p).sum(1, keepdims=True) if renorm or score == "softmax" else np.zeros((n, 1))
    g = p * (u - (mean if renorm else 0.0))
    gm = p * (np.abs(u) + (mag if renorm else 0.0))
    if score == "sigmoid":
        rest = 1 - np.take_along_axis(s, at, 1)
        g, gm = g * rest, gm * rest
    value, most = np.zeros((n, E)), np.zeros((n, E))
    rows = np.arange(n)[:, None]
    np.add.at(value, (rows, at), np.where(there, g, 0.0))
    np.add.at(most, (rows, at), np.where(there, gm, 0.0))
    if score == "softmax" and not renorm:
        value, most = value - s * mean, most + s * mag
    finite = np.where(np.isfinite(logits), logits, 0.0)
    span = finite.max(1, keepdims=True) - finite.min(1, keepdims=True) + np.abs(finite).max(1, keepdims=True)
    value, most = scale * value, abs(scale) * most
    return value, U * (16 * span + 2 * E + 64) * most + out(dtype) * np.abs(value) + TINY
