"""Layers and their gradients in the largest tiles of the general product, and joins past the caches, at the remainders
where they can go wrong."""
from __future__ import annotations

import math

import numpy as np
import pytest

from tests import layers_ref as ref
from tests.test_gpu_layer_grads import NAMES, draw_grad, grad_of_parts
from tests.test_gpu_layers import draw_layer, named
from tests.test_gpu_rows import cg, check, dev, host, rounded, strided  # noqa: F401

pytestmark = pytest.mark.gpu


def tiles(n, G, width, rows):
    """Tiles of `rows` by `rows` that a product of n rows has."""
    return (n // rows + G) * -(-width // rows)


def in_large_tiles(n, G, width, dtype, small_first):
    """Whether a product of long inputs takes tiles of 128 by 128: compute units have one each, and those of 64 by 64 would
    not end before."""
    if n < 40 * G or width <= 64 or tiles(n, G, width, 32) <= 1024:
        return False
    big = tiles(n, G, width, 128)
    return tiles(n, G, width, 64) > 1024 * -(-big // 512) if small_first or dtype == "f32" else big >= 256


# rows of x, rows that share one, groups, widths: remainders of rows, of a step's k and of columns, and none
LARGE = [(40000, 1, 3, 333, 203), (13400, 3, 3, 333, 200), (45000, 1, 7, 130, 257), (33000, 1, 2, 320, 256), (9100, 4, 5, 450, 450)]


@pytest.mark.parametrize("t,per,G,K,N", LARGE)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act,bias,residual,keep,pad,kind", [
    ("gelu", True, True, True, 3, "holes"), ("silu", True, False, True, 0, "even"), ("relu", False, True, False, 8, "holes"),
    ("none", False, False, False, 0, "one")])
def test_layers(cg, t, per, G, K, N, dtype, act, bias, residual, keep, pad, kind):
    import torch

    assert in_large_tiles(t * per, G, N, dtype, False)
    rng = np.random.default_rng(t + N)
    x, w, b, ids = draw_layer(rng, t, per, G, K, N, kind, dtype)
    r = rounded(rng.standard_normal((t * per, N)), dtype) if residual else None
    o = cg.group_rows(dev(ids), G)
    xd = dev(x, dtype)
    y = strided(torch.zeros(t * per, N, dtype=xd.dtype, device="cuda"), pad) if pad else None
    got = cg.grouped_layer(strided(xd, pad), dev(w, dtype), *o, bias=dev(b, dtype) if bias else None, activation=named(act),
                           residual=None if r is None else strided(dev(r, dtype), pad), per_row=per, y=y, z=None if keep else False)
    want = ref.layer(x, w, b if bias else None, r, ids, act, per, dtype)
    check(got[0] if keep else got, want[0], "y")
    if keep:
        check(got[1], want[1], "z")
    if pad:
        assert torch.isnan(y._base[:, N:]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t,per,G,K,N", LARGE + [(66000, 1, 4, 128, 448), (16700, 4, 33, 128, 168)])
@pytest.mark.parametrize("act,pad,kind", [("silu", 3, "holes"), ("gelu", 0, "even"), ("none", 1, "holes")])
def test_gradients(cg, t, per, G, K, N, dtype, act, pad, kind):
    import torch

    assert in_large_tiles(t * per, G, K, dtype, True)
    rng = np.random.default_rng(t + K)
    x, w, ids, z, dy = draw_grad(rng, t, per, G, K, N, kind, dtype)
    o = cg.group_rows(dev(ids), G)
    xd = dev(x, dtype)
    dx = strided(torch.zeros(t, K, dtype=xd.dtype, device="cuda"), pad) if pad else None
    a = (strided(xd, pad), dev(w, dtype), strided(dev(dy, dtype), pad), *o)
    kw = dict(z=None if act == "none" else strided(dev(z, dtype), pad), activation=named(act), per_row=per)
    got = cg.grouped_layer_grad(*a, dx=dx, **kw)
    want = grad_of_parts(x, w, z, dy, ids, act, per) if dtype == "bf16" else ref.layer_grad(x, w, z, dy, ids, act, per, dtype)
    for g, v, name in zip(got, want, NAMES):
        check(g, v, name)
    if pad:
        assert torch.isnan(dx._base[:, K:]).all()
    again = cg.grouped_layer_grad(*a, **kw)
    assert all(torch.equal(g, h) for g, h in zip(got, again))


@pytest.mark.parametrize("act", ["silu", "relu", "none"])
def test_values_that_are_not_finite(cg, act):
    """fp32: results that are not finite, and no others, are formed again in the first, middle and last tiles."""
    import torch

    t, per, G, K, N = 13400, 3, 3, 333, 203
    rng = np.random.default_rng(2)
    x, w, b, ids = draw_layer(rng, t, per, G, K, N, "even", "f32")
    o = cg.group_rows(dev(ids), G)
    run = lambda x: cg.grouped_layer(dev(x), dev(w), *o, bias=dev(b), activation=named(act), per_row=per, z=None)
    y0, z0 = run(x)
    x1 = x.copy()
    x1[0, 3], x1[t // 2, 332], x1[t - 1, 0] = math.inf, -math.inf, math.nan
    y, z = run(x1)
    hit = np.zeros(t, bool)
    hit[[0, t // 2, t - 1]] = True
    same = torch.from_numpy(np.repeat(~hit, per)).cuda()
    assert torch.equal(y[same], y0[same]) and torch.equal(z[same], z0[same])
    with np.errstate(invalid="ignore", over="ignore"):
        (_, _), (zr, _) = ref.layer(x1, w, b, None, ids, act, per, "f32")
    zr, h = zr[np.repeat(hit, per)], host(z[~same])
    assert np.array_equal(np.isnan(h), np.isnan(zr)) and np.array_equal(h[np.isinf(zr)], zr[np.isinf(zr)])
    dy, zz = (rounded(rng.standard_normal((t * per, N)), "f32") for _ in range(2))
    grad = lambda dy: cg.grouped_layer_grad(dev(x), dev(w), dev(dy), *o, z=dev(zz), activation=named(act), per_row=per)
    base = grad(dy)
    d1, zz[5, 7] = dy.copy(), 1.0
    base, d1[5, 7] = grad(dy), math.inf
    got = grad(d1)
    rows = torch.arange(t, device="cuda") != 5 // per
    assert torch.equal(got[0][rows], base[0][rows]) and not torch.isfinite(got[0][5 // per]).any()
    g, cols = ids[5], torch.arange(N, device="cuda") != 7
    assert torch.equal(got[1][g][:, cols], base[1][g][:, cols]) and not torch.isfinite(got[1][g][:, 7]).any()
    assert torch.equal(got[2][g][cols], base[2][g][cols]) and got[2][g][7].item() == math.inf


# ---------------------------------------------------------------- joins of more than the memory-side cache holds

# rows, rows of each, width, padding: rows on half lines or not, up to 64, 128 and 256 vectors, and more
JOINS = [(45000, 8, 449, 0), (70000, 16, 130, 0), (80000, 4, 896, 0), (80000, 4, 880, 16), (20000, 8, 1344, 0),
         (27000, 3, 2113, 3), (9000, 8, 4160, 0), (300000, 8, 64, 0), (300000, 9, 61, 2)]


def sample(n):
    return [0, 1, n // 3, n // 2, n - 2, n - 1]


def _strided_rand(gen, n, N, pad, t):
    import torch

    buf = torch.full((n, N + pad), float("nan"), dtype=t, device="cuda")
    buf[:, :N] = torch.randn(n, N, device="cuda", generator=gen, dtype=torch.float32).to(t)
    return buf[:, :N]


@pytest.mark.parametrize("n,k,N,pad", JOINS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("weights,residual", [(True, True), (False, False)])
def test_joins(cg, n, k, N, pad, dtype, weights, residual):
    import torch

    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    assert n * N * (k + 1) * t.itemsize > 2 ** 28
    gen = torch.Generator("cuda").manual_seed(n)
    y = _strided_rand(gen, n * k, N, pad, t)
    w = torch.rand(n, k, device="cuda", generator=gen) if weights else None
    r = _strided_rand(gen, n, N, pad, t) if residual else None
    base = torch.full((n, N + pad), float("nan"), dtype=t, device="cuda")
    out = cg.mix_rows(y, k, weights=w, residual=r, out=base[:, :N])
    assert torch.isnan(base[:, N:]).all() and torch.isfinite(out).all()
    for i in sample(n):
        want = ref.mix(host(y[i * k:i * k + k]), host(w[i:i + 1]) if weights else None, host(r[i:i + 1]) if residual else None, k, dtype)
        check(out[i:i + 1], want, i)
    # all rows: what the sums of a row are in 64 bits, each value off by its own bound at most
    rows = slice(0, n, max(1, n // 500))
    yk = y.reshape(n, k, N)[rows].double()
    v = (yk * (w[rows].double()[:, :, None] if weights else 1.0)).sum(1) + (r[rows].double() if residual else 0.0)
    most = (yk.abs() * (w[rows].double()[:, :, None] if weights else 1.0)).sum(1) + (r[rows].double().abs() if residual else 0.0)
    assert ((out[rows].double() - v).abs() <= 2.0 ** -23 * (k + 2) * most + ref.out(dtype) * v.abs() + ref.TINY).all()


@pytest.mark.parametrize("n,k,N,pad", JOINS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_join_gradients(cg, n, k, N, pad, dtype):
    import torch

    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    assert n * N * k * t.itemsize * 2 > 2 ** 28
    gen = torch.Generator("cuda").manual_seed(n + 1)
    d, y = _strided_rand(gen, n, N, pad, t), _strided_rand(gen, n * k, N, pad, t)
    w = torch.rand(n, k, device="cuda", generator=gen)
    base = torch.full((n * k, N + pad), float("nan"), dtype=t, device="cuda")
    dy, dw = cg.mix_rows_grad(d, k, weights=w, y=y, dy=base[:, :N])
    assert torch.isnan(base[:, N:]).all()
    for i in sample(n):
        want = ref.mix_grad(host(d[i:i + 1]), host(w[i:i + 1]), host(y[i * k:i * k + k]), k, dtype)
        check(dy[i * k:i * k + k], want[0], i)
        check(dw[i:i + 1], want[1], i)
    want = (w[:, :, None] * d.float()[:, None, :]).to(t).reshape(n * k, N)      # one product, rounded to fp32 and to the type
    assert torch.equal(dy, want)
    alone = cg.mix_rows_grad(d, k, weights=w, dweights=False, dy=torch.empty_like(want))
    assert alone[1] is None and torch.equal(alone[0], want)
    del want
    alone = cg.mix_rows_grad(d, k, weights=w, y=y, dy=False)
    assert alone[0] is None and torch.equal(alone[1], dw)
    rows = slice(0, n, max(1, n // 500))
    terms = y.reshape(n, k, N)[rows].double() * d[rows].double()[:, None, :]
    assert ((dw[rows].double() - terms.sum(2)).abs() <= 2.0 ** -23 * (N + 2) * terms.abs().sum(2) + ref.TINY).all()


@pytest.mark.parametrize("t,per,G,K,N", [(20000, 1, 3, 200, 24), (9000, 3, 2, 150, 32), (30000, 1, 3, 300, 8), (20000, 1, 2, 400, 5),
                                         (40000, 1, 4, 72, 30), (30000, 1, 3, 200, 60)])
@pytest.mark.parametrize("act,pad,kind", [("silu", 0, "even"), ("gelu", 3, "holes")])
def test_bf16_gradients_of_narrow_outputs(cg, t, per, G, K, N, act, pad, kind):
    """Column tiles of 32 and 64 of the weights' gradients, from dz that is held in parts and that is formed."""
    import torch

    rng = np.random.default_rng(t + K)
    x, w, ids, z, dy = draw_grad(rng, t, per, G, K, N, kind, "bf16")
    o = cg.group_rows(dev(ids), G)
    a = (strided(dev(x, "bf16"), pad), dev(w, "bf16"), strided(dev(dy, "bf16"), pad), *o)
    got = cg.grouped_layer_grad(*a, z=strided(dev(z, "bf16"), pad), activation=act, per_row=per)
    for g, v, name in zip(got, grad_of_parts(x, w, z, dy, ids, act, per), NAMES):
        check(g, v, name)
