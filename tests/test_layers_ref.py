"""The reference of layers, joining and routing against differences of its own forward forms, on the CPU."""
from __future__ import annotations

import os
import re

import numpy as np
import pytest
from scipy.special import erfcx, log_ndtr

from tests import layers_ref as ref

H = 1e-6


def differences(f, a):
    g = np.zeros_like(a)
    for i in np.ndindex(*a.shape):
        keep = a[i]
        a[i] = keep + H
        up = f()
        a[i] = keep - H
        g[i] = (up - f()) / (2 * H)
        a[i] = keep
    return g


@pytest.mark.parametrize("name", ["silu", "gelu", "relu", "none"])
@pytest.mark.parametrize("per", [1, 3])
def test_layer(name, per):
    rng = np.random.default_rng(0)
    ids = np.array([0, 2, -1, 1, 0, 2, 5, 0, 1], np.int32)
    x, w, b = rng.standard_normal((9 // per, 4)), rng.standard_normal((3, 4, 5)), rng.standard_normal((3, 5))
    dy = rng.standard_normal((9, 5))
    (_, _), (z, _) = ref.layer(x, w, b, None, ids, name, per, "f32")
    loss = lambda: (ref.layer(x, w, b, None, ids, name, per, "f32")[0][0] * dy).sum()
    for got, a in zip(ref.layer_grad(x, w, z, dy, ids, name, per, "f32"), (x, w, b)):
        assert np.abs(got[0] - differences(loss, a)).max() < 1e-7


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_route(score, renorm):
    rng = np.random.default_rng(1)
    logits, u = rng.standard_normal((5, 7)), rng.standard_normal((5, 3))
    logits[1, 2:] = logits[4] = -np.inf
    ids, _ = ref.route(logits, 3, None, score, 1, 1, renorm, 1.5)
    assert (ids[1] == -1).sum() == 1 and (ids[4] == -1).all()
    a = np.where(np.isinf(logits), 0.0, logits)
    gone = np.isinf(logits)
    loss = lambda: (ref.route(np.where(gone, -np.inf, a), 3, None, score, 1, 1, renorm, 1.5)[1][0] * u).sum()
    got = ref.route_grad(logits, ids, u, score, renorm, 1.5, "f32")[0]
    assert np.abs(got - differences(loss, a)).max() < 1e-7


def test_mix():
    rng = np.random.default_rng(2)
    y, w, d = rng.standard_normal((12, 5)), rng.standard_normal((4, 3)), rng.standard_normal((4, 5))
    loss = lambda: (ref.mix(y, w, None, 3, "f32")[0] * d).sum()
    for got, a in zip(ref.mix_grad(d, w, y, 3, "f32"), (y, w)):
        assert np.abs(got[0] - differences(loss, a)).max() < 1e-7


def _coefficients(part, first):
    number = r"(-?[\d.]+(?:e-?\d+)?)f"
    c = [float(v) for v in re.search(rf"q = fmaf\({number}, {first}, {number}\)", part).groups()]
    return c + [float(v) for v in re.findall(rf"q = fmaf\(q, {first}, {number}\)", part)]


def test_tail_of_gelu():
    """The polynomials of the sources: bf16's up to 8, and that it falls past it; fp32's for all z, and as fp32 evaluates
    it, where the reference allows 16 U for it, the exponential's 2 U, the reciprocal's and three products."""
    path = os.path.join(os.path.dirname(os.path.dirname(__file__)), "paper_2605_15073_amd", "csrc", "rows_layer.h")
    low, high = re.search(r"float normal_cdf\(.*?\n}", open(path).read(), re.S).group().split("} else {")
    c = _coefficients(low, "a")
    assert len(c) == 8
    z = np.linspace(0, 8, 400001)
    assert np.abs(np.exp2(np.polyval(c, z) - log_ndtr(-z) / np.log(2)) - 1).max() < 2.0 ** -14.9
    far = np.polyval(c, np.concatenate([np.linspace(8, 100, 100001), np.geomspace(101, 1e30, 1001)]))
    assert far[0] < -50 and (np.diff(far) < 0).all()
    c = _coefficients(high, "t")
    assert len(c) == 10 and "fmaf(0.25f, a, 1.f)" in high
    z = np.concatenate([np.linspace(0, 20, 400001), np.geomspace(20, 1e8, 2001)])
    t = 1 / (1 + 0.25 * z)
    assert np.abs(t * np.polyval(c, t) / (0.5 * erfcx(z / np.sqrt(2))) - 1).max() < 2.0 ** -24
    f = np.float32
    z = z.astype(f)
    t = f(1) / (f(1) + f(0.25) * z)
    q = np.full_like(z, f(c[0]))
    for k in c[1:]:
        q = q * t + f(k)
    assert np.abs((q * t).astype(float) / (0.5 * erfcx(z.astype(float) / np.sqrt(2))) - 1).max() < 8 * ref.U
