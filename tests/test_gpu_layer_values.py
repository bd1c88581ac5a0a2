"""Relative precision of single values: activations far from zero, the weights of far logits."""
from __future__ import annotations

import numpy as np
import pytest

from tests import layers_ref as ref
from tests.test_gpu_rows import cg, dev, host, rounded  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N", [1, 64])
def test_silu_of_far_values_in_fp32(cg, N):
    """z is x itself (its parts times 1 are exact). The exponential is off by 2 U, its correction, the product with it and the
    sum by U each, the reciprocal by 2 U, the product by U: 8 U of the value, however small it is."""
    import torch

    x = rounded(np.concatenate([np.linspace(-80, 80, 20001), np.linspace(-1, 1, 1001)])[:, None], "f32")
    o = cg.group_rows(torch.zeros(len(x), dtype=torch.int32, device="cuda"), 1)
    y, z = cg.grouped_layer(dev(x), torch.ones(1, 1, N, device="cuda"), *o, activation="silu", z=None)
    assert np.array_equal(host(z), np.broadcast_to(x, z.shape))
    want = x * ref.logistic(x)
    assert np.all(np.abs(host(y) - want) <= 8 * ref.U * np.abs(want) + ref.TINY)


def test_slope_of_silu_below_zero_in_fp32(cg):
    """The slope f (1 + z (1 - f)), f off by 7 U, 1 - f by 5 U and each of four operations by U, of terms of these magnitudes."""
    import torch

    z = rounded(np.linspace(-80, 0, 20001)[:, None], "f32")
    o = cg.group_rows(torch.zeros(len(z), dtype=torch.int32, device="cuda"), 1)
    one = torch.ones(1, 1, 1, device="cuda")
    dx, _, _ = cg.grouped_layer_grad(dev(z), one, torch.ones(len(z), 1, device="cuda"), *o, z=dev(z), activation="silu")
    f = ref.logistic(z)
    assert np.all(np.abs(host(dx) - f * (1 + z * (1 - f))) <= 16 * ref.U * (f + np.abs(z) * f * (1 - f)) + ref.TINY)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("E,k", [(8, 8), (48, 24), (130, 40)])
def test_routing_weights_of_far_logits(cg, dtype, score, renorm, E, k):
    """Logits that are multiples of 1/4 up to 60, whose differences fp32 holds. A share is an exponential, 4 U, over one plus
    another, 3 U, a quotient's U: 8 U. Their sum, of k or E, has the same and U of each addition; quotient and scale U each."""
    rng = np.random.default_rng(E)
    logits = rng.integers(-120, 121, (700, E)) * 0.25
    scale = 3.0 if score == "softmax" else 2.0
    ids, w = cg.route_rows(dev(logits, dtype), k, score=score, renormalize=renorm, scale=scale)
    want, (value, _) = ref.route(logits, k, None, score, 1, 1, renorm, scale)
    assert np.array_equal(ids.cpu().numpy(), want)
    assert np.all(np.abs(host(w) - value) <= (20 + E) * ref.U * np.abs(value) + ref.TINY)
