"""What the gradients of layers owe beside their values: that an output does not depend on the others that are asked for,
and how many bits they hold between the two factors of dz and its products."""
from __future__ import annotations

import itertools

import numpy as np
import pytest

from tests import layers_ref as ref
from tests.test_gpu_layers import draw_layer, named
from tests.test_gpu_rows import cg, check, dev, host, rounded, strided  # noqa: F401

pytestmark = pytest.mark.gpu
NAMES = ("dx", "dw", "dbias")


def draw_grad(rng, t, per, G, K, N, kind, dtype):
    x, w, _, ids = draw_layer(rng, t, per, G, K, N, kind, dtype)
    z, dy = (rounded(rng.standard_normal((t * per, N)), dtype) for _ in range(2))
    return x, w, ids, z, dy


@pytest.mark.parametrize("t,per,G,K,N,pad,kind", [
    (3000, 1, 2, 64, 64, 0, "even"), (700, 2, 3, 64, 64, 3, "holes"), (2500, 2, 6, 40, 56, 0, "holes"), (64, 1, 1, 4, 4, 1, "one"),
    (50000, 1, 1, 64, 64, 0, "even"), (20000, 1, 3, 33, 17, 1, "holes"), (9000, 4, 3, 33, 64, 8, "even"), (400, 1, 2, 8, 60, 0, "none")])
@pytest.mark.parametrize("act", ["silu", "gelu", "none"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_narrow_outputs_do_not_depend_on_each_other(cg, t, per, G, K, N, pad, kind, act, dtype):
    """Each of the three, and each two, have the bits that they have together. An x that dx does not need may be anything."""
    import torch

    rng = np.random.default_rng(t + K)
    x, w, ids, z, dy = draw_grad(rng, t, per, G, K, N, kind, dtype)
    o = cg.group_rows(dev(ids), G)
    xd, rest = strided(dev(x, dtype), pad), (dev(w, dtype), strided(dev(dy, dtype), pad), *o)
    kw = dict(z=None if act == "none" else strided(dev(z, dtype), pad), activation=named(act), per_row=per)
    whole = cg.grouped_layer_grad(xd, *rest, **kw)
    for asked in itertools.product((True, False), repeat=3):
        if not any(asked):
            continue
        got = cg.grouped_layer_grad(xd if asked[1] else torch.full_like(xd, float("nan")), *rest,
                                    **{n: None if a else False for n, a in zip(NAMES, asked)}, **kw)
        for g, h, a, name in zip(got, whole, asked, NAMES):
            assert torch.equal(g, h) if a else g is None, (name, asked)
