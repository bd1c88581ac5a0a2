"""Row operators at the ends of their ranges: widths, values, sizes, masks, streams."""
from __future__ import annotations

import numpy as np
import pytest

from tests import rows_ref as ref
from tests.test_gpu_rows import _adapters, _linear, cg, check, dev, draw_ids, host, rounded, strided  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,G,n_in,n_out", [(400, 2, 65, 8), (400, 2, 130, 9), (300, 3, 896, 12), (400, 2, 127, 16),
                                            (400, 2, 72, 7), (400, 2, 200, 24)])
def test_row_gradient_of_few_columns(cg, dtype, n, G, n_in, n_out):
    """dx of a narrow dy: a column tile of the weights has fewer units than a workgroup has threads."""
    rng = np.random.default_rng([n, n_in, n_out])
    x, w, dy = _linear(rng, n, G, n_in, n_out, dtype)
    ids = draw_ids(rng, n, G, "holes")
    offsets, order = cg.group_rows(dev(ids), G)
    dx, _ = cg.grouped_linear_grad(*(dev(t, dtype) for t in (x, w, dy)), offsets, order, dw=False)
    check(dx, ref.grouped_grad(x, w, dy, ids, dtype)[0], "dx")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("r", [1, 4, 12, 24])
@pytest.mark.parametrize("n,G,n_in,n_out", [(300, 2, 64, 128), (300, 2, 40, 131), (300, 80, 64, 128), (300, 2, 140, 72)])
def test_adapter_infinite_inputs(cg, dtype, r, n, G, n_in, n_out):
    """Infinite inputs meet weights of one sign: infinite rows, no NaN, and no other rows."""
    rng = np.random.default_rng([n, n_in, r])
    x, w, a, b, _, _ = _adapters(rng, n, G, n_in, n_out, r, dtype)
    w, a, b = (np.abs(t) + 2.0 ** -10 for t in (w, a, b))
    w, a, b = (rounded(t, dtype) for t in (w, a, b))
    ids = draw_ids(rng, n, G, "even")
    one = np.ones(G)
    want, bound = ref.adapter(x, w, a, b, one, ids, dtype)
    bad = {3: np.inf, 100: -np.inf, 101: np.inf, 299: -np.inf}
    for row, value in bad.items():
        x[row, row % n_in] = value
    offsets, order = cg.group_rows(dev(ids), G)
    y = host(cg.adapter_linear(*(dev(t, dtype) for t in (x, w, a, b)), offsets, order))
    fine = np.setdiff1d(np.arange(n), list(bad))
    assert np.all(np.abs(y - want)[fine] <= bound[fine])
    for row, value in bad.items():
        assert (y[row] == value).all(), row
