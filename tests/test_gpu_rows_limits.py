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
