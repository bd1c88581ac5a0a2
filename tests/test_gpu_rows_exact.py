"""Row operators on operands whose sums fp32 holds exactly, at any order: results are equal, not near."""
from __future__ import annotations

import numpy as np
import pytest

from tests.test_gpu_rows import cg, dev, host  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,G,n_in,n_out,r", [
    (700, 2, 64, 448, 8), (700, 2, 64, 200, 16), (900, 3, 40, 131, 32), (300, 90, 64, 200, 24), (300, 90, 33, 72, 4),
    (500, 2, 100, 60, 6), (500, 2, 200, 300, 64), (500, 2, 131, 40, 17), (64, 64, 48, 40, 8), (2000, 700, 64, 200, 24), (2000, 700, 40, 72, 4)])
def test_adapter_between_the_products(cg, dtype, n, G, n_in, n_out, r):
    """The narrow products between an adapter's two matrices are held in 24 bits. Operands are whole numbers;
    those products pass 2^18, and meet another of the same adapter that differs in one term, times -1."""
    rng = np.random.default_rng([n, G, n_in, n_out, r])
    top = min(255, int((2 ** 24 / max(n_in, n_out)) ** 0.5))
    whole = lambda *s: rng.integers(top // 2, top + 1, s).astype(np.float64)
    ids = np.sort(rng.integers(0, G, n)).astype(np.int32)
    offsets, order = cg.group_rows(dev(ids), G)
    w = np.zeros((n_in, n_out))

    # y = h_0 - h_1, and h_0 - h_1 = x_0
    x, a, b = whole(n, n_in), np.zeros((G, n_in, r)), np.zeros((G, r, n_out))
    a[:, :, 0] = whole(G, n_in)
    a[:, :, 1] = a[:, :, 0]
    a[:, 0, 1] -= 1
    b[:, 0], b[:, 1] = 1, -1
    X, W, A, B = (dev(t, dtype) for t in (x, w, a, b))
    assert np.array_equal(host(cg.adapter_linear(X, W, A, B, offsets, order)), np.repeat(x[:, :1], n_out, 1))

    # db_0 - db_1 by the rows: pairs of rows of a group that differ in one term and meet dy and -dy
    pair = np.arange(n // 2 * 2).reshape(-1, 2)
    pair = pair[ids[pair[:, 0]] == ids[pair[:, 1]]]
    xp, dy = np.zeros((n, n_in)), np.zeros((n, n_out))
    pick = pair[np.unique(ids[pair[:, 0]], return_index=True)[1]]     # one pair a group: sums of two terms
    xp[pick[:, 0]] = whole(len(pick), n_in)
    xp[pick[:, 1]] = xp[pick[:, 0]]
    xp[pick[:, 1], 0] -= 1
    dy[pick[:, 0]], dy[pick[:, 1]] = 1, -1
    want = np.zeros((G, r, n_out))
    want[ids[pick[:, 0]]] = a[ids[pick[:, 0]], 0][:, :, None]
    _, _, db = cg.adapter_linear_grad(dev(xp, dtype), W, A, B, dev(dy, dtype), offsets, order, dx=False, da=False)
    assert np.array_equal(host(db), want)

    # dx = u_0 - u_1 = dy_0 where b's first two rows differ in one term
    b = np.zeros((G, r, n_out))
    b[:, 0] = whole(G, n_out)
    b[:, 1] = b[:, 0]
    b[:, 1, 0] -= 1
    a = np.zeros((G, n_in, r))
    a[:, :, 0], a[:, :, 1] = 1, -1
    dyw = whole(n, n_out)
    A, B = dev(a, dtype), dev(b, dtype)
    both = cg.adapter_linear_grad(X, W, A, B, dev(dyw, dtype), offsets, order, db=False)
    assert np.array_equal(host(both[0]), np.repeat(dyw[:, :1], n_in, 1))
    # da by the rows, as db: x = 1 and -1 meet u's that differ by b's first column
    xs, dyp = np.zeros((n, n_in)), np.zeros((n, n_out))
    xs[pick[:, 0]], xs[pick[:, 1]] = 1, -1
    dyp[pick[:, 0]] = whole(len(pick), n_out)
    dyp[pick[:, 1]] = dyp[pick[:, 0]]
    dyp[pick[:, 1], 0] -= 1
    want = np.zeros((G, n_in, r))
    want[ids[pick[:, 0]]] = b[ids[pick[:, 0]], :, 0][:, None, :]
    for dx in (False, None):
        _, da, _ = cg.adapter_linear_grad(dev(xs, dtype), W, A, B, dev(dyp, dtype), offsets, order, dx=dx, db=False)
        assert np.array_equal(host(da), want)
