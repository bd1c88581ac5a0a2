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
@pytest.mark.parametrize("n,G,n_in,n_out", [(300, 2, 64, 128), (300, 2, 40, 131), (300, 80, 64, 128), (300, 2, 140, 72),
                                            (2000, 700, 64, 128), (2000, 700, 40, 131), (2000, 700, 140, 72)])
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


def _beside(rng, shape, tiny, axis):
    """Ones beside values of the size of `tiny`: half and half along an axis; and where the tiny ones are."""
    small = np.zeros(shape[axis], bool)
    small[rng.permutation(shape[axis])[: (shape[axis] + 1) // 2]] = True
    small = np.moveaxis(np.broadcast_to(small, np.moveaxis(np.empty(shape), axis, -1).shape), -1, axis)
    v = np.where(small, rng.uniform(1, 2, shape) * rng.choice([-1, 1], shape) * tiny, 1.0)
    return rounded(v, "f32"), small


def _sums(x, w, U=2.0 ** -23):
    """(value, bound) of x @ w: no slack for what is small in itself."""
    value, mag = x @ w, np.abs(x) @ np.abs(w)
    return value, U * (x.shape[1] + 4) * mag + 2.0 ** -149


PRODUCTS = [(300, 2, 64, 130), (300, 2, 16, 200), (300, 2, 9, 72), (300, 2, 130, 72), (700, 3, 96, 40), (300, 1, 200, 200),
            (90, 60, 64, 65), (200, 40, 70, 130)]


@pytest.mark.parametrize("tiny", [1e-30, 2.0 ** -109, 1.2345678e-37, 1e-38, 2.0 ** -130, 3 * 2.0 ** -149])
@pytest.mark.parametrize("n,G,n_in,n_out", PRODUCTS)
def test_fp32_tiny_beside_ordinary(cg, tiny, n, G, n_in, n_out):
    """Tiny values that meet large ones, beside ordinary values that meet zeros, keep fp32's precision."""
    rng = np.random.default_rng([n, n_in])
    ids = np.sort(draw_ids(rng, n, G, "even"))
    offsets, order = cg.group_rows(dev(ids), G)
    large = 0.25 / tiny if tiny > 2.0 ** -126 else 2.0 ** 124
    match = lambda small: rounded(np.where(small, rng.uniform(1, 2, small.shape) * large, 0.0), "f32")

    x, small = _beside(rng, (n, n_in), tiny, 1)
    w = match(np.broadcast_to(small[:1].T[None], (G, n_in, n_out)))
    y = host(cg.grouped_linear(dev(x), dev(w), offsets, order))
    w2, small = _beside(rng, (G, n_in, n_out), tiny, 2)
    dy = match(np.broadcast_to(small[0, :1], (n, n_out)))
    dx, _ = cg.grouped_linear_grad(dev(x), dev(w2), dev(dy), offsets, order, dw=False)
    x3, small = _beside(rng, (n, n_in), tiny, 0)
    dy3 = match(np.broadcast_to(small[:, :1], (n, n_out)))
    _, dw = cg.grouped_linear_grad(dev(x3), dev(w), dev(dy3), offsets, order, dx=False)
    for g in range(G):
        rows = np.flatnonzero(ids == g)
        for got, (want, bound), name in ((y[rows], _sums(x[rows], w[g]), "y"), (host(dx)[rows], _sums(dy[rows], w2[g].T), "dx"),
                                         (host(dw)[g], _sums(x3[rows].T, dy3[rows]), "dw")):
            err = np.abs(got - want)
            assert np.all(err <= bound), (name, g, float((err / bound).max()))


@pytest.mark.parametrize("tiny", [1.2345678e-37, 2.0 ** -130, 3 * 2.0 ** -149])
@pytest.mark.parametrize("n,G,n_in,n_out,r", [(300, 2, 64, 130, 8), (300, 60, 64, 72, 16), (300, 2, 200, 72, 20),
                                              (400, 2, 70, 40, 40), (2000, 700, 64, 130, 8)])
def test_fp32_adapter_tiny_beside_ordinary(cg, tiny, n, G, n_in, n_out, r):
    """The same through an adapter: a^T x from tiny inputs, and tiny values of b beside ordinary ones."""
    rng = np.random.default_rng([n, n_in, r])
    ids = np.sort(draw_ids(rng, n, G, "even"))
    offsets, order = cg.group_rows(dev(ids), G)
    large = 0.25 / tiny if tiny > 2.0 ** -126 else 2.0 ** 124
    x, small = _beside(rng, (n, n_in), tiny, 1)
    a = rounded(np.where(small[:1].T[None], rng.uniform(1, 2, (G, n_in, r)) * large, 0.0), "f32")
    b = rounded(rng.uniform(1, 2, (G, r, n_out)), "f32")
    w = np.zeros((n_in, n_out))
    y = host(cg.adapter_linear(dev(x), dev(w), dev(a), dev(b), offsets, order))
    b2, small = _beside(rng, (G, r, n_out), tiny, 2)
    dy = rounded(np.where(small[0, :1], rng.uniform(1, 2, (n, n_out)) * large, 0.0), "f32")
    a2 = rounded(rng.uniform(1, 2, (G, n_in, r)), "f32")
    x2 = rounded(rng.uniform(1, 2, (n, n_in)), "f32")
    dx, da, _ = (host(t) for t in cg.adapter_linear_grad(dev(x2), dev(w), dev(a2), dev(b2), dev(dy), offsets, order))
    U = 2.0 ** -23
    for g in range(G):
        rows = np.flatnonzero(ids == g)
        h, hm = x[rows] @ a[g], np.abs(x[rows]) @ np.abs(a[g])
        u, um = dy[rows] @ b2[g].T, np.abs(dy[rows]) @ np.abs(b2[g]).T
        for got, want, mag, terms, name in ((y[rows], h @ b[g], hm @ b[g], n_in + r, "y"), (dx[rows], u @ a2[g].T, um @ a2[g].T, n_out + r, "dx"),
                                            (da[g], x2[rows].T @ u, x2[rows].T @ um, len(rows) + n_out, "da")):
            err = np.abs(got - want)
            assert np.all(err <= U * (terms + 8) * mag + 2.0 ** -140), (name, g, float((err / (mag + 1e-300)).max()))


@pytest.mark.parametrize("n,G,n_in,n_out", PRODUCTS + [(3000, 1, 130, 72)])
@pytest.mark.parametrize("size", [1e10, 1e15, 1e18, 1e25, 1e37])
def test_fp32_large_products(cg, size, n, G, n_in, n_out):
    """Sums up to fp32's largest are as fp32 gives them; beyond it, infinities of the terms' sign and no NaN."""
    rng = np.random.default_rng([n, n_in])
    ids = draw_ids(rng, n, G, "even")
    offsets, order = cg.group_rows(dev(ids), G)
    x, w, dy = (rounded(rng.uniform(1, 2, s) * size, "f32") for s in ((n, n_in), (G, n_in, n_out), (n, n_out)))
    turn = rng.choice([-1.0, 1.0], n)           # whole rows of one sign
    x *= turn[:, None]
    y = host(cg.grouped_linear(dev(x), dev(w), offsets, order))
    dx, dw = (host(t) for t in cg.grouped_linear_grad(dev(np.abs(x)), dev(w), dev(dy), offsets, order))
    for g in range(G):
        rows = np.flatnonzero(ids == g)
        for got, (want, bound), name in ((y[rows], _sums(x[rows], w[g]), "y"), (dx[rows], _sums(dy[rows], w[g].T), "dx"),
                                         (dw[g], _sums(np.abs(x[rows]).T, dy[rows]), "dw")):
            fine, over = np.abs(want) < 3.4e38, np.abs(want) > 3.41e38
            with np.errstate(all="ignore"):
                assert np.all((np.abs(got - want) <= bound)[fine]), name
            assert np.array_equal(got[over], np.sign(want[over]) * np.inf), name
            assert not np.isnan(got).any(), name


@pytest.mark.parametrize("n,G,n_in,n_out", PRODUCTS)
def test_fp32_largest_finite_product(cg, n, G, n_in, n_out):
    """Terms whose parts round up past fp32's largest, though the product does not."""
    ids = np.arange(n, dtype=np.int32) % G
    offsets, order = cg.group_rows(dev(ids), G)
    big = (2.0 ** 24 - 1) * 2.0 ** 40           # squared: 2^128 (1 - 2^-23) and a little, rounded to fp32 below it
    x, w, dy = np.zeros((n, n_in)), np.zeros((G, n_in, n_out)), np.zeros((n, n_out))
    x[:, 2], w[:, 2, :] = big, big
    want = float(np.float32(big * big))
    assert np.isfinite(want)
    assert (host(cg.grouped_linear(dev(x), dev(w), offsets, order)) == want).all()
    dy[:, 3] = big
    dx, dw = cg.grouped_linear_grad(dev(x * (np.arange(n) < G)[:, None]), dev(w), dev(dy), offsets, order)
    assert (host(dx)[:, 2] == want).all() and (np.delete(host(dx), 2, 1) == 0).all()
    assert (host(dw)[:, 2, 3] == want).all()


@pytest.mark.parametrize("n,G,n_in,n_out", [(400, 5, 64, 130), (400, 5, 130, 72), (500, 200, 40, 72), (400, 5, 96, 30)])
def test_fp32_infinite_row_leaves_other_bits(cg, n, G, n_in, n_out):
    """An infinite input changes the bits of its own row alone, and of its group's weight gradient."""
    rng = np.random.default_rng([n, n_in])
    x, w, dy = _linear(rng, n, G, n_in, n_out, "f32")
    ids = draw_ids(rng, n, G, "even")
    offsets, order = cg.group_rows(dev(ids), G)
    X, W, DY = dev(x), dev(w), dev(dy)
    run = lambda: (cg.grouped_linear(X, W, offsets, order), *cg.grouped_linear_grad(X, W, DY, offsets, order))
    clean = run()
    X[0, 3] = DY[0, 5] = float("inf")
    y, dx, dw = run()
    assert (y[1:] == clean[0][1:]).all() and (dx[1:] == clean[1][1:]).all()
    others = np.arange(G) != ids[0]
    assert (dw[others] == clean[2][others]).all()
    keep = np.arange(n_in) != 3, np.arange(n_out) != 5
    mine = int(ids[0])
    assert (dw[mine][keep[0]][:, keep[1]] == clean[2][mine][keep[0]][:, keep[1]]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,G,n_in,n_out,r", [(300, 2, 64, 128, 4), (300, 2, 40, 131, 20), (300, 80, 64, 128, 8),
                                              (300, 2, 140, 72, 16), (300, 2, 100, 200, 12), (300, 2, 72, 140, 40),
                                              (2000, 700, 64, 128, 8), (2000, 700, 40, 131, 20), (2000, 700, 140, 72, 16)])
def test_adapter_infinite_weights_and_gradients(cg, dtype, n, G, n_in, n_out, r):
    """An infinite weight of an adapter, or an infinite row, among values of one sign: infinities, as fp32 sums
    give, and no NaN; other adapters' rows and gradients as without it."""
    rng = np.random.default_rng([n, n_in, r])
    x, w, a, b, dy, _ = (rounded(np.abs(t) + 2.0 ** -10, dtype) for t in _adapters(rng, n, G, n_in, n_out, r, dtype))
    ids = draw_ids(rng, n, G, "even")
    offsets, order = cg.group_rows(dev(ids), G)
    one = np.ones(G)
    mine, D = ids == ids[0], lambda *s: [dev(t, dtype) for t in s]
    put = lambda t, *at: (lambda c: (c.__setitem__(at, np.inf), c)[1])(t.copy())

    want, bound = ref.adapter(x, w, a, b, one, ids, dtype)
    wants = ref.adapter_grad(x, w, a, b, dy, one, ids, dtype)

    def near(got, exp, where):
        got = host(got)
        assert np.all(np.abs(got - exp[0])[where] <= exp[1][where])

    inf = lambda t: bool((host(t) == np.inf).all())
    y = cg.adapter_linear(*D(x, w, a, put(b, ids[0], 1, 5)), offsets, order)
    assert inf(y[np.flatnonzero(mine)][:, 5])
    near(y, (want, bound), ~mine)
    near(y[:, :5], (want[:, :5], bound[:, :5]), slice(None))
    dx, _, db = cg.adapter_linear_grad(*D(x, w, put(a, ids[0], 7, 2), b, dy), offsets, order)
    assert inf(dx[np.flatnonzero(mine)][:, 7])
    near(dx, wants[0], ~mine)
    assert inf(db[int(ids[0]), 2])
    xi, dyi = put(x, 0, 3), put(dy, 0, 6)
    _, da, db = cg.adapter_linear_grad(*D(xi, w, a, b, dy), offsets, order)
    assert inf(da[int(ids[0]), 3]) and inf(db[int(ids[0])])
    others = np.arange(G) != ids[0]
    near(da, wants[1], others)
    keep = np.arange(n_in) != 3
    near(da[int(ids[0])][keep], (wants[1][0][ids[0]][keep], wants[1][1][ids[0]][keep]), slice(None))
    dx, da, db = cg.adapter_linear_grad(*D(x, w, a, b, dyi), offsets, order)
    assert inf(dx[0]) and inf(da[int(ids[0])]) and inf(db[int(ids[0]), :, 6])
    near(dx[1:], (wants[0][0][1:], wants[0][1][1:]), slice(None))
    near(db, wants[2], others)


@pytest.mark.parametrize("value", [float("inf"), float("nan"), 3e38])
@pytest.mark.parametrize("n,G,n_in,n_out", [(900, 90, 130, 72), (900, 90, 64, 40), (900, 5, 200, 140)])
def test_fp32_first_row_of_the_input_is_no_other_tiles(cg, value, n, G, n_in, n_out):
    """Partly filled tiles, and places that order leaves out, take nothing from row 0."""
    import torch

    rng = np.random.default_rng([n, n_in])
    x, w, _ = _linear(rng, n, G, n_in, n_out, "f32")
    ids = draw_ids(rng, n, G, "even")
    offsets, order = cg.group_rows(dev(ids), G)
    order[17] = -1
    X, W = dev(x), dev(w)
    clean = cg.grouped_linear(X, W, offsets, order, y=torch.zeros(n, n_out, device="cuda"))
    X[0] = value
    y = cg.grouped_linear(X, W, offsets, order, y=torch.zeros(n, n_out, device="cuda"))
    assert torch.equal(y[1:], clean[1:])


@pytest.mark.parametrize("n,n_in,n_out,adapter", [(2 ** 31 - 1, 1, 1, False), (2 ** 30 + 1000, 1, 33, False),
                                                  (2 ** 30 + 1000, 1, 33, True)])
def test_as_many_rows_as_there_may_be(cg, n, n_in, n_out, adapter):
    """Launches of 2^32 threads and more."""
    import torch

    one = lambda *s: torch.ones(*s, dtype=torch.bfloat16, device="cuda")
    offsets = torch.tensor([0, n - 7], dtype=torch.int32, device="cuda")
    x, y = one(n, n_in), torch.empty(n, n_out, dtype=torch.bfloat16, device="cuda")
    ends = torch.tensor([0, 1, n // 2, n - 9, n - 8, n - 7, n - 1], device="cuda")
    x[ends] = torch.arange(2, 9, device="cuda", dtype=torch.bfloat16)[:, None]
    if adapter:
        cg.adapter_linear(x, one(n_in, n_out), one(1, n_in, 1), one(1, 1, n_out), offsets, y=y)
        inside, outside = 2, 1
    else:
        cg.grouped_linear(x, one(1, n_in, n_out), offsets, y=y)
        inside, outside = 1, 0
    step = 1 << 26
    for at in range(0, n, step):
        end = min(at + step, n)
        want = x[at:end].clone()
        want[:max(0, n - 7 - at)] *= inside
        want[max(0, n - 7 - at):] *= outside
        assert torch.equal(y[at:end], want.expand(end - at, n_out)), at
