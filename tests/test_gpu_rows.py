"""Row operators (row order by group, grouped products, adapters and their gradients) against the
64-bit reference, at the sizes, masks, strides and types where they can go wrong."""
from __future__ import annotations

import numpy as np
import pytest

from tests import rows_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cg():
    import torch

    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2605_15073_amd as lib

    lib.load_library()
    return lib


def draw_ids(rng, n, G, kind):
    if kind == "even":
        return rng.integers(0, G, n).astype(np.int32)
    if kind == "none":                      # no row has a group
        return np.where(rng.random(n) < 0.5, -1, G + 5).astype(np.int32)
    if kind == "one":                       # all rows in one group, the others empty
        return np.full(n, G // 2, np.int32)
    if kind == "holes":                     # uneven, some rows and some groups bare
        ids = (G * rng.random(n) ** 3).astype(np.int32)
        ids[rng.random(n) < 0.25] = -1
        return ids
    raise ValueError(kind)


def dev(a, dtype="f32"):
    import torch

    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    if t.dtype == torch.float64:
        t = t.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    return t


def host(t):
    return t.double().cpu().numpy()


def rounded(a, dtype):
    """a as the type holds it, in 64 bits."""
    return host(dev(a, dtype))


def strided(t, pad):
    """t's rows at a stride of width + pad, in a buffer of NaN."""
    import torch

    if pad == 0:
        return t
    buf = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=t.device)
    view = buf[:, :t.shape[1]]
    view.copy_(t)
    return view


def check(got, want, what):
    value, bound = want
    err = np.abs(host(got) - value)
    assert np.all(err <= bound), (what, float((err / bound).max()))


# ---------------------------------------------------------------- row order

@pytest.mark.parametrize("n", [0, 1, 63, 64, 65, 513, 4096, 4097, 20000, 131072 + 1, 525308])
@pytest.mark.parametrize("G", [1, 5, 255, 4096])
@pytest.mark.parametrize("kind", ["even", "holes"])
def test_group_rows(cg, n, G, kind):
    ids = draw_ids(np.random.default_rng(n + G), n, G, kind)
    offsets, order = cg.group_rows(dev(ids), G)
    roff, rord = ref.order(ids, G)
    assert np.array_equal(offsets.cpu().numpy(), roff)
    assert np.array_equal(order.cpu().numpy(), rord)


@pytest.mark.parametrize("n", [1048576, 1048577, 3000000])
def test_group_rows_in_rounds(cg, n):
    """More rows than 256 chunks of one round hold."""
    for G in (3, 1000):
        ids = draw_ids(np.random.default_rng(n), n, G, "holes")
        offsets, order = cg.group_rows(dev(ids), G)
        roff, rord = ref.order(ids, G)
        assert np.array_equal(offsets.cpu().numpy(), roff)
        assert np.array_equal(order.cpu().numpy(), rord)


@pytest.mark.parametrize("n", [100, 30000])
@pytest.mark.parametrize("kind", ["none", "one"])
def test_group_rows_degenerate(cg, n, kind):
    ids = draw_ids(np.random.default_rng(1), n, 7, kind)
    ids[0] = -2 ** 31 if kind == "none" else ids[0]
    ids[-1] = 2 ** 31 - 1 if kind == "none" else ids[-1]
    offsets, order = cg.group_rows(dev(ids), 7)
    roff, rord = ref.order(ids, 7)
    assert np.array_equal(offsets.cpu().numpy(), roff)
    assert np.array_equal(order.cpu().numpy(), rord)


# ---------------------------------------------------------------- products

# rows, groups, widths: one row, odd ones, tile edges, narrow and wide, many small groups
SIZES = [(1, 1, 1, 1), (1, 3, 64, 64), (2, 5, 7, 3), (64, 5, 64, 64), (65, 2, 8, 129),
         (127, 1, 33, 128), (129, 3, 128, 130), (300, 7, 37, 129), (1000, 4, 64, 448),
         (1000, 400, 24, 40), (257, 2, 896, 72), (700, 3, 130, 257), (515, 2, 1, 300),
         (515, 2, 300, 1), (2050, 5, 16, 1344), (90, 80, 200, 130), (4099, 2, 48, 96)]


def _linear(rng, n, G, n_in, n_out, dtype):
    x = rounded(rng.standard_normal((n, n_in)), dtype)
    w = rounded(rng.standard_normal((G, n_in, n_out)) * n_in ** -0.5, dtype)
    dy = rounded(rng.standard_normal((n, n_out)), dtype)
    return x, w, dy


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,G,n_in,n_out", SIZES)
@pytest.mark.parametrize("kind", ["even", "holes"])
def test_grouped(cg, dtype, n, G, n_in, n_out, kind):
    rng = np.random.default_rng([n, G, n_in, n_out])
    x, w, dy = _linear(rng, n, G, n_in, n_out, dtype)
    ids = draw_ids(rng, n, G, kind)
    offsets, order = cg.group_rows(dev(ids), G)
    X, W, DY = (dev(t, dtype) for t in (x, w, dy))
    check(cg.grouped_linear(X, W, offsets, order), ref.grouped(x, w, ids, dtype), "y")
    want = ref.grouped_grad(x, w, dy, ids, dtype)
    dx, dw = cg.grouped_linear_grad(X, W, DY, offsets, order)
    check(dx, want[0], "dx")
    check(dw, want[1], "dw")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,G,n_in,n_out", [(1, 9, 1344, 448), (8, 8, 520, 70), (65, 40, 64, 64),
                                            (900, 400, 70, 90), (900, 400, 96, 32),
                                            (3000, 4096, 37, 129), (2500, 600, 129, 257)])
@pytest.mark.parametrize("kind", ["even", "one", "holes", "none", "spikes"])
def test_grouped_few_rows_a_group(cg, dtype, n, G, n_in, n_out, kind):
    """Many groups, few rows on the mean: all even, or some groups of many rows among empty ones."""
    rng = np.random.default_rng([n, G, n_in, n_out])
    x, w, dy = _linear(rng, n, G, n_in, n_out, dtype)
    if kind == "spikes":
        ids = draw_ids(rng, n, G, "even")
        ids[: n // 2] = rng.integers(0, min(G, 3), n // 2)
    else:
        ids = draw_ids(rng, n, G, kind)
    offsets, order = cg.group_rows(dev(ids), G)
    X, W, DY = (dev(t, dtype) for t in (x, w, dy))
    check(cg.grouped_linear(X, W, offsets, order), ref.grouped(x, w, ids, dtype), "y")
    want = ref.grouped_grad(x, w, dy, ids, dtype)
    dx, dw = cg.grouped_linear_grad(X, W, DY, offsets, order)
    check(dx, want[0], "dx")
    check(dw, want[1], "dw")


@pytest.mark.parametrize("n_in,n_out", [(600, 5), (5, 600), (129, 70), (9, 8), (70, 4), (3, 40), (33, 65)])
@pytest.mark.parametrize("kind", ["even", "holes"])
@pytest.mark.parametrize("pad", [0, 1, 4])
def test_grouped_few_rows_strided_and_masked(cg, n_in, n_out, kind, pad):
    """Few rows a group in fp32, one group of many: strides, bare rows that hold NaN and infinities,
    inputs with a place that order leaves out, and rows without values past their end."""
    import torch

    n, G = 230, 90
    rng = np.random.default_rng([n_in, n_out, pad])
    x, w, dy = _linear(rng, n, G, n_in, n_out, "f32")
    ids = draw_ids(rng, n, G, kind)
    ids[:77] = 4                              # more rows than a workgroup, or a weight gradient's form, takes
    bare = np.flatnonzero((ids < 0) | (ids >= G))
    xn, dyn = x.copy(), dy.copy()
    xn[bare], dyn[bare] = np.nan, np.inf
    x[bare], dy[bare] = 0, 0
    offsets, order = cg.group_rows(dev(ids), G)
    lost = int(order[3])
    order[3] = -7
    x[lost], dy[lost] = 0, 0
    X, DY, W = strided(dev(xn), pad), strided(dev(dyn), pad), dev(w)
    y = strided(torch.full((n, n_out), 7.0, device="cuda"), pad)
    dx = strided(torch.full((n, n_in), 7.0, device="cuda"), pad)
    cg.grouped_linear(X, W, offsets, order, y=y)
    _, dw = cg.grouped_linear_grad(X, W, DY, offsets, order, dx=dx)
    assert (y[lost] == 7).all() and (dx[lost] == 7).all()
    y[lost], dx[lost] = 0, 0
    check(y, ref.grouped(x, w, ids, "f32"), "y")
    want = ref.grouped_grad(x, w, dy, ids, "f32")
    check(dx, want[0], "dx")
    check(dw, want[1], "dw")
    for t in (y, dx):
        assert pad == 0 or torch.isnan(t._base[:, t.shape[1]:]).all()


@pytest.mark.parametrize("where", ["x", "w", "dy"])
@pytest.mark.parametrize("value", [1e-38, 3e-40, 3.3e38, float("inf")])
@pytest.mark.parametrize("n,n_in,n_out", [(300, 64, 130), (300, 130, 72), (700, 96, 40)])
def test_grouped_fp32_extremes(cg, where, value, n, n_in, n_out):
    """Values that bf16 parts cannot hold, beside ordinary ones: the results of fp32 sums."""
    rng = np.random.default_rng([n, n_in])
    x, w, dy = _linear(rng, n, 2, n_in, n_out, "f32")
    ids = draw_ids(rng, n, 2, "even")
    t = dict(x=x, w=w, dy=dy)[where]
    if value < 1:                            # a whole operand of tiny values
        t *= value / 4
        other = dict(x=w, w=x, dy=w)[where]
        other *= 1e30
        t[...] = rounded(t, "f32")
        other[...] = rounded(other, "f32")
    else:                                    # single large ones, times others below 1/8
        t[..., 3, :] = np.where(rng.random(t[..., 3, :].shape) < 0.2, value, 0)
        for u in (x, w, dy):
            if u is not t:
                u[...] = rounded(u / 64, "f32")
        t[...] = rounded(t, "f32")
    offsets, order = cg.group_rows(dev(ids), 2)
    X, W, DY = (dev(v) for v in (x, w, dy))
    with np.errstate(all="ignore"):
        want = [ref.grouped(x, w, ids, "f32"), *ref.grouped_grad(x, w, dy, ids, "f32")]
    got = [cg.grouped_linear(X, W, offsets, order), *cg.grouped_linear_grad(X, W, DY, offsets, order)]
    for g, (v, bound), name in zip(got, want, ("y", "dx", "dw")):
        g = host(g)
        fine = np.isfinite(v) & (np.abs(v) < 3e38)
        assert np.array_equal(np.isfinite(g) & (np.abs(g) < 3e38), fine), name
        assert np.all(np.abs(g - v)[fine] <= bound[fine]), name
        inf = np.isinf(v)
        assert np.array_equal(g[inf], v[inf]), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,G,n_in,n_out", [(300, 5, 40, 56), (131, 3, 37, 29), (5000, 2, 64, 64)])
@pytest.mark.parametrize("kind", ["none", "one", "holes"])
@pytest.mark.parametrize("pad", [1, 8])
def test_grouped_strided_and_masked(cg, dtype, n, G, n_in, n_out, kind, pad):
    """Strides wider than the rows; rows of no group hold NaN and infinities, which reach no output;
    the gaps between the rows of an output keep their contents."""
    import torch

    rng = np.random.default_rng([n, G, pad])
    x, w, dy = _linear(rng, n, G, n_in, n_out, dtype)
    ids = draw_ids(rng, n, G, kind)
    bare = np.flatnonzero((ids < 0) | (ids >= G))
    xn, dyn = x.copy(), dy.copy()
    xn[bare], dyn[bare] = np.nan, np.inf
    xz, dyz = x.copy(), dy.copy()
    xz[bare], dyz[bare] = 0, 0
    offsets, order = cg.group_rows(dev(ids), G)
    X, DY, W = strided(dev(xn, dtype), pad), strided(dev(dyn, dtype), pad), dev(w, dtype)
    y = strided(torch.full((n, n_out), float("nan"), dtype=X.dtype, device="cuda"), pad)
    dx = strided(torch.full((n, n_in), float("nan"), dtype=X.dtype, device="cuda"), pad)
    dw = torch.full_like(W, float("nan"))
    cg.grouped_linear(X, W, offsets, order, y=y)
    cg.grouped_linear_grad(X, W, DY, offsets, order, dx=dx, dw=dw)
    check(y, ref.grouped(xz, w, ids, dtype), "y")
    want = ref.grouped_grad(xz, w, dyz, ids, dtype)
    check(dx, want[0], "dx")
    check(dw, want[1], "dw")
    for t in (y, dx):
        assert torch.isnan(t._base[:, t.shape[1]:]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_grouped_sorted_rows_need_no_order(cg, dtype):
    rng = np.random.default_rng(3)
    x, w, dy = _linear(rng, 777, 6, 64, 72, dtype)
    ids = np.sort(rng.integers(0, 6, 777)).astype(np.int32)
    ids[-40:] = 6                            # the tail has no group
    offsets, order = cg.group_rows(dev(ids), 6)
    X, W, DY = (dev(t, dtype) for t in (x, w, dy))
    with_order = cg.grouped_linear(X, W, offsets, order)
    assert (with_order == cg.grouped_linear(X, W, offsets)).all()
    check(with_order, ref.grouped(x, w, ids, dtype), "y")
    for a, b in zip(cg.grouped_linear_grad(X, W, DY, offsets, order),
                    cg.grouped_linear_grad(X, W, DY, offsets)):
        assert (a == b).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n_in,n_out", [(64, 72), (37, 41)])
def test_grouped_non_finite_rows_stay_to_themselves(cg, dtype, n_in, n_out):
    """An infinite or NaN input spoils its own row of y and its group's dw, nothing else; an infinite
    one gives the infinities that the sum has."""
    rng = np.random.default_rng(4)
    x, w, dy = _linear(rng, 200, 3, n_in, n_out, dtype)
    ids = draw_ids(rng, 200, 3, "even")
    ids[[5, 9]] = 0, 1
    clean = ref.grouped(x, w, ids, dtype)
    xb = x.copy()
    xb[5, 3], xb[9, 0] = np.nan, np.inf
    offsets, order = cg.group_rows(dev(ids), 3)
    X, W = dev(xb, dtype), dev(w, dtype)
    y = host(cg.grouped_linear(X, W, offsets, order))
    others = np.setdiff1d(np.arange(200), [5, 9])
    assert np.all(np.abs(y - clean[0])[others] <= clean[1][others])
    assert np.isnan(y[5]).all()
    assert np.array_equal(y[9], np.sign(w[1, 0]) * np.inf)
    _, dw = cg.grouped_linear_grad(X, W, dev(dy, dtype), offsets, order, dx=False)
    want, bound = ref.grouped_grad(x, w, dy, ids, dtype)[1]
    assert np.all(np.abs(host(dw)[2] - want[2]) <= bound[2])
    assert np.isnan(host(dw)[0, 3]).all()
    keep = np.arange(n_in) != 3
    assert np.all(np.abs(host(dw)[0, keep] - want[0, keep]) <= bound[0, keep])
    assert np.array_equal(host(dw)[1, 0], np.sign(dy[9]) * np.inf)


@pytest.mark.parametrize("scale", [1e-30, 1e30])
def test_grouped_fp32_range(cg, scale):
    """fp32 operands of very small and very large magnitude keep fp32's precision."""
    rng = np.random.default_rng(5)
    x = rounded(rng.standard_normal((300, 96)) * scale, "f32")
    w = rounded(rng.standard_normal((2, 96, 160)), "f32")
    ids = draw_ids(rng, 300, 2, "even")
    offsets, order = cg.group_rows(dev(ids), 2)
    check(cg.grouped_linear(dev(x), dev(w), offsets, order), ref.grouped(x, w, ids, "f32"), "y")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_grouped_empty(cg, dtype):
    import torch

    offsets, order = cg.group_rows(torch.zeros(0, dtype=torch.int32, device="cuda"), 3)
    w = dev(np.ones((3, 5, 7)), dtype)
    x, dy = w.new_empty(0, 5), w.new_empty(0, 7)
    assert cg.grouped_linear(x, w, offsets, order).shape == (0, 7)
    dx, dw = cg.grouped_linear_grad(x, w, dy, offsets, order, dw=torch.full_like(w, float("nan")))
    assert dx.shape == (0, 5) and (dw == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_grouped_gradient_against_differences(cg, dtype):
    """y is linear in x and in w: <dy, y(x + e) - y(x)> = <dx, e>, and the same for w, up to the
    rounding of the two products."""
    rng = np.random.default_rng(6)
    n, G, n_in, n_out = 210, 4, 40, 56
    x, w, dy = _linear(rng, n, G, n_in, n_out, dtype)
    e, f, _ = _linear(rng, n, G, n_in, n_out, dtype)
    x2, w2 = rounded(x + e, dtype), rounded(w + f, dtype)
    ids = draw_ids(rng, n, G, "holes")
    offsets, order = cg.group_rows(dev(ids), G)
    run = lambda a, b: host(cg.grouped_linear(dev(a, dtype), dev(b, dtype), offsets, order))
    dx, dw = cg.grouped_linear_grad(*(dev(t, dtype) for t in (x, w, dy)), offsets, order)
    y, yb = run(x, w), ref.grouped(x, w, ids, dtype)[1]
    (_, dxb), (_, dwb) = ref.grouped_grad(x, w, dy, ids, dtype)
    for y2, bound2, grad, gb, step in (
            (run(x2, w), ref.grouped(x2, w, ids, dtype)[1], dx, dxb, x2 - x),
            (run(x, w2), ref.grouped(x, w2, ids, dtype)[1], dw, dwb, w2 - w)):
        lhs, rhs = (dy * (y2 - y)).sum(), (host(grad) * step).sum()
        assert abs(lhs - rhs) <= (np.abs(dy) * (yb + bound2)).sum() + (gb * np.abs(step)).sum()


def test_grouped_beyond_32_bit_offsets(cg):
    """More than 2^31 elements of input and of output."""
    import torch

    n, n_in, n_out = 1300000, 1704, 1712
    rows = torch.arange(n, device="cuda", dtype=torch.int32)
    ids = (rows % 3).contiguous()
    offsets, order = cg.group_rows(ids, 3)
    x = torch.zeros(n, n_in, dtype=torch.bfloat16, device="cuda")
    x[:, 5] = (rows % 128).to(torch.bfloat16)
    w = torch.zeros(3, n_in, n_out, dtype=torch.bfloat16, device="cuda")
    w[:, 5, :] = torch.arange(1, 4, device="cuda")[:, None].to(torch.bfloat16)
    y = cg.grouped_linear(x, w, offsets, order)
    assert torch.equal(y[:, 0].float(), ((rows % 128) * (rows % 3 + 1)).to(torch.bfloat16).float())
    assert torch.equal(y[:, -1], y[:, 0])
    dx, _ = cg.grouped_linear_grad(x, w, y, offsets, order, dw=False)
    want = (y[:, 0].float() * n_out * (rows % 3 + 1)).to(torch.bfloat16)
    assert torch.equal(dx[:, 5], want) and (dx[:, 6:].abs().amax() == 0)


# ---------------------------------------------------------------- adapters

def _adapters(rng, n, G, n_in, n_out, r, dtype):
    x = rounded(rng.standard_normal((n, n_in)), dtype)
    w = rounded(rng.standard_normal((n_in, n_out)) * n_in ** -0.5, dtype)
    a = rounded(rng.standard_normal((G, n_in, r)) * n_in ** -0.5, dtype)
    b = rounded(rng.standard_normal((G, r, n_out)) * r ** -0.5, dtype)
    dy = rounded(rng.standard_normal((n, n_out)), dtype)
    scale = rounded(rng.uniform(-2, 2, G), "f32")
    return x, w, a, b, dy, scale


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,G,n_in,n_out,r", [
    (1, 1, 1, 1, 1), (1, 4, 64, 448, 8), (48, 12, 64, 448, 8), (70, 40, 33, 65, 3),
    (129, 3, 128, 130, 16), (300, 2, 37, 129, 64), (1000, 7, 64, 896, 16), (400, 300, 24, 40, 5),
    (257, 2, 896, 72, 33), (2050, 5, 16, 1344, 32), (3000, 1, 130, 72, 12)])
@pytest.mark.parametrize("kind", ["even", "holes"])
def test_adapter(cg, dtype, n, G, n_in, n_out, r, kind):
    rng = np.random.default_rng([n, G, n_in, n_out, r])
    x, w, a, b, dy, scale = _adapters(rng, n, G, n_in, n_out, r, dtype)
    ids = draw_ids(rng, n, G, kind)
    offsets, order = cg.group_rows(dev(ids), G)
    X, W, A, B, DY = (dev(t, dtype) for t in (x, w, a, b, dy))
    S = dev(scale)
    check(cg.adapter_linear(X, W, A, B, offsets, order, scale=S),
          ref.adapter(x, w, a, b, scale, ids, dtype), "y")
    want = ref.adapter_grad(x, w, a, b, dy, scale, ids, dtype)
    for got, exp, what in zip(cg.adapter_linear_grad(X, W, A, B, DY, offsets, order, scale=S), want,
                              ("dx", "da", "db")):
        check(got, exp, what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,G,n_in,n_out,r", [
    (1500, 3, 64, 200, 16), (1500, 3, 128, 72, 8), (900, 9, 40, 131, 4), (1300, 2, 121, 90, 32),
    (700, 1, 16, 96, 1), (2100, 4, 64, 129, 24), (3000, 300, 64, 200, 8), (3000, 300, 33, 131, 20)])
@pytest.mark.parametrize("kind", ["even", "holes", "one", "none"])
def test_adapter_forms(cg, dtype, n, G, n_in, n_out, r, kind):
    """Adapters with tiles of their own, whose narrow products are formed inside the shared one, and
    tiles that many adapters share."""
    rng = np.random.default_rng([n, G, n_in, n_out, r, 7])
    x, w, a, b, dy, scale = _adapters(rng, n, G, n_in, n_out, r, dtype)
    ids = draw_ids(rng, n, G, kind)
    offsets, order = cg.group_rows(dev(ids), G)
    X, W, A, B, DY = (dev(t, dtype) for t in (x, w, a, b, dy))
    S = dev(scale)
    check(cg.adapter_linear(X, W, A, B, offsets, order, scale=S),
          ref.adapter(x, w, a, b, scale, ids, dtype), "y")
    want = ref.adapter_grad(x, w, a, b, dy, scale, ids, dtype)
    grads = cg.adapter_linear_grad(X, W, A, B, DY, offsets, order, scale=S)
    for got, exp, what in zip(grads, want, ("dx", "da", "db")):
        check(got, exp, what)
    alone = [cg.adapter_linear_grad(X, W, A, B, DY, offsets, order, scale=S,
                                    **{k: False for k in ("dx", "da", "db") if k != keep})
             for keep in ("dx", "da", "db")]
    check(alone[0][0], want[0], "dx alone")
    check(alone[1][1], want[1], "da alone")
    check(alone[2][2], want[2], "db alone")


@pytest.mark.parametrize("where", ["x", "w", "a", "b", "dy"])
@pytest.mark.parametrize("value", [1e-38, float("inf")])
@pytest.mark.parametrize("n,G,n_in,n_out,r", [(400, 2, 64, 130, 8), (400, 2, 100, 72, 16),
                                              (600, 40, 64, 72, 8)])
def test_adapter_fp32_extremes(cg, where, value, n, G, n_in, n_out, r):
    """Values that bf16 parts cannot hold: the results of fp32 sums, infinities where those have them."""
    rng = np.random.default_rng([n, n_in])
    t = dict(zip(("x", "w", "a", "b", "dy"), _adapters(rng, n, G, n_in, n_out, r, "f32")[:5]))
    ids = draw_ids(rng, n, G, "even")
    if value < 1:
        t[where] = rounded(t[where] * value, "f32")
    else:
        flat = t[where].reshape(-1)
        flat[5] = value                      # the first row of x or dy, of w, of the first adapter
    one = np.ones(G)
    offsets, order = cg.group_rows(dev(ids), G)
    X, W, A, B, DY = (dev(t[k]) for k in ("x", "w", "a", "b", "dy"))
    with np.errstate(all="ignore"):
        want = [ref.adapter(t["x"], t["w"], t["a"], t["b"], one, ids, "f32"),
                *ref.adapter_grad(t["x"], t["w"], t["a"], t["b"], t["dy"], one, ids, "f32")]
    got = [cg.adapter_linear(X, W, A, B, offsets, order),
           *cg.adapter_linear_grad(X, W, A, B, DY, offsets, order)]
    for g, (v, bound), name in zip(got, want, ("y", "dx", "da", "db")):
        g = host(g)
        fine = np.isfinite(v) & np.isfinite(bound)
        # a product between that underflows loses its own smallest step, 2^-149, times what follows
        slack = 2.0 ** -149 * 4096 * 16
        assert np.isfinite(g[fine]).all(), name
        assert np.all(np.abs(g - v)[fine] <= bound[fine] + slack), name
        assert not np.isfinite(g[~fine]).any(), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, 3, 8])
def test_adapter_strided_bare_rows_and_no_scale(cg, dtype, pad):
    """Rows of no adapter get the shared projection alone; their NaN reaches no adapter's gradient."""
    import torch

    rng = np.random.default_rng(pad)
    n, G, n_in, n_out, r = 260, 4, 64, 56, 16
    x, w, a, b, dy, _ = _adapters(rng, n, G, n_in, n_out, r, dtype)
    one = np.ones(G)
    ids = draw_ids(rng, n, G, "holes")
    offsets, order = cg.group_rows(dev(ids), G)
    W, A, B = (dev(t, dtype) for t in (w, a, b))
    X, DY = strided(dev(x, dtype), pad), strided(dev(dy, dtype), pad)
    y = strided(torch.full((n, n_out), float("nan"), dtype=X.dtype, device="cuda"), pad)
    cg.adapter_linear(X, W, A, B, offsets, order, y=y)
    check(y, ref.adapter(x, w, a, b, one, ids, dtype), "y")
    if pad:
        assert torch.isnan(y._base[:, n_out:]).all()
    bare = torch.from_numpy(np.flatnonzero(ids < 0)).cuda()
    X[bare] = float("nan")
    DY[bare] = float("nan")
    _, da, db = cg.adapter_linear_grad(X, W, A, B, DY, offsets, order, dx=False)
    want = ref.adapter_grad(np.where(ids[:, None] < 0, 0, x), w, a, b,
                            np.where(ids[:, None] < 0, 0, dy), one, ids, dtype)
    check(da, want[1], "da")
    check(db, want[2], "db")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_adapter_empty(cg, dtype):
    import torch

    offsets, order = cg.group_rows(torch.zeros(0, dtype=torch.int32, device="cuda"), 3)
    w, a, b = (dev(np.ones(s), dtype) for s in ((5, 7), (3, 5, 2), (3, 2, 7)))
    x, dy = w.new_empty(0, 5), w.new_empty(0, 7)
    assert cg.adapter_linear(x, w, a, b, offsets, order).shape == (0, 7)
    nan = lambda t: torch.full_like(t, float("nan"))
    _, da, db = cg.adapter_linear_grad(x, w, a, b, dy, offsets, order, da=nan(a), db=nan(b))
    assert (da == 0).all() and (db == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_adapter_gradient_against_differences(cg, dtype):
    """Linear in each of x, a and b alone: <dy, y(a + e) - y(a)> = <da, e>, and so on."""
    rng = np.random.default_rng(8)
    n, G, n_in, n_out, r = 150, 3, 40, 48, 8
    x, w, a, b, dy, scale = _adapters(rng, n, G, n_in, n_out, r, dtype)
    ids = draw_ids(rng, n, G, "holes")
    offsets, order = cg.group_rows(dev(ids), G)
    S = dev(scale)

    def run(x, a, b):
        y = cg.adapter_linear(*(dev(t, dtype) for t in (x, w, a, b)), offsets, order, scale=S)
        return host(y), ref.adapter(x, w, a, b, scale, ids, dtype)[1]

    grads = cg.adapter_linear_grad(*(dev(t, dtype) for t in (x, w, a, b, dy)), offsets, order,
                                   scale=S)
    bounds = [v[1] for v in ref.adapter_grad(x, w, a, b, dy, scale, ids, dtype)]
    y, yb = run(x, a, b)
    base = [x, a, b]
    for i in range(3):
        moved = list(base)
        moved[i] = rounded(base[i] + rng.standard_normal(base[i].shape), dtype)
        y2, yb2 = run(*moved)
        step = moved[i] - base[i]
        lhs, rhs = (dy * (y2 - y)).sum(), (host(grads[i]) * step).sum()
        assert abs(lhs - rhs) <= (np.abs(dy) * (yb + yb2)).sum() + (bounds[i] * np.abs(step)).sum()


# ---------------------------------------------------------------- how calls behave

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_bits_every_time_and_on_another_stream(cg, dtype):
    import torch

    rng = np.random.default_rng(9)
    n, G, n_in, n_out, r = 9000, 3, 64, 200, 16
    x, w, a, b, dy, scale = _adapters(rng, n, G, n_in, n_out, r, dtype)
    ids = draw_ids(rng, n, G, "holes")
    X, W, A, B, DY = (dev(t, dtype) for t in (x, w, a, b, dy))
    WG = W[None].repeat(G, 1, 1).contiguous()
    S, I = dev(scale), dev(ids)

    def everything(stream=None):
        offsets, order = cg.group_rows(I, G, stream=stream)
        out = [offsets, order, cg.grouped_linear(X, WG, offsets, order, stream=stream)]
        out += cg.grouped_linear_grad(X, WG, DY, offsets, order, stream=stream)
        out.append(cg.adapter_linear(X, W, A, B, offsets, order, scale=S, stream=stream))
        out += cg.adapter_linear_grad(X, W, A, B, DY, offsets, order, scale=S, stream=stream)
        return out

    first = everything()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    second, third = everything(), everything(side)
    torch.cuda.synchronize()
    for p, q, t in zip(first, second, third):
        assert torch.equal(p, q) and torch.equal(p, t)


def test_captured_graph_replays(cg):
    """Order, product and gradients captured once and replayed on changed inputs."""
    import torch

    rng = np.random.default_rng(10)
    n, G, n_in, n_out = 6000, 5, 64, 96
    x, w, dy = _linear(rng, n, G, n_in, n_out, "bf16")
    X, W, DY = (dev(t, "bf16") for t in (x, w, dy))
    I = dev(draw_ids(rng, n, G, "holes"))

    def call():
        offsets, order = cg.group_rows(I, G)
        return (cg.grouped_linear(X, W, offsets, order),
                *cg.grouped_linear_grad(X, W, DY, offsets, order))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for k in range(4):
        I.copy_(dev(draw_ids(rng, n, G, "holes")))
        X.copy_(dev(rng.standard_normal((n, n_in)), "bf16"))
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(out, call()):
            assert torch.equal(got, want), k
        torch.cuda.synchronize()


def test_bad_offsets_and_order_stay_in_bounds(cg):
    """Entries outside the documented range are clamped or skipped, by the kernels' own checks."""
    import torch

    n, G = 100, 3
    x, w = torch.ones(n, 16, device="cuda"), torch.ones(G, 16, 24, device="cuda")
    offsets = torch.tensor([0, 40, 2 ** 31 - 1, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    order = torch.arange(n, dtype=torch.int32, device="cuda")
    order[7], order[60] = -5, 2 ** 30
    y = torch.full((n, 24), -1.0, device="cuda")
    cg.grouped_linear(x, w, offsets, order, y=y)
    keep = np.setdiff1d(np.arange(n), [7, 60])
    assert (y[keep] == 16).all() and (y[[7, 60]] == -1).all()
    dx, dw = cg.grouped_linear_grad(x, w, torch.ones_like(y), offsets, order)
    assert (dw[0] == 39).all() and (dw[1] == 59).all() and (dw[2] == 0).all()


# ---------------------------------------------------------------- lines, and rows of other adapters

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n_out,pad,start", [(96, 0, 0), (128, 0, 0), (128, 4, 0), (128, 64, 0), (128, 64, 32),
                                             (160, 0, 0), (164, 28, 0), (192, 0, 64), (196, 0, 4), (70, 2, 2)])
def test_wide_outputs_on_lines_and_apart(cg, dtype, n_out, pad, start):
    """Output rows that begin on lines and apart from them, in a buffer whose other values stay."""
    import torch

    rng = np.random.default_rng([n_out, pad, start])
    n, G, n_in = 700, 3, 40
    x, w, dy = _linear(rng, n, G, n_in, n_out, dtype)
    ids = draw_ids(rng, n, G, "holes")
    offsets, order = cg.group_rows(dev(ids), G)
    X, W = dev(x, dtype), dev(w, dtype)
    stride = n_out + pad
    buf = torch.full((start + n * stride + 64,), 7.0, dtype=X.dtype, device="cuda")
    y = buf[start:start + n * stride].view(n, stride)[:, :n_out]
    cg.grouped_linear(X, W, offsets, order, y=y)
    check(y, ref.grouped(x, w, ids, dtype), "y")
    assert (buf[:start] == 7).all() and (buf[start + n * stride:] == 7).all()
    assert (buf[start:start + n * stride].view(n, stride)[:, n_out:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("n,G,n_in,n_out,r", [
    (600, 40, 64, 72, 8), (3000, 300, 64, 200, 8), (3000, 300, 33, 131, 20),   # tiles of many adapters
    (600, 40, 64, 48, 8), (500, 40, 200, 130, 8), (300, 40, 200, 130, 64), (300, 40, 200, 130, 3),
    (50, 9, 896, 40, 16), (1500, 3, 64, 200, 16), (1500, 3, 64, 200, 40)])
def test_adapter_not_finite_stays_with_its_rows(cg, dtype, value, n, G, n_in, n_out, r):
    """One adapter's second (then first) matrix has such a value: y and dx of all other rows, of other
    adapters and of none, are what they are without it."""
    rng = np.random.default_rng([n, n_in, r])
    x, w, a, b, dy, scale = _adapters(rng, n, G, n_in, n_out, r, dtype)
    ids = draw_ids(rng, n, G, "even")
    ids[rng.random(n) < 0.1] = -1
    bad = G // 2
    others = ids != bad
    assert others.any() and not others.all()
    offsets, order = cg.group_rows(dev(ids), G)
    X, W, DY, S = dev(x, dtype), dev(w, dtype), dev(dy, dtype), dev(scale)
    y, y_bound = ref.adapter(x, w, a, b, scale, ids, dtype)
    (dx, dx_bound), _, _ = ref.adapter_grad(x, w, a, b, dy, scale, ids, dtype)
    for spoiled in ("b", "a"):
        A, B = dev(a, dtype), dev(b, dtype)
        if spoiled == "b":
            B[bad, r // 2, n_out // 3] = value
        else:
            A[bad, n_in // 3, r // 2] = value
        got = host(cg.adapter_linear(X, W, A, B, offsets, order, scale=S))
        assert np.isfinite(got[others]).all(), spoiled
        assert np.all(np.abs(got - y)[others] <= y_bound[others]), spoiled
        col = slice(n_out // 3, n_out // 3 + 1) if spoiled == "b" else slice(None)
        assert not np.isfinite(got[~others][:, col]).any(), spoiled
        got = host(cg.adapter_linear_grad(X, W, A, B, DY, offsets, order, scale=S, da=False, db=False)[0])
        assert np.isfinite(got[others]).all(), spoiled
        assert np.all(np.abs(got - dx)[others] <= dx_bound[others]), spoiled
        col = slice(None) if spoiled == "b" else slice(n_in // 3, n_in // 3 + 1)
        assert not np.isfinite(got[~others][:, col]).any(), spoiled
