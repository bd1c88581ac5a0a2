"""Routing, layers, joining and the gradients' norm against the 64-bit reference, at the sizes, masks, strides and
types where they can go wrong."""
from __future__ import annotations

import math

import numpy as np
import pytest

from tests import layers_ref as ref
from tests import rows_ref
from tests.test_gpu_rows import cg, check, dev, draw_ids, host, rounded, strided  # noqa: F401

pytestmark = pytest.mark.gpu
F32 = "f32"


# ---------------------------------------------------------------- routing

def draw_logits(rng, n, E, masked, dtype):
    a = 1.2 * rng.standard_normal((n, E)) + 0.5 * rng.standard_normal(E)
    a = rounded(a, dtype)
    if masked:
        a[rng.random((n, E)) < np.where(rng.random((n, 1)) < 0.05, 1.0, masked)] = -np.inf
    return a


# rows, experts, top_k, blocks, blocks kept
ROUTES = [(1, 1, 1, 1, 1), (1, 8, 2, 1, 1), (64, 8, 2, 1, 1), (3, 8, 8, 1, 1), (37, 7, 3, 1, 1), (200, 9, 4, 3, 2),
          (1000, 32, 4, 4, 4), (513, 33, 5, 1, 1), (300, 64, 4, 8, 4), (129, 128, 8, 1, 1), (77, 129, 16, 1, 1),
          (50, 130, 1, 13, 3), (65, 512, 16, 8, 1), (40, 520, 64, 1, 1), (9, 4096, 64, 64, 7), (5, 4001, 3, 1, 1),
          (260, 16, 2, 16, 5), (31, 64, 64, 1, 1)]


@pytest.mark.parametrize("n,E,k,blocks,keep", ROUTES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias,renorm,masked,pad", [(False, True, 0.0, 0), (True, True, 0.3, 3), (True, False, 0.0, 1),
                                                    (False, False, 0.8, 0)])
def test_route(cg, n, E, k, blocks, keep, dtype, score, bias, renorm, masked, pad):
    rng = np.random.default_rng(n + 7 * E + k)
    logits = draw_logits(rng, n, E, masked, dtype)
    b = rounded(0.05 * rng.standard_normal(E), F32) if bias else None
    ids, w = cg.route_rows(strided(dev(logits, dtype), pad), k, bias=None if b is None else dev(b), score=score,
                           n_blocks=blocks, keep_blocks=keep, renormalize=renorm, scale=1.5)
    want, weights = ref.route(logits, k, b, score, blocks, keep, renorm, 1.5)
    assert np.array_equal(ids.cpu().numpy(), want)
    check(w, weights, "weights")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_ties_go_to_the_lowest(cg, dtype, score):
    """Few different logits, with a bias of zeros and without one, in blocks and not."""
    rng = np.random.default_rng(3)
    logits = rng.integers(-1, 2, (500, 48)).astype(float)
    for b in (None, np.zeros(48)):
        for blocks, keep in ((1, 1), (6, 2)):
            ids, w = cg.route_rows(dev(logits, dtype), 7, bias=None if b is None else dev(b), score=score, n_blocks=blocks,
                                   keep_blocks=keep)
            want, weights = ref.route(logits, 7, b, score, blocks, keep, True, 1.0)
            assert np.array_equal(ids.cpu().numpy(), want), (b is None, blocks)
            check(w, weights, "weights")


def test_route_near_ties_are_told_apart(cg):
    """Keys that differ by far less than fp32's rounding of them."""
    rng = np.random.default_rng(4)
    logits = rounded(1.0 + 1e-6 * rng.standard_normal((3000, 40)), F32)
    b = rounded(0.25 + 1e-7 * rng.standard_normal(40), F32)
    for score in ("softmax", "sigmoid"):
        for blocks, keep in ((1, 1), (5, 2)):
            ids, _ = cg.route_rows(dev(logits), 6, bias=dev(b), score=score, n_blocks=blocks, keep_blocks=keep)
            assert np.array_equal(ids.cpu().numpy(), ref.route(logits, 6, b, score, blocks, keep, True, 1.0)[0])


@pytest.mark.parametrize("size", [8, 5])
def test_route_blocks_whose_keys_cancel(cg, size):
    """Biases of both signs, far larger than the scores: the sums of a block's keys keep what the scores say."""
    rng = np.random.default_rng(5)
    for by in (1.0, 30.0, 1e4):
        b = rounded(by * (1 + 1e-6 * rng.standard_normal(6 * size)) * np.where(np.arange(6 * size) % size == 0, 1, -1), F32)
        logits = rounded(0.01 * rng.standard_normal((2000, 6 * size)), F32)
        for score in ("softmax", "sigmoid"):
            ids, _ = cg.route_rows(dev(logits), 4, bias=dev(b), score=score, n_blocks=6, keep_blocks=2)
            assert np.array_equal(ids.cpu().numpy(), ref.route(logits, 4, b, score, 6, 2, True, 1.0)[0]), (by, score)


def test_route_values_that_are_not_finite(cg):
    import torch

    inf, nan = math.inf, math.nan
    rows = np.array([[0, 1, 2, 3, -1, -2, .5, .25], [nan, 1, 2, 3, -1, -2, .5, .25], [inf, 1, 2, 3, -1, -2, .5, .25],
                     [-inf] * 8, [nan] * 8, [-inf, 5, -inf, -inf, -inf, -inf, -inf, 4], [3e38, -3e38, 0, 0, 0, 0, 0, 0]])
    for kw in (dict(), dict(bias=dev(np.zeros(8))), dict(n_blocks=4, keep_blocks=3)):
        for score in ("softmax", "sigmoid"):
            ids, w = cg.route_rows(dev(rows), 4, score=score, renormalize=False, **kw)
            i, w = ids.cpu().numpy(), host(w)
            assert ((i >= -1) & (i < 8)).all()
            assert all(len(set(r[r >= 0])) == (r >= 0).sum() for r in i)          # no expert twice
            assert (i[3] == -1).all() and (w[3] == 0).all() and (i[4] == -1).all()
            assert i[5, 0] == 1 and i[5, 1] == 7 and (i[5, 2:] == -1).all() and (w[5, 2:] == 0).all()
            assert i[0, 0] == 3 and i[6, 0] == 0 and np.isfinite(w[[0, 3, 5, 6]]).all()
            assert 0 not in i[1]                                                  # NaN is not available
            if score == "softmax":
                assert np.isnan(w[[1, 2, 4]]).all()
            else:
                assert i[2, 0] == 0 and w[2, 0] == 1
    # a bias that shuts an expert out, or wins it every row
    b = np.zeros(8)
    b[2], b[5], b[6] = -inf, inf, nan
    ids, _ = cg.route_rows(dev(np.zeros((3, 8))), 6, bias=dev(b))
    assert torch.equal(ids.cpu(), torch.tensor([[5, 0, 1, 3, 4, 7]] * 3, dtype=torch.int32))
    # scores that leave fp32's range keep their shares
    for score in ("softmax", "sigmoid"):
        far = np.full((1, 8), -200.0)
        far[0, 1], far[0, 5] = -199.0, -198.0
        if score == "softmax":
            far[0, 0] = 300.0
        ids, w = cg.route_rows(dev(far), 2, bias=dev(np.array([-9., 1, 0, 0, 0, 2, 0, 0])), score=score)
        assert ids.tolist() == [[5, 1]]
        assert np.abs(host(w) - np.array([[1, math.exp(-1)]]) / (1 + math.exp(-1))).max() < 200 * 8 * ref.U


@pytest.mark.parametrize("n,E,k,blocks,keep", ROUTES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm,masked,pad", [(False, 0.0, 0), (True, 0.0, 3), (False, 0.7, 1), (True, 0.7, 0)])
def test_route_grad(cg, n, E, k, blocks, keep, dtype, score, renorm, masked, pad):
    rng = np.random.default_rng(n + 5 * E + k)
    logits = draw_logits(rng, n, E, masked, dtype)
    ids, _ = ref.route(logits + 0.3 * rng.standard_normal((n, E)), k, None, score, 1, 1, renorm, 1.0)
    u = rounded(rng.standard_normal((n, k)), F32)
    import torch

    out = strided(torch.empty(n, E, dtype=dev(logits, dtype).dtype, device="cuda"), pad)
    got = cg.route_rows_grad(strided(dev(logits, dtype), pad), dev(ids), dev(u), score=score, renormalize=renorm, scale=1.5,
                             dlogits=out if pad else None)
    check(got, ref.route_grad(logits, ids, u, score, renorm, 1.5, dtype), "dlogits")


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_route_grad_ids_given(cg, score, renorm):
    """Ids out of range have no part, and one that is there twice counts twice."""
    rng = np.random.default_rng(6)
    logits, u = rounded(rng.standard_normal((20, 24)), F32), rounded(rng.standard_normal((20, 5)), F32)
    ids = rng.integers(-3, 30, (20, 5)).astype(np.int32)
    ids[:, 4] = ids[:, 1]
    got = cg.route_rows_grad(dev(logits), dev(ids), dev(u), score=score, renormalize=renorm)
    check(got, ref.route_grad(logits, ids, u, score, renorm, 1.0, F32), "dlogits")


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_route_grad_against_differences(cg, score, renorm):
    """A loss of the weights moved both ways along each logit: h^2 / 6 of its third derivative (below 2 of it, as the
    scores' are), and fp32's rounding of the weights over h, are what they may differ by."""
    import torch

    h, n, E, k = 2.0 ** -7, 6, 8, 3
    rng = np.random.default_rng(7)
    logits = dev(np.round(rng.permuted(np.tile(np.arange(E), (n, 1)), axis=1) * 0.5, 2))   # choices stay under h
    u = dev(rounded(rng.standard_normal((n, k)), F32))
    kw = dict(score=score, renormalize=renorm)
    ids, _ = cg.route_rows(logits, k, **kw)
    got = host(cg.route_rows_grad(logits, ids, u, **kw))
    for e in range(E):
        step = torch.zeros_like(logits)
        step[:, e] = h
        up, down = (cg.route_rows(logits + s, k, **kw) for s in (step, -step))
        assert torch.equal(up[0], ids) and torch.equal(down[0], ids)
        d = ((up[1] - down[1]).double() * u).sum(1).cpu().numpy() / (2 * h)
        size = host(u.abs()).sum(1)
        assert np.all(np.abs(d - got[:, e]) <= size * (h * h / 3 + 40 * ref.U / h))


# ---------------------------------------------------------------- layers

# rows of x, rows that share one, groups, widths
LAYERS = [(1, 1, 1, 1, 1), (1, 1, 3, 64, 64), (2, 1, 5, 7, 3), (64, 1, 5, 64, 64), (65, 1, 2, 8, 129), (127, 1, 1, 33, 128),
          (129, 1, 3, 128, 130), (300, 1, 7, 37, 129), (1000, 1, 400, 24, 40), (257, 1, 2, 896, 72), (2050, 1, 5, 16, 448),
          (515, 1, 2, 1, 300), (515, 1, 2, 300, 1), (90, 1, 80, 200, 130), (1, 8, 8, 64, 64), (33, 3, 5, 31, 67),
          (500, 4, 32, 128, 448), (700, 2, 3, 64, 64), (129, 64, 40, 9, 20), (600, 2, 4, 8, 64), (400, 4, 1000, 16, 24),
          (3000, 1, 2, 64, 64), (2500, 2, 6, 40, 56), (1000, 4, 5, 128, 448), (900, 1, 3, 100, 130), (700, 2, 2, 128, 250),
          (3000, 1, 4, 40, 128), (1200, 1, 3, 33, 447), (800, 1, 2, 128, 100), (600, 1, 2, 4, 5), (600, 1, 2, 129, 90),
          (70, 1, 3, 1344, 33), (31, 2, 40, 647, 8), (200, 3, 2, 8, 1345), (6000, 1, 3, 450, 96)]
ACTS = ["silu", "gelu", "relu", "none"]


def draw_layer(rng, t, per, G, K, N, kind, dtype):
    x = rounded(rng.standard_normal((t, K)), dtype)
    w = rounded(1.5 * K ** -0.5 * rng.standard_normal((G, K, N)), dtype)
    b = rounded(0.3 * rng.standard_normal((G, N)), dtype)
    return x, w, b, draw_ids(rng, t * per, G, kind)


def named(act):
    return None if act == "none" else act


@pytest.mark.parametrize("t,per,G,K,N", LAYERS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act,bias,residual,keep,pad,kind", [
    ("silu", True, False, True, 0, "even"), ("gelu", True, True, False, 3, "holes"), ("relu", False, True, True, 1, "holes"),
    ("none", False, False, False, 0, "one"), ("silu", False, True, True, 8, "none"), ("gelu", True, False, True, 0, "holes")])
def test_layer(cg, t, per, G, K, N, dtype, act, bias, residual, keep, pad, kind):
    import torch

    rng = np.random.default_rng(t + 3 * G + N)
    x, w, b, ids = draw_layer(rng, t, per, G, K, N, kind, dtype)
    r = rounded(rng.standard_normal((t * per, N)), dtype) if residual else None
    o = cg.group_rows(dev(ids), G)
    xd = dev(x, dtype)
    like = lambda more=0: strided(torch.zeros(t * per, N, dtype=xd.dtype, device="cuda"), pad + more) if pad else None
    got = cg.grouped_layer(strided(xd, pad), dev(w, dtype), *o, bias=dev(b, dtype) if bias else None, activation=named(act),
                           residual=None if r is None else strided(dev(r, dtype), pad), per_row=per, y=like(),
                           z=like(int(pad == 1 and t % 2)) if keep else False)   # of y's stride, and of another
    want = ref.layer(x, w, b if bias else None, r, ids, act, per, dtype)
    check(got[0] if keep else got, want[0], "y")
    if keep:
        check(got[1], want[1], "z")
    if pad:                                                     # what lies between the rows is left as it was
        y = got[0] if keep else got
        assert torch.isnan(y._base[:, N:]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_is_the_product_without_extras(cg, dtype):
    """No bias, activation or residual, rows in order: grouped_linear's bits."""
    import torch

    rng = np.random.default_rng(9)
    for t, G, K, N in ((300, 7, 37, 129), (1000, 3, 300, 200), (65, 2, 8, 40)):
        x, w, _, ids = draw_layer(rng, t, 1, G, K, N, "holes", dtype)
        o = cg.group_rows(dev(ids), G)
        value, bound = rows_ref.grouped(x, w, ids, dtype)
        check(cg.grouped_layer(dev(x, dtype), dev(w, dtype), *o), (value, bound), "y")
        sorted_x = dev(x, dtype)[o[1].long()].contiguous()
        y = cg.grouped_layer(sorted_x, dev(w, dtype), o[0])      # no order: rows sorted already
        assert torch.equal(y, cg.grouped_layer(dev(x, dtype), dev(w, dtype), *o)[o[1].long()])


@pytest.mark.parametrize("t,per,G,K,N", LAYERS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act,pad,kind", [("silu", 0, "even"), ("gelu", 3, "holes"), ("relu", 8, "one"), ("none", 1, "holes"),
                                          ("silu", 0, "none")])
def test_layer_grad(cg, t, per, G, K, N, dtype, act, pad, kind):
    import torch

    rng = np.random.default_rng(t + 3 * G + N)
    x, w, b, ids = draw_layer(rng, t, per, G, K, N, kind, dtype)
    z, dy = (rounded(rng.standard_normal((t * per, N)), dtype) for _ in range(2))
    o = cg.group_rows(dev(ids), G)
    a = (strided(dev(x, dtype), pad), dev(w, dtype), strided(dev(dy, dtype), pad), *o)
    kw = dict(z=None if act == "none" else strided(dev(z, dtype), pad), activation=named(act), per_row=per)
    dx = strided(torch.zeros(t, K, dtype=a[0].dtype, device="cuda"), pad) if pad else None
    got = cg.grouped_layer_grad(*a, dx=dx, **kw)
    want = ref.layer_grad(x, w, z, dy, ids, act, per, dtype)
    for g, v, name in zip(got, want, ("dx", "dw", "dbias")):
        check(g, v, name)
    if pad:
        assert torch.isnan(got[0]._base[:, K:]).all()
    # each alone
    for skip in range(3):
        one = cg.grouped_layer_grad(*a, **{n: None if i == skip else False for i, n in enumerate(("dx", "dw", "dbias"))}, **kw)
        assert [i for i in range(3) if one[i] is not None] == [skip]
        check(one[skip], want[skip], skip)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_layer_grad_of_long_groups(cg, dtype, act):
    """Groups of several chunks, whose sums are joined; odd widths, so that a cell's quad holds both outputs."""
    rng = np.random.default_rng(11)
    for t, per, G, K, N in ((40000, 1, 2, 15, 17), (9000, 4, 3, 33, 64), (50000, 1, 1, 64, 64), (30000, 1, 3, 16, 130),
                           (9000, 2, 3, 128, 448), (20000, 1, 2, 127, 255), (9000, 1, 2, 130, 64)):
        x, w, b, ids = draw_layer(rng, t, per, G, K, N, "holes", dtype)
        z, dy = (rounded(rng.standard_normal((t * per, N)), dtype) for _ in range(2))
        o = cg.group_rows(dev(ids), G)
        got = cg.grouped_layer_grad(dev(x, dtype), dev(w, dtype), dev(dy, dtype), *o, z=dev(z, dtype), activation=act, per_row=per)
        again = cg.grouped_layer_grad(dev(x, dtype), dev(w, dtype), dev(dy, dtype), *o, z=dev(z, dtype), activation=act,
                                      per_row=per)
        for g, h, v, name in zip(got, again, ref.layer_grad(x, w, z, dy, ids, act, per, dtype), ("dx", "dw", "dbias")):
            check(g, v, name)
            assert (g == h).all(), name                          # the same bits again
        only = cg.grouped_layer_grad(dev(x, dtype), dev(w, dtype), dev(dy, dtype), *o, z=dev(z, dtype), activation=act,
                                     per_row=per, dx=False, dw=False)[2]
        check(only, ref.layer_grad(x, w, z, dy, ids, act, per, dtype)[2], "dbias alone")


@pytest.mark.parametrize("t,per,G,K,N,act,kind,pad", [
    (66001, 1, 3, 100, 72, "silu", "holes", 3), (16700, 4, 33, 128, 168, "gelu", "holes", 8), (70000, 1, 7, 33, 200, "relu", "one", 1),
    (33000, 2, 2, 16, 136, "none", "holes", 0), (65600, 1, 1, 90, 8, "silu", "even", 0), (66000, 1, 4, 128, 448, "silu", "even", 0),
    (65537, 1, 128, 65, 16, "gelu", "even", 0), (70000, 1, 3, 40, 24, "silu", "none", 0)])
def test_layer_grad_of_many_rows(cg, t, per, G, K, N, act, kind, pad):
    """Rows in order and not, and rows that the order does not hold."""
    import torch

    rng = np.random.default_rng(17)
    x, w, b, ids = draw_layer(rng, t, per, G, K, N, kind, "bf16")
    z, dy = (rounded(rng.standard_normal((t * per, N)), "bf16") for _ in range(2))
    kw = dict(z=None if act == "none" else strided(dev(z, "bf16"), pad), activation=named(act), per_row=per)
    a = (strided(dev(x, "bf16"), pad), dev(w, "bf16"), strided(dev(dy, "bf16"), pad))
    o = cg.group_rows(dev(ids), G)
    want = ref.layer_grad(x, w, z, dy, ids, act, per, "bf16")
    got = cg.grouped_layer_grad(*a, *o, **kw)
    again = cg.grouped_layer_grad(*a, *o, **kw)
    for g, h, v, name in zip(got, again, want, ("dx", "dw", "dbias")):
        check(g, v, name)
        assert torch.equal(g, h), name
    check(cg.grouped_layer_grad(*a, *o, dw=False, dbias=False, **kw)[0], want[0], "dx alone")
    if per > 1:
        return
    by = o[1].long()
    sorted_kw = {**kw, "z": None if act == "none" else kw["z"][by]}
    for g, h, name in zip(cg.grouped_layer_grad(a[0][by], a[1], a[2][by], o[0], **sorted_kw), got, ("dx", "dw", "dbias")):
        assert torch.equal(g, h[by] if name == "dx" else h), name
    # every 97th position without a row
    order = o[1].clone()
    order[::97] = -1
    gone = torch.zeros(t, dtype=torch.bool, device="cuda")
    gone[o[1][::97].long()] = True
    dx = torch.full((t, K), 7.0, dtype=a[0].dtype, device="cuda")
    got = cg.grouped_layer_grad(*a, o[0], order, dx=dx, **kw)
    assert (dx[gone] == 7).all() and torch.equal(dx[~gone], again[0][~gone])
    rest = ref.layer_grad(x, w, z, dy, np.where(gone.cpu().numpy(), -1, ids), act, per, "bf16")
    for g, v, name in zip(got[1:], rest[1:], ("dw", "dbias")):
        check(g, v, name)


def test_layer_grad_of_no_rows(cg):
    import torch

    o = cg.group_rows(torch.zeros(0, dtype=torch.int32, device="cuda"), 3)
    x, w, dy = torch.zeros(0, 8, device="cuda"), torch.ones(3, 8, 5, device="cuda"), torch.zeros(0, 5, device="cuda")
    dx, dw, db = cg.grouped_layer_grad(x, w, dy, *o, z=dy, activation="silu", per_row=2)
    assert dx.shape == (0, 8) and (dw == 0).all() and (db == 0).all()
    assert cg.grouped_layer(x, w, *o, per_row=2).shape == (0, 5)


@pytest.mark.parametrize("act", ACTS)
def test_layer_grad_against_differences(cg, act):
    """A loss of y moved both ways along each input. y's third derivative along a direction of size d is below
    4 d^3, and fp32 rounds sums of K + 5 terms of magnitude below 20; relu's kink is kept out of reach."""
    import torch

    h, t, per, G, K, N = 2.0 ** -6, 6, 2, 3, 5, 4
    rng = np.random.default_rng(13)
    x, w, b, ids = draw_layer(rng, t, per, G, K, N, "even", F32)
    if act == "relu":
        b = b + np.where(rng.random((G, N)) < 0.5, 40.0, -40.0)
    args = [dev(rounded(a, F32)) for a in (x, w, b)]
    o = cg.group_rows(dev(ids), G)
    dy = dev(rounded(rng.standard_normal((t * per, N)), F32))
    f = lambda: cg.grouped_layer(args[0], args[1], *o, bias=args[2], activation=named(act), per_row=per).double()
    _, z = cg.grouped_layer(args[0], args[1], *o, bias=args[2], activation=named(act), per_row=per, z=None)
    got = cg.grouped_layer_grad(args[0], args[1], dy, *o, z=z, activation=named(act), per_row=per)
    size = host(dy.abs()).sum()
    most = max(1.0, np.abs(x).max(), np.abs(w).max())
    for a, g in zip(args, got):
        flat = a.view(-1)
        for i in range(flat.numel()):
            keep = flat[i].clone()
            flat[i] = keep + h
            up, hi = f(), flat[i].double()
            flat[i] = keep - h
            d = ((up - f()) * dy).sum() / (hi - flat[i].double())
            flat[i] = keep
            bound = size * (4 * h * h * most ** 3 + (K + 5) * 64 * ref.U * most * (40 if act == "relu" else 1) / h)
            assert abs(d.item() - g.view(-1)[i].item()) <= bound


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("N,keep,K", [(72, True, 40), (96, True, 40), (96, False, 40), (73, False, 40), (61, True, 40),
                                      (70, True, 333), (65, False, 256)])
def test_layer_keeps_values_that_are_not_finite_apart(cg, dtype, act, N, keep, K):
    """An infinite or NaN input, weight or residual reaches its own rows' results and no others."""
    import torch

    rng = np.random.default_rng(15)
    t, per, G = 400, 2, 4
    x, w, b, ids = draw_layer(rng, t, per, G, K, N, "even", dtype)
    o = cg.group_rows(dev(ids), G)

    def run(x, w, b):
        layer = lambda **kw: cg.grouped_layer(dev(x, dtype), dev(w, dtype), *o, bias=dev(b, dtype), per_row=per, **kw)
        return layer(activation=named(act), z=None) if keep else (layer(activation=named(act)), layer())
    y0, z0 = run(x, w, b)
    for bad in (math.inf, -math.inf, math.nan):
        x1, w1, b1 = x.copy(), w.copy(), b.copy()
        x1[7, 3] = bad
        w1[2, 5, 11] = bad
        b1[1, 60] = bad
        y, z = run(x1, w1, b1)
        hit = np.zeros((t * per, N), bool)
        hit[7 * per:7 * per + per] = True
        hit[ids == 2, 11] = True
        hit[ids == 1, 60] = True
        same = torch.from_numpy(~hit).cuda()
        assert torch.equal(z[same], z0[same]) and torch.equal(y[same], y0[same])
        assert not torch.isfinite(z[~same]).any()
        with np.errstate(invalid="ignore", over="ignore"):
            (_, _), (zr, _) = ref.layer(x1, w1, b1, None, ids, act, per, dtype)
        h = host(z)
        assert np.array_equal(np.isnan(h), np.isnan(zr)) and np.array_equal(h[np.isinf(zr)], zr[np.isinf(zr)])
        # and the activation is that of z
        zt = z.double()
        f = {"silu": zt * torch.sigmoid(zt), "gelu": zt * 0.5 * torch.special.erfc(-zt / math.sqrt(2)),
             "relu": torch.relu(zt), "none": zt}[act]
        assert torch.equal(torch.isfinite(y), torch.isfinite(f)) and torch.equal(torch.isnan(y), torch.isnan(f))


@pytest.mark.parametrize("act", ["silu", "relu", "none"])
def test_layer_of_large_sums(cg, act):
    """fp32 sums beyond what the parts of the operands hold are formed again, and infinite only where fp32's are."""
    rng = np.random.default_rng(16)
    t, G, K, N = 200, 2, 24, 72
    x, w, b, ids = draw_layer(rng, t, 1, G, K, N, "even", F32)
    x[5] *= 2.0 ** 100
    x[9] *= 2.0 ** -120
    x, o = rounded(x, F32), cg.group_rows(dev(ids), G)
    y, z = cg.grouped_layer(dev(x), dev(w), *o, bias=dev(b), activation=named(act), z=None)
    want = ref.layer(x, w, b, None, ids, act, 1, F32)
    check(z, want[1], "z")
    check(y, want[0], "y")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [72, 56, 300, 500])
def test_layer_grad_keeps_values_that_are_not_finite_apart(cg, dtype, N):
    import torch

    rng = np.random.default_rng(17)
    t, per, G, K = 300, 2, 4, 40
    x, w, b, ids = draw_layer(rng, t, per, G, K, N, "even", dtype)
    z, dy = (rounded(rng.standard_normal((t * per, N)), dtype) for _ in range(2))
    o = cg.group_rows(dev(ids), G)
    run = lambda dy: cg.grouped_layer_grad(dev(x, dtype), dev(w, dtype), dev(dy, dtype), *o, z=dev(z, dtype), activation="silu",
                                           per_row=per)
    base = run(dy)
    w0 = w.copy()
    w[1, 6, 9] = math.inf                                        # a weight: dx of its group's rows, input 6
    own = np.repeat(np.arange(t), per)[ids == 1]
    got = run(dy)
    hit = torch.zeros(t, K, dtype=torch.bool, device="cuda")
    hit[torch.from_numpy(own).cuda(), 6] = True
    assert torch.equal(got[0][~hit], base[0][~hit]) and not torch.isfinite(got[0][hit]).any()
    assert torch.equal(got[1], base[1]) and torch.equal(got[2], base[2])
    sign = np.sign(dy * ref.slope(z, "silu")[0])[:, 9]           # infinite by the sign of dz alone, where no two meet
    for i in own[:20]:
        s = {sign[r] for r in range(i * per, i * per + per) if ids[r] == 1}
        if len(s) == 1:
            assert got[0][i, 6].item() == s.pop() * math.inf
    w = w0
    for bad in (math.inf, math.nan):
        d1 = dy.copy()
        d1[31, 8] = bad
        got = run(d1)
        g = ids[31]
        rows = torch.arange(t, device="cuda") != 31 // per
        others = torch.arange(G, device="cuda") != g
        assert torch.equal(got[0][rows], base[0][rows]) and not torch.isfinite(got[0][31 // per]).any()
        assert torch.equal(got[1][others], base[1][others]) and torch.equal(got[2][others], base[2][others])
        cols = torch.arange(N, device="cuda") != 8
        assert torch.equal(got[1][g][:, cols], base[1][g][:, cols]) and torch.equal(got[2][g][cols], base[2][g][cols])
        assert not torch.isfinite(got[1][g][:, 8]).any() and not torch.isfinite(got[2][g][8])


# ---------------------------------------------------------------- joining

MIXES = [(1, 1, 1), (1, 3, 8), (5, 2, 7), (64, 4, 64), (33, 8, 449), (300, 16, 130), (100, 64, 24), (1000, 2, 16),
         (70, 4, 896), (9, 5, 4099), (2049, 1, 12)]


@pytest.mark.parametrize("n,k,N", MIXES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("weights,residual,pad", [(True, True, 0), (True, False, 3), (False, True, 1), (False, False, 8)])
def test_mix(cg, n, k, N, dtype, weights, residual, pad):
    import torch

    rng = np.random.default_rng(n + N)
    y = rounded(rng.standard_normal((n * k, N)), dtype)
    w = rounded(rng.standard_normal((n, k)), F32) if weights else None
    r = rounded(rng.standard_normal((n, N)), dtype) if residual else None
    yd = dev(y, dtype)
    out = strided(torch.zeros(n, N, dtype=yd.dtype, device="cuda"), pad) if pad else None
    got = cg.mix_rows(strided(yd, pad), k, weights=None if w is None else dev(w),
                      residual=None if r is None else strided(dev(r, dtype), pad), out=out)
    check(got, ref.mix(y, w, r, k, dtype), "out")
    if pad:
        assert torch.isnan(got._base[:, N:]).all()


@pytest.mark.parametrize("n,k,N", MIXES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("weights,pad", [(True, 0), (True, 3), (False, 8)])
def test_mix_grad(cg, n, k, N, dtype, weights, pad):
    import torch

    rng = np.random.default_rng(n + N)
    y, d = rounded(rng.standard_normal((n * k, N)), dtype), rounded(rng.standard_normal((n, N)), dtype)
    w = rounded(rng.standard_normal((n, k)), F32) if weights else None
    wd, dd, yd = None if w is None else dev(w), strided(dev(d, dtype), pad), strided(dev(y, dtype), pad)
    out = strided(torch.zeros(n * k, N, dtype=dd.dtype, device="cuda"), pad) if pad else None
    got = cg.mix_rows_grad(dd, k, weights=wd, y=yd, dy=out)
    want = ref.mix_grad(d, w, y, k, dtype)
    check(got[0], want[0], "dy")
    check(got[1], want[1], "dweights")
    if pad:
        assert torch.isnan(got[0]._base[:, N:]).all()
    alone = cg.mix_rows_grad(dd, k, weights=wd, dweights=False)
    assert alone[1] is None and torch.equal(alone[0], got[0])
    alone = cg.mix_rows_grad(dd, k, weights=wd, y=yd, dy=False)
    assert alone[0] is None and torch.equal(alone[1], got[1])


def test_mix_of_no_rows(cg):
    import torch

    y = torch.zeros(0, 8, device="cuda")
    assert cg.mix_rows(y, 4).shape == (0, 8)
    dy, dw = cg.mix_rows_grad(y, 4, y=y)
    assert dy.shape == (0, 8) and dw.shape == (0, 4)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_past_32_bits(cg, dtype):
    """More than 2^31 values of y: rows at the end, and what a layer reads and writes there."""
    import torch

    n, k, N = 34000, 8, 8192
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    y = torch.zeros(n * k, N, dtype=t, device="cuda")
    w = torch.rand(n, k, device="cuda")
    at = [0, 1, n // 2, n - 2, n - 1]
    for i in at:
        y[i * k:(i + 1) * k] = torch.randn(k, N, device="cuda").to(t)
    out = cg.mix_rows(y, k, weights=w)
    dy, dw = cg.mix_rows_grad(out, k, weights=w, y=y)
    for i in at:
        rows = slice(i * k, (i + 1) * k)
        check(out[i:i + 1], ref.mix(host(y[rows]), host(w[i:i + 1]), None, k, dtype), i)
        want = ref.mix_grad(host(out[i:i + 1]), host(w[i:i + 1]), host(y[rows]), k, dtype)
        check(dy[rows], want[0], i)
        check(dw[i:i + 1], want[1], i)
    del dy, out
    ids = torch.full((n * k,), -1, dtype=torch.int32, device="cuda")
    ids[[0, 5, n * k - 9, n * k - 1]] = torch.tensor([0, 1, 1, 0], dtype=torch.int32, device="cuda")
    o = cg.group_rows(ids, 2)
    x, wt = torch.randn(n, 16, device="cuda").to(t), torch.randn(2, 16, N, device="cuda").to(t)
    some = [0, 5, n * k - 9, n * k - 1]
    (v, b), _ = ref.layer(host(x[[i // k for i in some]]), host(wt), None, None, ids[some].cpu().numpy(), "silu", 1, dtype)
    del y
    y = cg.grouped_layer(x, wt, *o, activation="silu", per_row=k)
    check(y[some], (v, b), "layer")
    dx, dw, db = cg.grouped_layer_grad(x, wt, y, *o, z=y, activation="silu", per_row=k)
    keep = host(y[some])
    full = ref.layer_grad(host(x[[i // k for i in some]]), host(wt), keep, keep, ids[some].cpu().numpy(), "silu", 1, dtype)
    check(dw, full[1], "dw")
    check(db, full[2], "dbias")


# ---------------------------------------------------------------- the gradients' norm

def _adam(cg, grads, dtype):
    import torch

    like = lambda: [torch.zeros(g.shape, device="cuda") for g in grads]
    return cg.AdamWTensors(like(), [dev(g, dtype) for g in grads], like(), like())


@pytest.mark.parametrize("sizes", [(1,), (0, 3), (0,), (256, 4096, 4097), (5,) * 31, (5,) * 32, (5,) * 33, (5,) * 300,
                                   (1000003, 7, 0, 64), (2048 * 4096,), (2049 * 4096 + 1, 3)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_grad_norm(cg, sizes, dtype):
    rng = np.random.default_rng(len(sizes))
    grads = [rounded(rng.standard_normal(s) * 10.0 ** -(i % 4), dtype) for i, s in enumerate(sizes)]
    a = _adam(cg, grads, dtype)
    want = math.sqrt(math.fsum(float((g ** 2).sum()) for g in grads))       # sums of up to 2^23 in 64 bits: 2^-30 at most
    for gs in (None, 0.5, -2.0):
        g = None if gs is None else dev(np.array([gs]))
        f = 1.0 if gs is None else gs
        for most in (0.5 * abs(f) * want or 1.0, 2 * abs(f) * want or 1.0):
            norm, scale = (t.item() for t in cg.adamw_grad_norm(a, most, grad_scale=g))
            assert abs(norm - abs(f) * want) <= (ref.U + 1e-12) * norm + 1e-45
            clip = f * min(1.0, most / (abs(f) * want)) if want else f
            assert abs(scale - clip) <= (ref.U + 1e-12) * abs(clip)
    both = cg.adamw_grad_norm(a, 1.0)
    assert cg.adamw_grad_norm(a, 1.0, norm=False)[0] is None and cg.adamw_grad_norm(a, 1.0, scale=False)[1] is None
    again = cg.adamw_grad_norm(a, 1.0)
    assert all((x == y).all() for x, y in zip(both, again))


def test_grad_norm_range_and_order(cg):
    """Gradients whose squares leave fp32's range; NaN and infinities; read where they lie; grad_scale in place."""
    import torch

    for size in (1e30, 1e-30):
        a = _adam(cg, [np.full(5000, size)], F32)
        norm, _ = cg.adamw_grad_norm(a, 1.0)
        v = float(np.float32(size)) * math.sqrt(5000)
        assert abs(norm.item() - v) <= ref.U * v
    a = _adam(cg, [np.ones(10), np.ones(6)], F32)
    g = a._keep[1][1]
    for bad, norm, scale in ((math.nan, math.nan, 1.0), (math.inf, math.inf, 0.0)):
        g[2] = bad
        got = [t.item() for t in cg.adamw_grad_norm(a, 2.0)]
        assert got[1] == scale and (got[0] == norm or (math.isnan(got[0]) and math.isnan(norm)))
    g[2] = 1.0
    s = torch.full((1,), 0.5, device="cuda")
    norm, out = cg.adamw_grad_norm(a, 1.0, grad_scale=s, scale=s)
    assert norm.item() == 2.0 and out is s and s.item() == 0.25


def test_grad_norm_refusals(cg):
    import torch

    a = _adam(cg, [np.ones(10)], F32)
    for most in (0.0, -1.0, math.nan):
        with pytest.raises(cg.CgtpError):
            cg.adamw_grad_norm(a, most)
    with pytest.raises(cg.CgtpError):
        cg.adamw_grad_norm(a, 1.0, norm=False, scale=False)
    with pytest.raises(cg.CgtpError):
        cg.adamw_grad_norm(_adam(cg, [np.ones(10), np.ones(10)], F32), 1.0, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        cg.adamw_grad_norm(a, 1.0, norm=torch.zeros(2, device="cuda"))
    with pytest.raises(ValueError):
        cg.adamw_grad_norm(a, 1.0, grad_scale=torch.zeros(1))
