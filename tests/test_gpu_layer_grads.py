"""What the gradients of layers owe beside their values: that an output does not depend on the others that are asked for,
and how many bits they hold between the two factors of dz and its products."""
from __future__ import annotations

import itertools

import numpy as np
import pytest

from tests import layers_ref as ref
from tests.test_gpu_layers import LAYERS, draw_layer, named
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


def grad_of_parts(x, w, z, dy, ids, name, per):
    """(dx, dw, dbias), each (value, bound), of bf16 layers whose dz is held in two bf16 parts between its forming and the
    products: dz in [1, 2) leaves at most 2^-8 to the second part, which rounds that by 2^-17. Sums have two terms for each
    product; dbias adds dz itself or its parts. Without an activation dz is dy."""
    G, K, N = w.shape
    s, sb = ref.slope(z, name, "bf16")
    dz = dy * s
    formed = np.abs(dy) * sb + ref.U * np.abs(dz)
    held = formed + (2.0 ** -17 * (np.abs(dz) + formed) if name != "none" else 0.0)
    n, u_sum, half = ids.size, 2.0 ** -23, ref.out("bf16")
    dx, dxb = np.zeros((n, K)), np.zeros((n, K))
    dw, dwb, db, dbb = np.zeros(w.shape), np.zeros(w.shape), np.zeros((G, N)), np.zeros((G, N))
    for g in range(G):
        rows = np.flatnonzero(ids == g)
        d, xs = dz[rows], x[rows // per]
        dx[rows] = d @ w[g].T
        dxb[rows] = (held[rows] + u_sum * (2 * N + 4) * np.abs(d)) @ np.abs(w[g]).T
        dw[g] = xs.T @ d
        dwb[g] = np.abs(xs).T @ (held[rows] + u_sum * (2 * len(rows) + 4) * np.abs(d)) + half * np.abs(dw[g])
        db[g] = d.sum(0)
        dbb[g] = (held[rows] + u_sum * (len(rows) + 4) * np.abs(d)).sum(0) + half * np.abs(db[g])
    of = lambda a: a.reshape(n // per, per, K).sum(1)
    v = of(dx)
    return ((v, of(dxb + u_sum * per * np.abs(dx)) + half * np.abs(v) + ref.TINY), (dw, dwb + ref.TINY), (db, dbb + ref.TINY))


# rows of x, rows that share one, groups, widths: each form of the two products, with whole steps and remainders
HELD = LAYERS + [(20000, 1, 3, 128, 448), (9000, 4, 7, 128, 448), (20000, 1, 3, 448, 128), (6000, 3, 3, 900, 130),
                 (30000, 1, 4, 72, 100), (12000, 2, 5, 300, 333), (40000, 1, 3, 333, 200), (5000, 1, 100, 70, 450),
                 (2000, 1, 900, 100, 70), (300, 2, 300, 200, 90), (30000, 1, 2, 66, 5), (30000, 1, 2, 5, 66)]


@pytest.mark.parametrize("t,per,G,K,N", HELD)
@pytest.mark.parametrize("act,pad,kind", [("silu", 0, "even"), ("gelu", 3, "holes"), ("relu", 8, "holes"), ("none", 1, "even")])
def test_bf16_gradients_hold_dz_in_two_parts(cg, t, per, G, K, N, act, pad, kind):
    import torch

    rng = np.random.default_rng(t + 5 * G + N)
    x, w, ids, z, dy = draw_grad(rng, t, per, G, K, N, kind, "bf16")
    o = cg.group_rows(dev(ids), G)
    a = (strided(dev(x, "bf16"), pad), dev(w, "bf16"), strided(dev(dy, "bf16"), pad), *o)
    kw = dict(z=None if act == "none" else strided(dev(z, "bf16"), pad + pad % 2), activation=named(act), per_row=per)
    dx = strided(torch.zeros(t, K, dtype=torch.bfloat16, device="cuda"), pad) if pad else None
    got = cg.grouped_layer_grad(*a, dx=dx, **kw)
    for g, v, name in zip(got, grad_of_parts(x, w, z, dy, ids, act, per), NAMES):
        check(g, v, name)
    if pad:                                                     # what lies between the rows is left as it was
        assert torch.isnan(got[0]._base[:, K:]).all()
    # dx and dw are those of a call for them alone
    assert torch.equal(cg.grouped_layer_grad(*a, dw=False, dbias=False, **kw)[0], got[0])
    assert torch.equal(cg.grouped_layer_grad(*a, dx=False, dbias=False, **kw)[1], got[1])


@pytest.mark.parametrize("t,per,G,K,N", [(300, 2, 4, 40, 500), (300, 1, 4, 40, 72), (400, 1, 2, 100, 96), (6000, 1, 3, 200, 200),
                                         (600, 3, 3, 150, 130), (900, 1, 2, 300, 8), (500, 1, 400, 90, 70)])
@pytest.mark.parametrize("act", ["silu", "relu"])
def test_bf16_gradients_beside_what_is_not_finite(cg, t, per, G, K, N, act):
    """Infinite weights and rows, and an infinite dy: dx and dw hold the infinities and NaN of the formula, and what they do
    not reach keeps its bits."""
    import torch

    rng = np.random.default_rng(t + N)
    x, w, ids, z, dy = draw_grad(rng, t, per, G, K, N, "even", "bf16")
    o = cg.group_rows(dev(ids), G)
    run = lambda x, w, dy: cg.grouped_layer_grad(dev(x, "bf16"), dev(w, "bf16"), dev(dy, "bf16"), *o, z=dev(z, "bf16"),
                                                 activation=act, per_row=per)
    base = run(x, w, dy)
    x1, w1, dy1 = x.copy(), w.copy(), dy.copy()
    g = ids[5]
    w1[g, 3, 2] = np.inf
    x1[1, 4] = -np.inf
    dy1[7, 1] = np.inf
    z[7, 1] = 1.0                                                # whose slope is no zero
    base, got = run(x, w, dy), run(x1, w1, dy1)
    with np.errstate(invalid="ignore", over="ignore"):
        want = [v for v, _ in grad_of_parts(x1, w1, z, dy1, ids, act, per)]
        plain = [v for v, _ in grad_of_parts(x, w, z, dy, ids, act, per)]
    for h, b, v, p, name in zip(got, base, want, plain, NAMES):
        fine = np.isfinite(v)
        assert np.array_equal(np.isfinite(host(h)), fine), name
        assert np.array_equal(host(h)[np.isinf(v)], v[np.isinf(v)]), name
        same = torch.from_numpy(fine & (v == p)).cuda()
        assert torch.equal(h[same], b[same]), name


@pytest.mark.parametrize("G,K,N", [(512, 8, 60), (376, 8, 72)])
def test_bias_gradient_of_many_small_terms(cg, G, K, N):
    """Groups of 4,096 rows, the first 1 and the others 2^-25, which are lost where they are added to it one by one. Eight
    rows of 32 or 64 are added first, so that a sum takes 128 additions of those, 3 within them and 16 of lanes, each off by
    U of it."""
    import torch

    n = 4096
    dy = torch.full((G * n, N), 2.0 ** -25, device="cuda")
    dy[::n] = 1.0
    x, w = torch.zeros(G * n, K, device="cuda"), torch.zeros(G, K, N, device="cuda")
    offsets = torch.arange(0, G * n + 1, n, dtype=torch.int32, device="cuda")
    got = cg.grouped_layer_grad(x, w, dy, offsets, dx=False)[2].double()
    want = 1 + (n - 1) * 2.0 ** -25
    assert (got - want).abs().max().item() <= (128 + 3 + 16) * ref.U * want


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t,per,G,K,N", [(3000, 4, 3, 64, 64), (3000, 4, 3, 200, 72), (500, 3, 900, 64, 64)])
def test_workspace_without_row_gradients(cg, dtype, t, per, G, K, N):
    """dw and dbias alone take the workspace that the query gives for rows of their own, and no less."""
    import torch

    rng = np.random.default_rng(t)
    x, w, ids, z, dy = draw_grad(rng, t, per, G, K, N, "even", dtype)
    o = cg.group_rows(dev(ids), G)
    run = lambda **kw: cg.grouped_layer_grad(dev(x, dtype), dev(w, dtype), dev(dy, dtype), *o, z=dev(z, dtype), activation="silu",
                                             per_row=per, **kw)
    need = cg._bytes("cgtp_grouped_layer_grad_bytes", cg.CGTP_BF16 if dtype == "bf16" else cg.CGTP_F32, t * per, G, K, N, 1,
                     cg.CGTP_ACT_SILU)
    space = torch.empty(need, dtype=torch.uint8, device="cuda")
    whole = run()
    _, dw, db = run(dx=False, workspace=space)
    assert torch.equal(dw, whole[1]) and torch.equal(db, whole[2])
    with pytest.raises(cg.CgtpError):
        run(workspace=space)
    if need > 0:
        with pytest.raises(cg.CgtpError):
            run(dx=False, workspace=space[:need - 1])


def test_forms_on_two_streams_and_in_graphs(cg):
    """bf16 gradients of every form, at once on two streams and replayed, give the bits of a call by itself."""
    import torch

    calls = []
    for i, (t, per, G, K, N) in enumerate([(20000, 1, 5, 100, 130), (5000, 4, 7, 128, 448), (6000, 2, 3, 300, 90), (3000, 1, 900, 64, 64),
                                           (9000, 1, 3, 64, 64), (700, 1, 5, 200, 16), (700, 1, 5, 16, 200), (9000, 1, 3, 333, 200)]):
        rng = np.random.default_rng(i)
        x, w, ids, z, dy = draw_grad(rng, t, per, G, K, N, "holes", "bf16")
        a = [dev(v, "bf16") for v in (x, w, dy, z)]
        o = cg.group_rows(dev(ids), G)
        calls.append(lambda a=a, o=o, per=per: cg.grouped_layer_grad(*a[:3], *o, z=a[3], activation="silu", per_row=per))
    want = [c() for c in calls]
    same = lambda got: all(torch.equal(g, h) for o, v in zip(got, want) for g, h in zip(o, v))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for i, c in enumerate(calls):
            with torch.cuda.stream(streams[i % 2]):
                got.append(c())
        torch.cuda.synchronize()
        assert same(got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [c() for c in calls]
    for _ in range(4):
        for o in got:
            for g in o:
                g.fill_(7)
        graph.replay()
        torch.randn(500, 500, device="cuda").sum()
        torch.cuda.synchronize()
        assert same(got)
