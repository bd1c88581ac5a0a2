"""Row operators at the sizes they are made for: workgroups that run over many column tiles, chunks that are joined,
stores past the caches, offsets beyond 32 bits. References in 64 bits, on the GPU."""
from __future__ import annotations

import numpy as np
import pytest

from tests import rows_ref as ref
from tests.test_gpu_rows import cg  # noqa: F401

pytestmark = pytest.mark.gpu

TYPES = {"f32": "float32", "bf16": "bfloat16"}


def normal(seed, dtype, *shape, by=1.0):
    import torch

    g = torch.Generator("cuda")
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * by).to(getattr(torch, TYPES[dtype]))


def uneven(n, G, seed=0):
    """Ids of an uneven composition; a twentieth of the rows has none."""
    import torch

    g = torch.Generator("cuda")
    g.manual_seed(seed)
    u = torch.rand(n, generator=g, device="cuda")
    ids = (G * u * u).to(torch.int32).clamp(max=G - 1)
    ids[torch.rand(n, generator=g, device="cuda") < 0.05] = -1
    return ids


def bound(terms, magnitude, value, dtype):
    return ref.U_SUM * (terms + 4) * magnitude + ref._out(dtype) * value.abs() + 1e-37


def near(got, want, terms, magnitude, dtype, what):
    err, most = (got.double() - want).abs(), bound(terms, magnitude, want, dtype)
    assert bool((err <= most).all()), (what, float((err / most).max()))


def rows_of(ids, G, most=64, seed=0):
    """{group: up to `most` of its rows}, the first and the last among them, for all groups or 200 of them."""
    import torch

    rng, out = np.random.default_rng(seed), {}
    ids = ids.cpu().numpy()
    by = np.argsort(ids, kind="stable")
    values, first = np.unique(ids[by], return_index=True)
    parts = dict(zip(values.tolist(), np.split(by, first[1:])))
    for g in sorted(parts) if G <= 200 else rng.choice(sorted(parts), 200, replace=False).tolist():
        rows = parts[g]
        if len(rows) > most:
            rows = np.unique(np.concatenate([rows[:2], rows[-2:], rng.choice(rows, most - 4, replace=False)]))
        out[g] = torch.from_numpy(rows).cuda()
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,G,n_in,n_out", [(40000, 7, 64, 896), (40000, 7, 64, 900), (70000, 3, 16, 452), (70000, 40, 33, 451),
                                            (270000, 10, 64, 480), (270000, 300, 8, 897), (40000, 7, 128, 912),
                                            (60000, 5, 200, 700), (60000, 5, 140, 1345), (90000, 2, 300, 40), (90000, 2, 257, 130)])
def test_products_over_many_column_tiles(cg, dtype, n, G, n_in, n_out):
    ids = uneven(n, G)
    offsets, order = cg.group_rows(ids, G)
    x, w = normal(1, dtype, n, n_in), normal(2, dtype, G, n_in, n_out, by=n_in ** -0.5)
    y = cg.grouped_linear(x, w, offsets, order)
    wt = w.transpose(1, 2).contiguous()                   # the row gradient of the transposed weights: the same products
    dx, _ = cg.grouped_linear_grad(y, wt, x, offsets, order, dw=False)
    for g, rows in rows_of(ids, G).items():
        if g < 0:
            assert bool((y[rows] == 0).all()) and bool((dx[rows] == 0).all())
            continue
        xg, wg = x[rows].double(), w[g].double()
        for got, what in ((y, "y"), (dx, "dx")):
            near(got[rows], xg @ wg, n_in, xg.abs() @ wg.abs(), dtype, (what, g))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,G,n_in,n_out,r", [
    (60000, 8, 64, 896, 16), (60000, 8, 64, 900, 32), (60000, 8, 33, 451, 5),           # one adapter a tile
    (100000, 2000, 64, 896, 16), (100000, 2000, 64, 452, 24), (100000, 2000, 40, 451, 4),  # several
    (60000, 8, 200, 700, 16), (30000, 1000, 140, 900, 40)])
@pytest.mark.parametrize("runs", [True, False])
def test_adapters_over_many_column_tiles(cg, dtype, n, G, n_in, n_out, r, runs):
    import torch

    ids = uneven(n, G)
    if runs:
        ids = torch.sort(ids).values
    offsets, order = cg.group_rows(ids, G)
    x, w = normal(1, dtype, n, n_in), normal(2, dtype, n_in, n_out, by=n_in ** -0.5)
    a, b = normal(3, dtype, G, n_in, r, by=n_in ** -0.5), normal(4, dtype, G, r, n_out, by=r ** -0.5)
    scale = normal(5, "f32", G)
    y = cg.adapter_linear(x, w, a, b, offsets, order, scale=scale)
    for g, rows in rows_of(ids, G).items():
        xg, wd = x[rows].double(), w.double()
        want, mag = xg @ wd, xg.abs() @ wd.abs()
        if g >= 0:
            want = want + float(scale[g]) * (xg @ a[g].double()) @ b[g].double()
            mag = mag + abs(float(scale[g])) * (xg.abs() @ a[g].double().abs()) @ b[g].double().abs()
        near(y[rows], want, 2 * n_in + 2 * r, mag, dtype, g)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,G,n_in,n_out,r", [(130000, 3, 128, 896, 16), (130000, 3, 64, 451, 32), (60000, 40, 200, 300, 8),
                                              (200000, 1, 37, 129, 4), (50000, 4000, 40, 130, 8)])
def test_gradients_over_many_chunks(cg, dtype, n, G, n_in, n_out, r):
    ids = uneven(n, G)
    offsets, order = cg.group_rows(ids, G)
    x, dy, w = normal(1, dtype, n, n_in), normal(2, dtype, n, n_out), normal(3, dtype, G, n_in, n_out)
    _, dw = cg.grouped_linear_grad(x, w, dy, offsets, order, dx=False)
    a, b = normal(4, dtype, G, n_in, r, by=n_in ** -0.5), normal(5, dtype, G, r, n_out, by=r ** -0.5)
    dx, da, db = cg.adapter_linear_grad(x, w[0].contiguous(), a, b, dy, offsets, order)
    wd = w[0].double()
    for g, rows in rows_of(ids, G, most=n).items():
        few = rows[:: max(1, len(rows) // 64)]
        dyf = dy[few].double()
        want, mag = dyf @ wd.t(), dyf.abs() @ wd.abs().t()
        if g >= 0:
            xg, dg, ag, bg = x[rows].double(), dy[rows].double(), a[g].double(), b[g].double()
            near(dw[g], xg.t() @ dg, len(rows), xg.abs().t() @ dg.abs(), dtype, ("dw", g))
            u, um, h, hm = dg @ bg.t(), dg.abs() @ bg.abs().t(), xg @ ag, xg.abs() @ ag.abs()
            near(da[g], xg.t() @ u, len(rows) + n_out, xg.abs().t() @ um, dtype, ("da", g))
            near(db[g], h.t() @ dg, len(rows) + n_in, hm.t() @ dg.abs(), dtype, ("db", g))
            want = want + (dyf @ bg.t()) @ ag.t()
            mag = mag + (dyf.abs() @ bg.abs().t()) @ ag.abs().t()
        near(dx[few], want, 2 * n_out + 2 * r, mag, dtype, ("dx", g))


def test_gradients_and_adapters_beyond_32_bit_offsets(cg):
    """More than 2^31 elements of x, of dy and of y; whole numbers, exact at any order."""
    import torch

    n, n_in, n_out, r = 1300000, 1704, 1712, 2
    i = torch.arange(n, device="cuda")
    ids = (i % 3).to(torch.int32)
    offsets, order = cg.group_rows(ids, 3)
    x = torch.zeros(n, n_in, dtype=torch.bfloat16, device="cuda")
    dy = torch.zeros(n, n_out, dtype=torch.bfloat16, device="cuda")
    late = i >= n - 3000                                      # rows whose elements lie beyond 2^31
    x[:, 5], x[:, n_in - 1] = (i % 2).to(x.dtype), late.to(x.dtype)
    dy[:, 7], dy[:, n_out - 1] = late.to(x.dtype), (1 + i % 3).to(x.dtype) * late.to(x.dtype)
    w = torch.zeros(3, n_in, n_out, dtype=torch.bfloat16, device="cuda")
    _, dw = cg.grouped_linear_grad(x, w, dy, offsets, order, dx=False)
    xd, dd = x[late].double(), dy[late].double()
    for g in range(3):
        at = ids[late] == g
        want = xd[at].t() @ dd[at]
        assert torch.equal(dw[g].double(), want.to(torch.bfloat16).double()), g
    a = torch.zeros(3, n_in, r, dtype=torch.bfloat16, device="cuda")
    b = torch.zeros(3, r, n_out, dtype=torch.bfloat16, device="cuda")
    a[:, 5, 0] = a[:, n_in - 1, 1] = 1
    b[:, 0, 3], b[:, 1, 3], b[:, 1, n_out - 1] = 1, 2, torch.arange(1, 4, device="cuda").to(b.dtype)
    w0 = w[0].contiguous()
    y = cg.adapter_linear(x, w0, a, b, offsets, order)
    assert torch.equal(y[:, 3].double(), (i % 2 + 2 * late).double())
    assert torch.equal(y[:, n_out - 1].double(), ((1 + i % 3) * late).double())
    del y
    b[:, 0, 7] = b[:, 1, 7] = 1
    dx, da, db = cg.adapter_linear_grad(x, w0, a, b, dy, offsets, order)
    u = dd @ torch.stack([b[0, 0], b[0, 1]]).double().t()     # b's first rows are alike but for the last column
    u[:, 1] = dd[:, 7] + dd[:, n_out - 1] * (1 + ids[late])
    assert torch.equal(dx[late][:, [5, n_in - 1]].double(), u) and bool((dx[~late] == 0).all())
    for g in range(3):
        at = ids[late] == g
        h = torch.stack([xd[at][:, 5], xd[at][:, n_in - 1]], 1)
        for got, want in ((da[g], xd[at].t() @ u[at]), (db[g], h.t() @ dd[at])):
            assert torch.equal(got.double(), want.to(torch.bfloat16).double()), g


@pytest.mark.parametrize("bits,gdtype,total", [(32, "f32", 11000000), (8, "bf16", 28000000), (8, "f32", 28000000)])
def test_adamw_past_the_caches(cg, bits, gdtype, total):
    """More bytes than the memory-side cache holds: two steps and the states, bit for bit."""
    import torch

    from tests.test_gpu_adamw import HYPER, Model, step_reference

    m = Model((total - 70001, 70001), bits, gdtype)
    scales = () if bits == 32 else (m.ms, m.vs)
    t = cg.AdamWTensors(m.p, m.g, m.m, m.v, *(scales or (None, None)), m.copy)
    get = lambda x: [a.cpu().numpy() for a in x]
    host = list(zip(get(m.p), get(m.m), get(m.v), *(map(get, scales) if scales else ([None] * 2,) * 2)))
    for step in (1, 2):
        m.new_gradients(step)
        host = step_reference(m, host, step, 0.5)
        cg.adamw(t, step, grad_scale=torch.full((1,), 0.5, device="cuda"), **HYPER)
        for i, want in enumerate(host):
            got = [m.p[i], m.m[i], m.v[i]] + ([m.ms[i], m.vs[i]] if scales else [])
            for g, w in zip(got, want):
                assert np.array_equal(g.cpu().numpy(), w), (step, i)
            assert torch.equal(m.copy[i], m.p[i].to(torch.bfloat16))
    if scales:
        for i, (mv, vv) in enumerate(zip(*cg.adamw_states(t))):
            assert np.array_equal(mv.cpu().numpy(), ref.decode(host[i][1], host[i][3], True))
            assert np.array_equal(vv.cpu().numpy(), ref.decode(host[i][2], host[i][4], False))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_a_graph(cg, dtype):
    """Forward and backward passes and a step of AdamW, captured and replayed on new inputs."""
    import torch

    n, G, n_in, n_out, r = 5000, 6, 64, 200, 8
    ids, x, dy = uneven(n, G), normal(1, dtype, n, n_in), normal(2, dtype, n, n_out)
    w, w0 = normal(3, dtype, G, n_in, n_out), normal(4, dtype, n_in, n_out)
    a, b = normal(5, dtype, G, n_in, r), normal(6, dtype, G, r, n_out)
    dw = torch.empty_like(w)
    param = normal(7, "f32", G, n_in, n_out)
    opt = cg.AdamWTensors([param], [dw], [torch.zeros_like(param)], [torch.zeros_like(param)])

    def call():
        o = cg.group_rows(ids, G)
        y = cg.grouped_linear(x, w, *o)
        dx, _ = cg.grouped_linear_grad(x, w, dy, *o, dw=dw)
        z = cg.adapter_linear(x, w0, a, b, *o)
        grads = cg.adapter_linear_grad(x, w0, a, b, dy, *o)
        cg.adamw(opt, 5, 1e-3)
        return [*o, y, dx, dw, z, *grads, param]

    start = param.clone()
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = call()
    for k in range(4):
        x.copy_(normal(10 + k, dtype, n, n_in))
        ids.copy_(uneven(n, G, k))
        opt2 = [t.clone() for t in (start, opt._keep[2][0], opt._keep[3][0])]
        param.copy_(start)
        graph.replay()
        got = [t.clone() for t in outs]
        for t, v in zip((param, opt._keep[2][0], opt._keep[3][0]), opt2):
            t.copy_(v)
        torch.cuda.synchronize()
        for g, t in zip(got, call()):
            assert torch.equal(g, t), k
