"""AdamW over many tensors against the formulas: in single fp32 operations bit for bit (codes and
scales of 8-bit states too), and in 64 bits."""
from __future__ import annotations

import numpy as np
import pytest

from tests import rows_ref as ref

pytestmark = pytest.mark.gpu

HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.98, eps=1e-8, weight_decay=0.02)
SIZES = (1, 3, 4, 255, 256, 257, 1023, 4096, 4097, 70001)


@pytest.fixture(scope="module")
def cg():
    import torch

    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2605_15073_amd as lib

    lib.load_library()
    return lib


class Model:
    """Tensors of the given sizes with gradients of the given type; skew shifts every array by that
    many elements from an aligned start."""

    def __init__(self, sizes, bits, gdtype, skew=0, seed=0):
        import torch

        self.rng = np.random.default_rng(seed)
        self.bits, self.sizes = bits, sizes

        def place(a):
            t = torch.from_numpy(a).cuda()
            buf = torch.empty(t.numel() + skew, dtype=t.dtype, device="cuda")
            view = buf[skew:]
            view.copy_(t)
            return view

        f = lambda n: self.rng.standard_normal(n).astype(np.float32)
        self.p = [place(f(n)) for n in sizes]
        self.g = [place(f(n)).to(torch.bfloat16 if gdtype == "bf16" else torch.float32)
                  for n in sizes]
        if skew and gdtype == "bf16":
            self.g = [torch.cat([t.new_zeros(skew), t])[skew:] for t in self.g]
        nb = [(n + 255) // 256 for n in sizes]
        z = lambda n, t: place(np.zeros(n, t))
        self.m = [z(n, np.float32 if bits == 32 else np.int8) for n in sizes]
        self.v = [z(n, np.float32 if bits == 32 else np.uint8) for n in sizes]
        self.ms = [z(n, np.float32) for n in nb] if bits == 8 else None
        self.vs = [z(n, np.float32) for n in nb] if bits == 8 else None
        self.copy = [place(np.zeros(n, np.float32)).to(torch.bfloat16) for n in sizes]

    def new_gradients(self, k):
        import torch

        for i, g in enumerate(self.g):
            g.copy_(torch.from_numpy(self.rng.standard_normal(g.numel()) * 10.0 ** -(i % 5)))


def step_reference(model, host, k, grad_scale):
    """One step of the host copies, in fp32 operations."""
    out = []
    for i in range(len(model.sizes)):
        p, m, v, ms, vs = host[i]
        g = model.g[i].float().cpu().numpy()
        if model.bits == 8:
            m, v = ref.decode(m, ms, True), ref.decode(v, vs, False)
        p, m, v = ref.adamw(p, g, m, v, k, grad_scale=grad_scale, **HYPER)
        if model.bits == 8:
            m, v, ms, vs = ref.encode(m, v)
        out.append((p, m, v, ms, vs))
    return out


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gdtype", ["f32", "bf16"])
@pytest.mark.parametrize("skew", [0, 1])
def test_steps(cg, bits, gdtype, skew):
    import torch

    model = Model(SIZES, bits, gdtype, skew)
    tensors = cg.AdamWTensors(model.p, model.g, model.m, model.v, model.ms, model.vs, model.copy)
    num = lambda t: t.cpu().numpy().copy()
    host = [(num(model.p[i]), num(model.m[i]), num(model.v[i]),
             num(model.ms[i]) if bits == 8 else None, num(model.vs[i]) if bits == 8 else None)
            for i in range(len(SIZES))]
    scale = torch.tensor([0.25], device="cuda")
    for k in range(1, 6):
        model.new_gradients(k)
        host = step_reference(model, host, k, 0.25 if k % 2 else 1.0)
        cg.adamw(tensors, step=k, grad_scale=scale if k % 2 else None, **HYPER)
    torch.cuda.synchronize()
    for i, (p, m, v, ms, vs) in enumerate(host):
        assert np.array_equal(num(model.p[i]), p), (i, "p")
        assert np.array_equal(num(model.m[i]), m), (i, "m")
        assert np.array_equal(num(model.v[i]), v), (i, "v")
        if bits == 8:
            assert np.array_equal(num(model.ms[i]), ms), (i, "m_scale")
            assert np.array_equal(num(model.vs[i]), vs), (i, "v_scale")
        assert torch.equal(model.copy[i], model.p[i].to(torch.bfloat16)), (i, "copy")
    if bits == 8:
        mv, vv = cg.adamw_states(tensors)
        for i, (p, m, v, ms, vs) in enumerate(host):
            assert np.array_equal(num(mv[i]), ref.decode(m, ms, True))
            assert np.array_equal(num(vv[i]), ref.decode(v, vs, False))


def test_against_64_bits(cg):
    """One step from given moments. Each of about ten roundings is 2^-24 of an intermediate no
    larger than |p|, or than the terms of m', v' and the update; 2^-20 of their sum covers them."""
    import torch

    model = Model((5000,), 32, "f32", seed=2)
    model.m[0].copy_(torch.from_numpy(model.rng.standard_normal(5000)))
    model.v[0].copy_(torch.from_numpy(model.rng.standard_normal(5000) ** 2))
    p, g, m, v = (t[0].double().cpu().numpy() for t in (model.p, model.g, model.m, model.v))
    h, k = HYPER, 7
    cg.adamw(cg.AdamWTensors(model.p, model.g, model.m, model.v), step=k, **h)
    m2, v2 = h["beta1"] * m + (1 - h["beta1"]) * g, h["beta2"] * v + (1 - h["beta2"]) * g * g
    mag = h["beta1"] * np.abs(m) + (1 - h["beta1"]) * np.abs(g)
    den = np.sqrt(v2 / (1 - h["beta2"] ** k)) + h["eps"]
    rate = h["lr"] / (1 - h["beta1"] ** k)
    want = p * (1 - h["lr"] * h["weight_decay"]) - rate * m2 / den
    got = lambda t: t[0].double().cpu().numpy()
    u = 2.0 ** -20
    assert np.all(np.abs(got(model.m) - m2) <= u * mag)
    assert np.all(np.abs(got(model.v) - v2) <= u * v2)
    assert np.all(np.abs(got(model.p) - want) <= u * (np.abs(p) + rate * mag / den))


def test_eight_bit_states_stand_for_their_moments(cg):
    """A code is within half a step of the companded magnitude: |m| to (1/127) sqrt(|m| s) + s/4/127^2,
    v's fourth root to 1/510 of the scale's (or one step, where the floor of 1 holds)."""
    import torch

    model = Model((10000,), 8, "f32", seed=3)
    model.g[0].mul_(torch.logspace(-8, 0, 10000, device="cuda"))
    tensors = cg.AdamWTensors(model.p, model.g, model.m, model.v, model.ms, model.vs)
    cg.adamw(tensors, step=1, **HYPER)
    m, v = (t[0].double().cpu().numpy() for t in cg.adamw_states(tensors))
    g = model.g[0].double().cpu().numpy()
    m0, v0 = (1 - HYPER["beta1"]) * g, (1 - HYPER["beta2"]) * g * g
    sm = np.repeat(model.ms[0].double().cpu().numpy(), 256)[:10000]
    sv = np.repeat(model.vs[0].double().cpu().numpy(), 256)[:10000]
    assert np.all(np.abs(m - m0) <= 1.001 * (np.sqrt(np.abs(m0) * sm) / 127 + sm / 4 / 127 ** 2))
    step = np.abs(v ** 0.25 - v0 ** 0.25) / sv ** 0.25
    low = v0 ** 0.25 < sv ** 0.25 / 255
    assert np.all(step[~low] <= 1.001 / 510) and np.all(v[low] <= 1.001 * sv[low] / 255 ** 4)
    assert np.all(v[v0 > 0] > 0)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_non_finite_gradient(cg, bits, bad):
    """It spoils its element; with 8-bit states also the states of its block, no other block's."""
    import torch

    model = Model((1000,), bits, "f32", seed=4)
    model.g[0][300] = bad
    tensors = cg.AdamWTensors(model.p, model.g, model.m, model.v, model.ms, model.vs)
    cg.adamw(tensors, step=1, **HYPER)
    p = model.p[0].cpu().numpy()
    assert np.isnan(p[300]) and np.isfinite(np.delete(p, 300)).all()
    if bits == 8:
        assert np.isfinite(model.ms[0].cpu().numpy()[[0, 2, 3]]).all()
        assert not np.isfinite(model.ms[0].cpu().numpy()[1])


def test_zero_gradients_and_empty_tensors(cg):
    import torch

    for bits in (32, 8):
        model = Model((0, 300, 0), bits, "bf16", seed=5)
        model.g[1].zero_()
        before = model.p[1].clone()
        tensors = cg.AdamWTensors(model.p, model.g, model.m, model.v, model.ms, model.vs)
        cg.adamw(tensors, step=1, lr=0.5, weight_decay=0.0)
        assert torch.equal(model.p[1], before)
        assert (model.m[1] == 0).all() and (model.v[1] == 0).all()
        only = Model((0,), bits, "f32")
        cg.adamw(cg.AdamWTensors(only.p, only.g, only.m, only.v, only.ms, only.vs), step=1, lr=0.1)


def test_many_tensors(cg):
    """More tensors than one launch of the decoding takes; every one gets its own step."""
    sizes = tuple(1 + (i * 37) % 700 for i in range(150))
    model = Model(sizes, 8, "f32", seed=6)
    tensors = cg.AdamWTensors(model.p, model.g, model.m, model.v, model.ms, model.vs)
    host = [(model.p[i].cpu().numpy().copy(), np.zeros(n, np.int8), np.zeros(n, np.uint8),
             np.zeros((n + 255) // 256, np.float32), np.zeros((n + 255) // 256, np.float32))
            for i, n in enumerate(sizes)]
    host = step_reference(model, host, 1, 1.0)
    cg.adamw(tensors, step=1, **HYPER)
    mv, vv = cg.adamw_states(tensors)
    for i, (p, m, v, ms, vs) in enumerate(host):
        assert np.array_equal(model.p[i].cpu().numpy(), p), i
        assert np.array_equal(mv[i].cpu().numpy(), ref.decode(m, ms, True)), i
        assert np.array_equal(vv[i].cpu().numpy(), ref.decode(v, vs, False)), i


def test_another_stream_and_graph(cg):
    import torch

    a, b = Model((9000, 77), 8, "bf16", seed=7), Model((9000, 77), 8, "bf16", seed=7)
    ta = cg.AdamWTensors(a.p, a.g, a.m, a.v, a.ms, a.vs)
    tb = cg.AdamWTensors(b.p, b.g, b.m, b.v, b.ms, b.vs)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    cg.adamw(tb, step=1, stream=side, **HYPER)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cg.adamw(tb, step=2, **HYPER)
    cg.adamw(ta, step=1, **HYPER)
    for _ in range(3):
        graph.replay()
        cg.adamw(ta, step=2, **HYPER)
        torch.cuda.synchronize()
        for x, y in zip(a.p + a.m + a.v, b.p + b.m + b.v):
            assert torch.equal(x, y)


def test_refusals(cg):
    m = Model((8, 9), 32, "f32")
    good = lambda **kw: cg.AdamWTensors(**{**dict(params=m.p, grads=m.g, m=m.m, v=m.v), **kw})
    for kw in (dict(params=[]), dict(grads=m.g[:1]), dict(m=m.g[::-1]), dict(m_scale=m.p),
               dict(grads=[m.g[0], m.g[1].half()]), dict(copies=m.p),
               dict(params=[p.cpu() for p in m.p])):
        with pytest.raises((ValueError, cg.CgtpError)):
            good(**kw)
    t = good()
    for kw in (dict(step=0), dict(lr=float("nan")), dict(beta1=1.0), dict(beta2=-0.1),
               dict(eps=-1.0)):
        with pytest.raises(cg.CgtpError):
            cg.adamw(t, **{**dict(step=1, lr=0.1), **kw})
    with pytest.raises(ValueError):
        cg.adamw(t, step=1, lr=0.1, grad_scale=m.p[0])
    with pytest.raises(cg.CgtpError):
        cg.adamw_states(t)                   # states in 32 bits have nothing to decode
    t.close()
    with pytest.raises(cg.CgtpError):
        cg.adamw(t, step=1, lr=0.1)
