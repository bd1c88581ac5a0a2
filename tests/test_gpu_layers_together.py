"""Routing, layers, joining and clipping as a training step runs them: against torch's own differentiation in 64 bits,
captured into graphs, and on another stream."""
from __future__ import annotations

import math

import numpy as np
import pytest

from tests.test_gpu_rows import cg, dev, host, rounded  # noqa: F401
from tests.test_gpu_rows_streams import WAIT

pytestmark = pytest.mark.gpu

OPTIONS = dict(score="sigmoid", renormalize=True, scale=1.5)


def _weights(rng, E, width, hidden):
    f = lambda *s, by=1.0: dev(rounded(by * rng.standard_normal(s), "f32"))
    return dict(router=f(1, width, E, by=width ** -0.5), w1=f(E, width, hidden, by=width ** -0.5), b1=f(E, hidden, by=0.1),
                w2=f(E, hidden, width, by=hidden ** -0.5), b2=f(E, width, by=0.1))


class Step:
    """Rows to k of E experts of two layers each, joined and added to the rows; the gradients of all weights, clipped, and
    one step of them."""

    def __init__(self, cg, n=700, E=6, k=2, width=24, hidden=40, seed=0):
        import torch

        rng = np.random.default_rng(seed)
        self.cg, self.n, self.E, self.k = cg, n, E, k
        self.x = dev(rounded(rng.standard_normal((n, width)), "f32"))
        self.dout = dev(rounded(rng.standard_normal((n, width)), "f32"))
        self.balance = dev(rounded(0.05 * rng.standard_normal(E), "f32"))
        self.p = _weights(rng, E, width, hidden)
        self.g = {name: torch.zeros_like(t) for name, t in self.p.items()}
        zeros = lambda: [torch.zeros_like(t) for t in self.p.values()]
        self.m, self.v = zeros(), zeros()
        self.opt = cg.AdamWTensors(list(self.p.values()), list(self.g.values()), self.m, self.v)
        self.all = cg.group_rows(torch.zeros(n, dtype=torch.int32, device="cuda"), 1)

    def forward(self):
        cg, p = self.cg, self.p
        self.logits = cg.grouped_layer(self.x, p["router"], *self.all)
        self.ids, self.share = cg.route_rows(self.logits, self.k, bias=self.balance, **OPTIONS)
        self.order = cg.group_rows(self.ids.view(-1), self.E)
        self.h, self.z = cg.grouped_layer(self.x, p["w1"], *self.order, bias=p["b1"], activation="silu", per_row=self.k, z=None)
        self.y = cg.grouped_layer(self.h, p["w2"], *self.order, bias=p["b2"])
        return cg.mix_rows(self.y, self.k, weights=self.share, residual=self.x)

    def backward(self):
        cg, p, g = self.cg, self.p, self.g
        dy, dshare = cg.mix_rows_grad(self.dout, self.k, weights=self.share, y=self.y)
        dh, _, _ = cg.grouped_layer_grad(self.h, p["w2"], dy, *self.order, dw=g["w2"], dbias=g["b2"])
        dx, _, _ = cg.grouped_layer_grad(self.x, p["w1"], dh, *self.order, z=self.z, activation="silu", per_row=self.k,
                                         dw=g["w1"], dbias=g["b1"])
        dlogits = cg.route_rows_grad(self.logits, self.ids, dshare, **OPTIONS)
        dr, _, _ = cg.grouped_layer_grad(self.x, p["router"], dlogits, *self.all, dw=g["router"], dbias=False)
        self.dx = self.dout + dx + dr
        return self.dx

    def run(self, step=1):
        out = self.forward()
        dx = self.backward()
        self.norm, scale = self.cg.adamw_grad_norm(self.opt, 1.0)
        self.cg.adamw(self.opt, step=step, lr=1e-3, grad_scale=scale)
        return [out, dx, self.norm, scale, self.ids, self.share, *self.g.values(), *self.p.values()]


def test_against_torch(cg):
    """Sums of at most 40 products of each of four layers in fp32, of 1,400 rows in the weights' gradients: 1e-5 of the
    largest, where they are off by 2^-24 times a few hundred at most."""
    import torch

    s = Step(cg)
    p = {name: t.double().requires_grad_() for name, t in s.p.items()}
    x = s.x.double().requires_grad_()
    out, dx, norm, scale, ids, share, *grads = s.run()[:6 + len(s.g)]
    at = ids.long()
    score = torch.sigmoid(x @ p["router"][0])
    chosen = torch.gather(score, 1, at)
    assert torch.equal(torch.topk(score + s.balance.double(), s.k, dim=1).indices, at)
    w = 1.5 * chosen / chosen.sum(1, keepdim=True)
    want = x
    for j in range(s.k):
        rows = torch.zeros_like(x)
        for e in range(s.E):
            on = (at[:, j] == e).double()[:, None]
            z = x @ p["w1"][e] + p["b1"][e]
            rows = rows + on * ((z * torch.sigmoid(z)) @ p["w2"][e] + p["b2"][e])
        want = want + w[:, j:j + 1] * rows
    want.backward(s.dout.double())
    near = lambda a, b: (a.double() - b).abs().max() <= 1e-5 * b.abs().max()
    assert near(out, want.detach()) and near(share, w.detach()) and near(dx, x.grad)
    for name, g in zip(s.g, grads):
        assert near(g, p[name].grad), name
    total = math.sqrt(sum(float(t.grad.square().sum()) for t in p.values()))
    assert abs(norm.item() - total) <= 1e-5 * total and abs(scale.item() - min(1, 1 / total)) <= 1e-5


def test_captured_and_replayed(cg):
    """A whole step in a graph: every replay gives the eager step's bits, with eager work of other sizes between them."""
    import torch

    eager, graphed = Step(cg, seed=3), Step(cg, seed=3)
    start = [t.clone() for t in (*graphed.p.values(), *graphed.m, *graphed.v)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graphed.run()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = graphed.run()
    for t, s in zip((*graphed.p.values(), *graphed.m, *graphed.v), start):
        t.copy_(s)
    for k in range(4):
        new = torch.randn(eager.x.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(k))
        eager.x.copy_(new)
        graphed.x.copy_(new)
        want = [t.clone() for t in eager.run()]
        Step(cg, n=50 + 300 * k, E=4, seed=k).run()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(outs, want)):
            assert torch.equal(a, b), (k, i)


def test_two_graphs_at_once(cg):
    """Two captured steps of their own tensors, replayed on two streams at the same time."""
    import torch

    steps, graphs, outs, want = [Step(cg, seed=k) for k in (5, 6)], [], [], []
    for s in steps:
        keep = [t.clone() for t in (*s.p.values(), *s.m, *s.v)]
        want.append([t.clone() for t in s.run()])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(s.run())
        graphs.append(g)
        for t, k in zip((*s.p.values(), *s.m, *s.v), keep):
            t.copy_(k)
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    for g, t in zip(graphs, streams):
        with torch.cuda.stream(t):
            g.replay()
    torch.cuda.synchronize()
    for a, b in zip(outs, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def _calls(cg):
    """{name: (call(stream, outputs or None), the tensor whose values arrive late, outputs)}"""
    import torch

    s = Step(cg, n=3000)
    s.forward()
    s.backward()
    p, e = s.p, torch.empty_like
    dh = e(s.h).copy_(s.h)
    wide = torch.empty(s.n, s.E, device="cuda")
    one = lambda: torch.empty(1, device="cuda")
    return {
        "route_rows": (lambda st, o: cg.route_rows(s.logits, s.k, **OPTIONS, **dict(zip(("ids", "weights"), o or ())), stream=st),
                       s.logits, [e(s.ids), e(s.share)]),
        "route_rows_grad": (lambda st, o: (cg.route_rows_grad(s.logits, s.ids, s.share, **OPTIONS, dlogits=(o or [None])[0],
                                                              stream=st),), s.share, [wide]),
        "grouped_layer": (lambda st, o: cg.grouped_layer(s.x, p["w1"], *s.order, bias=p["b1"], activation="gelu", per_row=s.k,
                                                         y=(o or [None])[0], z=(o or [None, None])[1], stream=st),
                          s.x, [e(s.h), e(s.h)]),
        "grouped_layer_grad": (lambda st, o: cg.grouped_layer_grad(s.x, p["w1"], dh, *s.order, z=s.z, activation="silu",
                                                                   per_row=s.k, **dict(zip(("dx", "dw", "dbias"), o or ())),
                                                                   stream=st), dh, [e(s.x), e(p["w1"]), e(p["b1"])]),
        "mix_rows": (lambda st, o: (cg.mix_rows(s.y, s.k, weights=s.share, residual=s.x, out=(o or [None])[0], stream=st),), s.y,
                     [e(s.x)]),
        "mix_rows_grad": (lambda st, o: cg.mix_rows_grad(s.dout, s.k, weights=s.share, y=s.y, **dict(zip(("dy", "dweights"),
                                                         o or ())), stream=st), s.dout, [e(s.y), e(s.share)]),
        "adamw_grad_norm": (lambda st, o: cg.adamw_grad_norm(s.opt, 1.0, **dict(zip(("norm", "scale"), o or ())), stream=st),
                            s.g["w1"], [one(), one()]),
    }


@pytest.mark.parametrize("name", ["route_rows", "route_rows_grad", "grouped_layer", "grouped_layer_grad", "mix_rows",
                                  "mix_rows_grad", "adamw_grad_norm"])
@pytest.mark.parametrize("given", [False, True])
def test_another_stream_takes_pending_work(cg, name, given):
    import torch

    call, late, outs = _calls(cg)[name]
    values = late.clone()
    want = [t.clone() for t in call(None, None)]
    late.zero_()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(WAIT)
    late.copy_(values)                             # on the current stream, behind the wait
    got = call(side, outs if given else None)
    side.synchronize()
    for g, t in zip(got, want):
        assert torch.equal(g, t), name
