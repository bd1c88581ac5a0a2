"""The row operators on another stream than the current one: they take what the current stream has pending, whoever
allocated the outputs, and their tensors' memory stays until they are done."""
from __future__ import annotations

import numpy as np
import pytest

from tests.test_gpu_rows import cg, dev  # noqa: F401

pytestmark = pytest.mark.gpu

WAIT = 40_000_000   # cycles of the device's clock that a stream is kept busy for: tens of milliseconds at most


def _calls(cg, n=3000, G=4, n_in=64, n_out=72, r=8):
    """{name: (call(stream, outputs or None), the tensor whose values arrive late, outputs)}"""
    import torch

    rng = np.random.default_rng(0)
    ids = dev(rng.integers(0, G, n).astype(np.int32))
    offsets, order = cg.group_rows(ids, G)
    f = lambda *s: dev(rng.standard_normal(s))
    x, w, w0, a, b, dy = f(n, n_in), f(G, n_in, n_out), f(n_in, n_out), f(G, n_in, r), f(G, r, n_out), f(n, n_out)
    e = torch.empty_like
    o = offsets, order
    p, m, v, g = f(9000), f(9000), f(9000).abs(), f(9000)
    adam = cg.AdamWTensors([p], [g], [m], [v])
    p8, m8, v8 = f(9000), torch.zeros(9000, dtype=torch.int8, device="cuda"), torch.zeros(9000, dtype=torch.uint8, device="cuda")
    ms, vs = torch.zeros(36, device="cuda"), torch.zeros(36, device="cuda")
    m8.fill_(50), v8.fill_(90), ms.fill_(1), vs.fill_(1)
    codes = cg.AdamWTensors([p8], [f(9000)], [m8], [v8], [ms], [vs])
    return {
        "group_rows": (lambda s, y: cg.group_rows(ids, G, *(y or ()), stream=s), ids, [e(offsets), e(order)]),
        "grouped_linear": (lambda s, y: (cg.grouped_linear(x, w, *o, *(y or ()), stream=s),), x, [e(dy)]),
        "grouped_linear_grad": (lambda s, y: cg.grouped_linear_grad(x, w, dy, *o, *(y or ()), stream=s), dy, [e(x), e(w)]),
        "adapter_linear": (lambda s, y: (cg.adapter_linear(x, w0, a, b, *o, None, *(y or ()), stream=s),), x, [e(dy)]),
        "adapter_linear_grad": (lambda s, y: cg.adapter_linear_grad(x, w0, a, b, dy, *o, None, *(y or ()), stream=s), dy,
                                [e(x), e(a), e(b)]),
        "adamw": (lambda s, y: (cg.adamw(adam, 3, 1e-3, stream=s), p)[1:], g, [p]),
        "adamw_states": (lambda s, y: sum(cg.adamw_states(codes, *([t] for t in y or ()), stream=s), []), ms, [e(p8), e(p8)]),
    }


NAMES = ["group_rows", "grouped_linear", "grouped_linear_grad", "adapter_linear", "adapter_linear_grad", "adamw",
         "adamw_states"]


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("given", [False, True])
def test_another_stream_takes_pending_work(cg, name, given):
    import torch

    call, late, outs = _calls(cg)[name]
    values = late.clone()
    want = [t.clone() for t in call(None, None)]
    call, late, outs = _calls(cg)[name]            # the same start again, for what updates in place
    late.zero_()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(WAIT)
    late.copy_(values)                             # on the current stream, behind the wait
    got = call(side, outs if given else None)
    side.synchronize()
    for g, t in zip(got, want):
        assert torch.equal(g, t), name


def test_another_stream_keeps_inputs(cg):
    """Memory of an input that the caller drops is not handed out again before the call has read it."""
    import torch

    x, w = torch.ones(4000, 64, device="cuda"), torch.ones(1, 64, 96, device="cuda")
    offsets = torch.tensor([0, 4000], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    at = x.data_ptr()
    with torch.cuda.stream(side):
        torch.cuda._sleep(WAIT)
    y = cg.grouped_linear(x, w, offsets, stream=side)
    del x
    again = [torch.full((4000, 64), float("nan"), device="cuda") for _ in range(3)]
    assert all(t.data_ptr() != at for t in again)
    side.synchronize()
    assert (y == 64).all()
