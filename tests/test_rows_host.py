"""Refusals of the row operators and of AdamW, reported before anything touches a GPU, and the
binding's checks of its tensors."""
from __future__ import annotations

import ctypes

import pytest
import torch

import paper_2605_15073_amd as cg

P = ctypes.c_void_p(4096)          # a pointer that passes every check and is never read


@pytest.fixture(scope="module")
def lib():
    return cg.load_library()


def refused(lib, status, want=cg.CGTP_ERR_ARG):
    assert status == want
    assert lib.cgtp_last_error()


BAD_SIZES = [dict(dtype=1), dict(dtype=7), dict(n=-1), dict(n=2 ** 31), dict(G=0), dict(G=4097),
             dict(n_in=0), dict(n_out=0), dict(n_in=65537), dict(n_out=65537)]


def sizes(dtype=0, n=10, G=2, n_in=8, n_out=16):
    return dtype, n, G, n_in, n_out


@pytest.mark.parametrize("bad", BAD_SIZES)
def test_sizes(lib, bad):
    head, sz = sizes(**bad), ctypes.c_size_t()
    refused(lib, lib.cgtp_grouped_linear(*head, P, None, P, 8, P, P, 16, None))
    refused(lib, lib.cgtp_grouped_linear_grad_bytes(*head, ctypes.byref(sz)))
    refused(lib, lib.cgtp_grouped_linear_grad(*head, P, None, P, 8, P, P, 16, P, 8, P, P, 1 << 40, None))
    refused(lib, lib.cgtp_adapter_linear_bytes(*head, 4, ctypes.byref(sz)))
    refused(lib, lib.cgtp_adapter_linear(*head, 4, P, None, P, 8, P, P, P, None, P, 16, P, 1 << 40, None))
    refused(lib, lib.cgtp_adapter_linear_grad_bytes(*head, 4, ctypes.byref(sz)))
    refused(lib, lib.cgtp_adapter_linear_grad(*head, 4, P, None, P, 8, P, P, P, None, P, 16, P, 8, P, P,
                                              P, 1 << 40, None))


def test_group_rows(lib):
    sz = ctypes.c_size_t()
    for n, G in ((-1, 2), (2 ** 31, 2), (10, 0), (10, 4097)):
        refused(lib, lib.cgtp_group_rows_bytes(n, G, ctypes.byref(sz)))
        refused(lib, lib.cgtp_group_rows(n, G, P, P, P, P, 1 << 30, None))
    refused(lib, lib.cgtp_group_rows_bytes(10, 2, None))
    assert lib.cgtp_group_rows_bytes(10, 2, ctypes.byref(sz)) == cg.CGTP_OK and sz.value == 0
    assert lib.cgtp_group_rows_bytes(100000, 2, ctypes.byref(sz)) == cg.CGTP_OK and sz.value > 0
    refused(lib, lib.cgtp_group_rows(10, 2, None, P, P, None, 0, None))
    refused(lib, lib.cgtp_group_rows(10, 2, P, None, P, None, 0, None))
    refused(lib, lib.cgtp_group_rows(10, 2, P, P, None, None, 0, None))
    refused(lib, lib.cgtp_group_rows(10, 2, ctypes.c_void_p(4098), P, P, None, 0, None))
    refused(lib, lib.cgtp_group_rows(100000, 2, P, P, P, None, 0, None), cg.CGTP_ERR_WORKSPACE)
    refused(lib, lib.cgtp_group_rows(100000, 2, P, P, P, P, 16, None), cg.CGTP_ERR_WORKSPACE)
    refused(lib, lib.cgtp_group_rows(100000, 2, P, P, P, ctypes.c_void_p(4100), 1 << 30, None))


def test_pointers_and_strides(lib):
    odd = ctypes.c_void_p(4097)
    head = sizes()
    ok = dict(off=P, order=None, x=P, xs=8, w=P, y=P, ys=16)
    for bad in (dict(off=None), dict(order=ctypes.c_void_p(4098)), dict(x=None), dict(w=None),
                dict(y=None), dict(xs=7), dict(ys=15), dict(xs=2 ** 32), dict(x=odd), dict(y=odd)):
        a = {**ok, **bad}
        refused(lib, lib.cgtp_grouped_linear(*head, a["off"], a["order"], a["x"], a["xs"], a["w"], a["y"],
                                             a["ys"], None))
    grad = lambda x, w, dy, dx, dw, ws, nb: lib.cgtp_grouped_linear_grad(
        *head, P, None, x, 8, w, dy, 16, dx, 8, dw, ws, nb, None)
    refused(lib, grad(P, P, P, None, None, P, 1 << 30))
    refused(lib, grad(P, P, None, P, None, P, 1 << 30))
    refused(lib, grad(None, P, P, None, P, P, 1 << 30))
    refused(lib, grad(P, None, P, P, None, P, 1 << 30))


def test_adapters(lib):
    head, sz = sizes(), ctypes.c_size_t()
    for r in (0, -1, 65):
        refused(lib, lib.cgtp_adapter_linear_bytes(*head, r, ctypes.byref(sz)))
        refused(lib, lib.cgtp_adapter_linear(*head, r, P, None, P, 8, P, P, P, None, P, 16, P, 1 << 30, None))
    assert lib.cgtp_adapter_linear_bytes(*head, 4, ctypes.byref(sz)) == cg.CGTP_OK and sz.value > 0
    for hole in range(5):
        p = [P] * 5                          # x, w, a, b, y
        p[hole] = None
        refused(lib, lib.cgtp_adapter_linear(*head, 4, P, None, p[0], 8, p[1], p[2], p[3], None, p[4], 16, P,
                                             1 << 30, None))
    refused(lib, lib.cgtp_adapter_linear(*head, 4, P, None, P, 8, P, P, P, None, P, 16, None, 0, None),
            cg.CGTP_ERR_WORKSPACE)
    refused(lib, lib.cgtp_adapter_linear_grad(*head, 4, P, None, P, 8, P, P, P, None, P, 16, None, 8, None,
                                              None, P, 1 << 30, None))
    refused(lib, lib.cgtp_adapter_linear_grad(*head, 4, P, None, P, 8, P, P, P, None, P, 16, P, 8, P, P,
                                              P, 0, None), cg.CGTP_ERR_WORKSPACE)


def test_no_rows_is_no_work(lib):
    head = sizes(n=0)
    assert lib.cgtp_grouped_linear(*head, None, None, None, 0, None, None, 0, None) == cg.CGTP_OK
    assert lib.cgtp_adapter_linear(*head, 4, None, None, None, 0, None, None, None, None, None, 0, None, 0,
                                   None) == cg.CGTP_OK


def test_adamw(lib):
    h = ctypes.c_void_p()
    t = (cg._AdamWTensor * 1)(cg._AdamWTensor(4096, 4096, 4096, 4096, None, None, None, 5))
    create = lambda n, tab, gd, bits: lib.cgtp_adamw_create(n, tab, gd, bits, ctypes.byref(h))
    refused(lib, create(0, t, 0, 32))
    refused(lib, create(1, None, 0, 32))
    refused(lib, create(1, t, 1, 32))
    refused(lib, create(1, t, 0, 16))
    refused(lib, create(1, t, 0, 8))         # no scales
    refused(lib, lib.cgtp_adamw_create(1, t, 0, 32, None))
    for field, value in (("n", -1), ("param", None), ("grad", None), ("m", None), ("v", None),
                         ("param", 4098), ("grad", 4097), ("copy", 4097)):
        b = (cg._AdamWTensor * 1)(cg._AdamWTensor(4096, 4096, 4096, 4096, None, None, None, 5))
        setattr(b[0], field, value)
        refused(lib, create(1, b, 0, 32))
        assert h.value is None
    refused(lib, lib.cgtp_adamw_step(None, 0.1, 0.9, 0.99, 1e-8, 0.0, 1, None, None))
    refused(lib, lib.cgtp_adamw_states(None, None, None, None))
    assert lib.cgtp_adamw_destroy(None) == cg.CGTP_OK


def test_binding_refuses_host_tensors_and_shapes():
    i = torch.zeros(4, dtype=torch.int32)
    x, w, off = torch.zeros(4, 8), torch.zeros(2, 8, 3), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        cg.group_rows(i, 2)
    with pytest.raises(ValueError):
        cg.group_rows(i.view(2, 2), 2)
    with pytest.raises(ValueError):
        cg.grouped_linear(x, w, off)
    with pytest.raises(ValueError):
        cg.grouped_linear(x, w[0], off)
    with pytest.raises(ValueError):
        cg.adapter_linear(x, w[0], torch.zeros(2, 8, 4), torch.zeros(2, 4, 3), off)
    with pytest.raises(ValueError):
        cg.AdamWTensors([], [], [], [])
