"""Refusals of routing, layers, joining and the gradients' norm, reported before anything touches a GPU, and the
binding's checks of its tensors."""
from __future__ import annotations

import ctypes

import pytest
import torch

import paper_2605_15073_amd as cg

P = ctypes.c_void_p(4096)          # a pointer that passes every check and is never read
ODD = ctypes.c_void_p(4097)
BIG = 1 << 50


@pytest.fixture(scope="module")
def lib():
    return cg.load_library()


def refused(lib, status, want=cg.CGTP_ERR_ARG):
    assert status == want
    assert lib.cgtp_last_error()


def route(lib, **over):
    a = dict(dtype=0, n=10, E=8, k=2, logits=P, stride=8, bias=P, score=0, blocks=1, keep=1, renorm=1, scale=1.0, ids=P,
             weights=P) | over
    return lib.cgtp_route_rows(*a.values(), None)


@pytest.mark.parametrize("bad", [
    dict(dtype=1), dict(n=-1), dict(n=2 ** 31), dict(E=0), dict(E=4097, stride=4097), dict(k=0), dict(k=9), dict(k=-1),
    dict(E=128, stride=128, k=65), dict(n=2 ** 30, k=2), dict(logits=None), dict(stride=7), dict(bias=ODD),
    dict(score=2), dict(score=-1), dict(blocks=0), dict(blocks=3), dict(blocks=128, E=128, stride=128), dict(blocks=2, keep=0),
    dict(blocks=2, keep=3), dict(blocks=4, keep=1, k=3), dict(renorm=2), dict(scale=float("nan")), dict(scale=float("inf")),
    dict(ids=None), dict(ids=ODD), dict(weights=None), dict(weights=ODD)])
def test_route(lib, bad):
    refused(lib, route(lib, **bad))


@pytest.mark.parametrize("bad", [
    dict(dtype=1), dict(n=-1), dict(k=0), dict(k=9), dict(logits=None), dict(stride=7), dict(ids=None), dict(du=None),
    dict(du=ODD), dict(score=2), dict(renorm=-1), dict(scale=float("nan")), dict(dl=None), dict(ds=7)])
def test_route_grad(lib, bad):
    a = dict(dtype=0, n=10, E=8, k=2, logits=P, stride=8, ids=P, du=P, score=0, renorm=1, scale=1.0, dl=P, ds=8) | bad
    refused(lib, lib.cgtp_route_rows_grad(*a.values(), None))


LAYER_SIZES = [dict(dtype=1), dict(n=-1), dict(n=2 ** 31), dict(G=0), dict(G=4097), dict(n_in=0), dict(n_out=65537),
               dict(per=0), dict(per=65), dict(per=4), dict(act=-1), dict(act=4)]


@pytest.mark.parametrize("bad", LAYER_SIZES + [
    dict(off=None), dict(order=ctypes.c_void_p(4098)), dict(x=None), dict(x=ODD), dict(xs=7), dict(w=None), dict(bias=ODD),
    dict(res=ODD), dict(rs=15), dict(y=None), dict(ys=15), dict(z=ODD), dict(zs=15)])
def test_layer(lib, bad):
    a = dict(dtype=0, n=10, G=2, n_in=8, n_out=16, per=2, off=P, order=P, x=P, xs=8, w=P, bias=P, act=1, res=P, rs=16, y=P,
             ys=16, z=P, zs=16) | bad
    refused(lib, lib.cgtp_grouped_layer(*a.values(), None))


def grad(lib, **over):
    a = dict(dtype=0, n=10, G=2, n_in=8, n_out=16, per=2, off=P, order=P, x=P, xs=8, w=P, z=P, zs=16, act=1, dy=P, dys=16,
             dx=P, dxs=8, dw=P, db=P, ws=P, nb=BIG) | over
    return lib.cgtp_grouped_layer_grad(*a.values(), None)


@pytest.mark.parametrize("bad", LAYER_SIZES + [
    dict(off=None), dict(x=None), dict(w=None), dict(z=None), dict(zs=15), dict(dy=None), dict(dys=15), dict(dxs=7),
    dict(dx=ODD), dict(dw=ODD), dict(db=ODD), dict(dx=None, dw=None, db=None), dict(ws=ctypes.c_void_p(4100))])
def test_layer_grad(lib, bad):
    refused(lib, grad(lib, **bad))


def test_layer_grad_workspace(lib):
    sz = ctypes.c_size_t()
    query = lambda *a: lib.cgtp_grouped_layer_grad_bytes(*a, ctypes.byref(sz))
    for bad in LAYER_SIZES:
        a = dict(dtype=0, n=10, G=2, n_in=8, n_out=16, per=2, act=1) | bad
        refused(lib, query(*a.values()))
    refused(lib, lib.cgtp_grouped_layer_grad_bytes(0, 10, 2, 8, 16, 2, 1, None))
    assert query(0, 10, 2, 8, 16, 2, 1) == cg.CGTP_OK and sz.value > 0
    refused(lib, grad(lib, ws=None, nb=0), cg.CGTP_ERR_WORKSPACE)
    refused(lib, grad(lib, nb=sz.value - 1), cg.CGTP_ERR_WORKSPACE)


@pytest.mark.parametrize("bad", [
    dict(dtype=1), dict(n=-1), dict(n=2 ** 30, per=2), dict(per=0), dict(per=65), dict(width=0), dict(width=65537),
    dict(y=None), dict(ys=15), dict(w=ODD), dict(res=ODD), dict(rs=15), dict(out=None), dict(os=15)])
def test_mix(lib, bad):
    a = dict(dtype=0, n=10, per=2, width=16, y=P, ys=16, w=P, res=P, rs=16, out=P, os=16) | bad
    refused(lib, lib.cgtp_mix_rows(*a.values(), None))


@pytest.mark.parametrize("bad", [
    dict(dtype=1), dict(n=-1), dict(n=2 ** 30, per=2), dict(per=0), dict(per=65), dict(width=0), dict(d=None), dict(ds=15),
    dict(w=ODD), dict(y=None), dict(ys=15), dict(dy=ODD), dict(dys=15), dict(dw=ODD), dict(dy=None, dw=None)])
def test_mix_grad(lib, bad):
    a = dict(dtype=0, n=10, per=2, width=16, d=P, ds=16, w=P, y=P, ys=16, dy=P, dys=16, dw=P) | bad
    refused(lib, lib.cgtp_mix_rows_grad(*a.values(), None))


def test_no_rows_is_no_work(lib):
    assert route(lib, n=0, logits=None, bias=None, ids=None, weights=None, stride=0) == cg.CGTP_OK
    assert lib.cgtp_route_rows_grad(0, 0, 8, 2, None, 0, None, None, 0, 1, 1.0, None, 0, None) == cg.CGTP_OK
    assert lib.cgtp_grouped_layer(0, 0, 2, 8, 16, 2, None, None, None, 0, None, None, 1, None, 0, None, 0, None, 0,
                                  None) == cg.CGTP_OK
    assert grad(lib, n=0, dw=None, db=None, x=None, dy=None, z=None, dx=None, off=None, ws=None, nb=0) == cg.CGTP_OK
    assert lib.cgtp_mix_rows(0, 0, 2, 16, None, 0, None, None, 0, None, 0, None) == cg.CGTP_OK
    assert lib.cgtp_mix_rows_grad(0, 0, 2, 16, None, 0, None, None, 0, None, 0, None, None) == cg.CGTP_OK


def test_grad_norm(lib):
    sz = ctypes.c_size_t()
    refused(lib, lib.cgtp_adamw_grad_norm_bytes(None, ctypes.byref(sz)))
    refused(lib, lib.cgtp_adamw_grad_norm(None, 1.0, None, P, P, P, BIG, None))


def test_binding_refuses_host_tensors_and_choices():
    x, w, off = torch.zeros(4, 8), torch.zeros(2, 8, 3), torch.zeros(3, dtype=torch.int32)
    i = torch.zeros(4, 2, dtype=torch.int32)
    for call in (lambda: cg.route_rows(x, 2), lambda: cg.route_rows(x, 2, score="max"), lambda: cg.route_rows(x[0], 2),
                 lambda: cg.route_rows_grad(x, i, torch.zeros(4, 2)), lambda: cg.route_rows_grad(x, i[0], torch.zeros(4, 2)),
                 lambda: cg.grouped_layer(x, w, off), lambda: cg.grouped_layer(x, w[0], off),
                 lambda: cg.grouped_layer(x, w, off, activation="tanh"),
                 lambda: cg.grouped_layer_grad(x, w, torch.zeros(4, 3), off),
                 lambda: cg.grouped_layer_grad(x, w, torch.zeros(4, 3), off, activation="silu"),
                 lambda: cg.mix_rows(x, 2), lambda: cg.mix_rows(x, 3), lambda: cg.mix_rows(x, 0), lambda: cg.mix_rows(x[0], 1),
                 lambda: cg.mix_rows_grad(x, 2, y=torch.zeros(8, 8)), lambda: cg.mix_rows_grad(x, 2)):
        with pytest.raises(ValueError):
            call()
