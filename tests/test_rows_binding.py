"""The binding of the row operators, without a GPU."""
from __future__ import annotations

import ctypes
import types

import pytest
import torch

import paper_2605_15073_amd as cg


@pytest.fixture
def fresh():
    cg._current.cache_clear()
    yield
    cg._current.cache_clear()


def test_torch_without_its_own_calls(fresh, monkeypatch):
    """A torch that lacks the calls which the binding prefers is asked through its public ones."""
    for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        monkeypatch.delattr(torch._C, name, raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda index: types.SimpleNamespace(cuda_stream=100 + index))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    stream, device = cg._current()
    assert stream(2) == 102 and device() == 3
    like = types.SimpleNamespace(is_cuda=True, device=types.SimpleNamespace(index=2))
    assert cg._row_call(like, None) == (102, None)


def _tensor(at, n=1000, **over):
    """A table entry whose arrays lie 8,192 bytes apart; they are never read."""
    names = ("param", "grad", "m", "v", "m_scale", "v_scale", "copy")
    return cg._AdamWTensor(**{k: at + 8192 * i for i, k in enumerate(names)} | dict(n=n) | over)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_arrays_lie_apart(bits):
    """A tensor listed twice, or arrays that share bytes, are refused; neighbours and shared gradients are not."""
    lib, a, b = cg.load_library(), 1 << 20, 1 << 21

    def create(*tensors):
        handle = ctypes.c_void_p()
        status = lib.cgtp_adamw_create(len(tensors), (cg._AdamWTensor * len(tensors))(*tensors), cg.CGTP_F32, bits,
                                       ctypes.byref(handle))
        text = lib.cgtp_last_error().decode()
        if status == cg.CGTP_OK:
            lib.cgtp_adamw_destroy(handle)
        return status == cg.CGTP_ERR_ARG and "overlap" in text

    assert not create(_tensor(a), _tensor(b))
    assert not create(_tensor(a), _tensor(b, grad=a + 8192))
    assert not create(_tensor(a), _tensor(b, param=a + 4000))              # the next byte
    assert create(_tensor(a), _tensor(a))
    assert create(_tensor(b), _tensor(a, n=1, param=b + 3996))
    assert create(_tensor(a), _tensor(b, param=a + 3996))
    assert create(_tensor(a, m=a))
    assert create(_tensor(a, copy=a))
    assert create(_tensor(a), _tensor(b, v_scale=a + 5 * 8192)) == (bits == 8)
    assert not create(_tensor(a), _tensor(a, n=0))
