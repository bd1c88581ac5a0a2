"""The binding of the row operators, without a GPU."""
from __future__ import annotations

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
