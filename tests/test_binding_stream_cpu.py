"""The binding's way to the current stream and device: torch's raw calls where they are there, its public ones where they are not.  A torch
without them imports the binding, and fails at a GPU call only."""
import importlib.util
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _import_again():
    at = os.path.join(ROOT, "paper_2506_13497_amd", "binding.py")
    spec = importlib.util.spec_from_file_location("_binding_again", at)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


class _Stream:
    def __init__(self, device):
        self.cuda_stream = 0x7000 + device


@pytest.mark.parametrize("gone", [("_cuda_getCurrentRawStream",), ("_cuda_getDevice",), ("_cuda_getCurrentRawStream", "_cuda_getDevice")])
def test_without_the_raw_calls(monkeypatch, gone):
    for name in gone:
        monkeypatch.delattr(torch._C, name, raising=False)
    b = _import_again()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: _Stream(3 if device is None else device))
    assert b._device() == 3 and b._raw_stream(3) == 0x7003 and b._stream().value == 0x7003
    assert b._on_device(None) == [None, 0x7003]
    with pytest.raises(b.DditError) as e:
        b._on_device(torch.zeros(4))
    assert e.value.status == b.DDIT_ERR_INVALID_ARG and "cuda:3" in str(e.value)


def test_with_the_raw_calls(monkeypatch):
    """They are taken together, and they are what answers."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 2, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0x5000 + device, raising=False)
    b = _import_again()
    assert b._device() == 2 and b._stream().value == 0x5002 and b._on_device() == [0x5002]
