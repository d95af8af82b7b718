"""A stream of another device than the tensors' is refused: a kernel launched there may not reach them.  Stand-ins, no GPU."""
import types

import pytest
import torch

import paper_2601_17917_amd as sd


def tensor(index):
    return types.SimpleNamespace(get_device=lambda: index, device=f"cuda:{index}")


def test_streams_and_tensors_on_the_current_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    stream = lambda index: types.SimpleNamespace(device=torch.device("cuda", index), cuda_stream=0)
    sd._on_current_device(None, tensor(1), None)
    sd._on_current_device(stream(1), tensor(1))
    for args in ((None, tensor(1), tensor(0)), (stream(0), tensor(1)), (stream(0), tensor(0)), (stream(2),)):
        with pytest.raises(sd.SdllmError, match="current device"):
            sd._on_current_device(*args)
