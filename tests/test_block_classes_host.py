"""The Python classes of the operators around the attention, as far as they go without a GPU."""

import importlib.util
import types

import torch

import paper_2512_02541_b200 as P


def test_short_forms_that_torch_may_not_have(monkeypatch):
    """Without torch's private names for the current device and stream, the public ones serve."""
    for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
        monkeypatch.delattr(torch._C, name, raising=False)
    spec = importlib.util.spec_from_file_location("paper_2512_02541_b200.block_again", P.block.__file__)
    again = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(again)
    assert again._current_device is torch.cuda.current_device
    monkeypatch.setattr(torch.cuda, "current_stream", lambda index: types.SimpleNamespace(cuda_stream=100 + index))
    assert again._stream(3) == 103
