"""The Python classes of the operators around the attention, as far as they go without a GPU."""

import importlib.util
import types

import numpy as np
import pytest
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


@pytest.mark.parametrize("per_group", (2.0, 0.5, "3"))
def test_groups_of_a_fraction_of_a_token_are_refused(per_group):
    with pytest.raises(ValueError, match="tokens_per_group"):
        P.ResidualNorm(64, tokens_per_group=per_group)
    assert P.ResidualNorm(64, tokens_per_group=np.int64(3)).tokens_per_group == 3


@pytest.mark.parametrize("per_group", (None, 0, -2))
@pytest.mark.parametrize("name", ("weight", "bias", "gate"))
def test_parameters_of_groups_without_any_tokens_are_refused(name, per_group):
    """Found before anything asks for a device: the parameters are checked on the host."""
    op = P.ResidualNorm(16, tokens_per_group=per_group)
    params = dict.fromkeys(("weight", "bias", "gate", "post_weight", "post_bias"))
    params[name] = torch.zeros(2, 16)
    with pytest.raises(ValueError, match="tokens_per_group"):
        op._params(6, 0, P.AVGGT_TYPE_FP32, P.AVGGT_TYPE_FP32, **params)
