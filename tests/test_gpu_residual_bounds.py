"""The residual stream and its gradients against the fp64 statement, within bounds made of the rows' own sizes (``block_bounds``): a lost token, a
lost term or a lost segment is beyond them (``test_block_bounds_host.py``)."""

import pytest
import torch

from oracle import block_bounds as bounds
from test_gpu_residual import BF16, FP16, FP32, SIZES, TYPES, Problem, np64

pytestmark = pytest.mark.gpu


def step_of(dtype):
    info = torch.finfo(dtype)
    return (0.0 if dtype is FP32 else info.eps, info.tiny * info.eps / 2)


def check(pr):
    x, y, params = np64(pr.x), np64(pr.y), pr.np_params()
    limits = bounds.residual_forward(pr.orc, x, y, **params)
    got, want = ({n: t for n, t in zip("rh", both) if n in limits} for both in (map(np64, pr.forward()), pr.orc.forward(x, y, **params)))
    assert not bounds.beyond(got, want, limits, step_of(pr.res), step_of(pr.branch))
    args = [np64(pr.dh) if pr.norm != "none" else None, np64(pr.dr), np64(pr.r), np64(pr.y)]
    want, _ = pr.orc.backward(*args, **params)
    got = {n: np64(t) for n, t in pr.backward()._asdict().items() if t is not None}
    assert set(got) == set(want)
    assert not bounds.beyond(got, want, bounds.residual_backward(pr.orc, *args, **params), step_of(pr.res), step_of(pr.branch))


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("post", ("none", "layer", "rms"))
@pytest.mark.parametrize("size", SIZES + [(2000, 2304), (1374, 96), (300, 5120)])
def test_forward_and_backward(size, post, types):
    check(Problem(*size, *types, post=post))


@pytest.mark.parametrize("norm", ("layer", "rms", "none"))
@pytest.mark.parametrize("post", ("layer", "rms", "none"))
@pytest.mark.parametrize("types", [(BF16, BF16), (FP32, BF16), (FP32, FP32)])
@pytest.mark.parametrize("T,C,per_group,gate", [(26, 96, 5, "group"), (900, 1024, 300, "group"), (1600, 72, 1, "group"), (3001, 300, 2, "channel"),
                                                (1300, 520, 1, "group"), (7, 640, 1000, "group"), (400, 8192, 1, "group")])
def test_groups(T, C, per_group, gate, types, post, norm):
    check(Problem(T, C, *types, norm, post, gate, grouped=True, per_group=per_group, scale=0.7))


@pytest.mark.parametrize("gate,grouped", [("group", False), ("channel", True)])
@pytest.mark.parametrize("T,per_group", [(1500, 500), (2600, 1)])
def test_only_some_parameters_grouped(T, per_group, gate, grouped):
    check(Problem(T, 400, FP16, FP16, "layer", "layer", gate, grouped=grouped, per_group=per_group))


@pytest.mark.parametrize("stride,shift", [(1030, 0), (1027, 3), (1056, 16)])
@pytest.mark.parametrize("types", TYPES)
def test_strided_rows(stride, shift, types):
    check(Problem(300, 1024, *types, stride=stride, shift=shift, post="layer"))


def test_rows_far_from_zero():
    pr = Problem(12, 1024, FP32, FP32, post="rms")
    pr.x.add_(1000.0)                               # the mean is taken off before squares are summed
    check(pr)


def test_a_segments_rows_in_the_shared_memory_sums():
    """Every group's own row of the gate, one token each, more of them than a wave of blocks: sums that wait in shared memory."""
    for post in ("layer", "rms"):
        pr = Problem(400, 8192, FP32, BF16, "rms", post, "group", grouped=True, per_group=1)
        assert pr.T > torch.cuda.get_device_properties(0).multi_processor_count * 2
        check(pr)


@pytest.mark.parametrize("per_group", (1200, 2400, 5))
def test_sums_of_one_row_that_every_token_repeats(per_group):
    """Gradients of stride 0, where the roundings of a sum all go the same way."""
    pr = Problem(2400, 264, FP32, FP32, post="rms", gate="group", grouped=True, per_group=per_group)
    pr.dh, pr.dr = pr.dh[:1].expand(2400, 264), pr.dr[:1].expand(2400, 264)
    check(pr)
