"""The residual stream's gradients over the range of 32 bits: rows of large and of small values, rows of zeros behind a tiny eps, on the
GPU against the fp64 statement within bounds made of the rows' own sizes (``block_bounds``)."""

import numpy as np
import pytest
import torch

import paper_2512_02541_b200 as P
from oracle import block_bounds as bounds
from oracle import block_oracle as orc

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
NORMS = {"none": P.AVGGT_NORM_NONE, "layer": P.AVGGT_NORM_LAYER, "rms": P.AVGGT_NORM_RMS}


def np64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def step_of(dtype):
    info = torch.finfo(dtype)
    return (0.0 if dtype is FP32 else info.eps, info.tiny * info.eps / 2)


def check(T, C, res, branch, norm, post, eps, r, y, dr, dh, per_group=None):
    gen = torch.Generator(device="cuda").manual_seed(5)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda")
    rows = (C,) if per_group is None else (-(-T // per_group), C)
    params = dict(weight=normal(*rows) if norm != "none" else None, bias=normal(*rows) if norm != "none" else None, gate=normal(*rows),
                  post_weight=1 + 0.2 * normal(C) if post != "none" else None, post_bias=0.2 * normal(C) if post != "none" else None)
    op = P.ResidualNorm(C, norm=NORMS[norm], eps=eps, post_norm=NORMS[post], post_eps=eps, tokens_per_group=per_group)
    g = op.backward(dh, dr, r, y, **params)
    eps32 = float(np.float32(eps))                  # what the library is given
    ref = orc.Residual(NORMS[norm], eps32, NORMS[post], eps32, per_group=per_group or 1)
    args = [np64(t) for t in (dh, dr, r, y)], {k: np64(t) for k, t in params.items()}
    want, _ = ref.backward(*args[0], **args[1])
    limits = bounds.residual_backward(ref, *args[0], **args[1])
    got = {n: np64(t) for n, t in g._asdict().items() if t is not None}
    assert set(got) == set(limits)
    assert not bounds.beyond(got, want, limits, step_of(res), step_of(branch))


@pytest.mark.parametrize("size", (1e-12, 1e12, 1e15, 1e17))
@pytest.mark.parametrize("norm,post", [("layer", "none"), ("rms", "none"), ("layer", "rms"), ("rms", "layer")])
@pytest.mark.parametrize("T,C,res,branch", [(7, 1024, FP32, FP32), (7, 1024, FP32, BF16), (30, 200, FP32, FP32), (5, 301, FP32, BF16), (3, 4100, FP32, FP32)])
def test_rows_of_large_and_of_small_values(T, C, res, branch, norm, post, size):
    """The gradient through the norm of a row is as large as 1 / its deviation, whatever that is.  (The sum of a row's squares is within 32
    bits: 4100 times 1e34.)"""
    gen = torch.Generator(device="cuda").manual_seed(3)
    normal = lambda dtype, scale=1.0: (scale * torch.randn(T, C, generator=gen, device="cuda")).to(dtype)
    eps = 1e-5 if size > 1 else 1e-30
    r, y, dh = normal(res, size), normal(branch, size), normal(branch)
    check(T, C, res, branch, norm, post, eps, r, y, None, dh)                       # nothing beside it
    check(T, C, res, branch, norm, post, eps, r, y, normal(res, 1 / size), dh)


@pytest.mark.parametrize("eps", (1e-5, 1e-27, 1e-37))
@pytest.mark.parametrize("norm,post", [("layer", "none"), ("rms", "none"), ("layer", "rms"), ("rms", "layer"), ("none", "rms")])
@pytest.mark.parametrize("T,C,per_group", [(1, 1024, None), (7, 64, None), (301, 520, None), (9, 1024, 3), (1300, 512, 1), (3, 8192, None), (5, 1001, None)])
def test_a_tiny_eps_and_rows_that_fill_up_a_batch(T, C, per_group, norm, post, eps):
    """Ordinary rows behind an eps that only rows of zeros would notice: those that the kernel puts in where a segment or a group ends
    inside its batch must add nothing to the sums, however small eps is."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    r, y, dr, dh = (torch.randn(T, C, generator=gen, device="cuda") for _ in range(4))
    check(T, C, FP32, FP32, norm, post, eps, r, y, dr, None if norm == "none" else dh, per_group)


@pytest.mark.parametrize("norm,post", [("layer", "none"), ("rms", "none"), ("layer", "rms"), ("rms", "layer")])
@pytest.mark.parametrize("T,C,types", [(6, 1024, (FP32, FP32)), (5, 1024, (FP32, BF16)), (4, 1001, (FP32, FP32)), (9, 128, (BF16, BF16))])
def test_rows_of_zeros_behind_a_tiny_eps(T, C, types, norm, post):
    """Their gradient is 1 / sqrt(eps) times what comes in (less its mean); nothing comes of the product with the row itself."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    r, dr = (torch.randn(T, C, generator=gen, device="cuda").to(types[0]) for _ in range(2))
    y, dh = (torch.randn(T, C, generator=gen, device="cuda").to(types[1]) for _ in range(2))
    r[1], y[2], r[3], y[3] = 0, 0, 0, 0
    check(T, C, *types, norm, post, 1e-30, r, y, dr, dh)
