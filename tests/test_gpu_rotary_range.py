"""Gradients through the norm of the heads over the range of 32 bits: large and small values, heads of zeros behind a tiny eps, on the GPU
against the fp64 statement within bounds made of the heads' own sizes (``block_bounds``)."""

import numpy as np
import pytest
import torch

import paper_2512_02541_b200 as P
from oracle import block_bounds as bounds
from oracle import block_oracle as orc

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
NORMS = {"layer": P.AVGGT_NORM_LAYER, "rms": P.AVGGT_NORM_RMS}


def np64(t):
    return t.detach().double().cpu().numpy()


def check(T, heads, d, pairs, dtype, norm, eps, size, zeros=False, adjacent=False):
    gen = torch.Generator(device="cuda").manual_seed(2)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda")
    q, dq = (size * normal(T, heads, d)).to(dtype), normal(T, heads, d).to(dtype)
    if zeros:
        q[1], q[:, 1] = 0, 0
    w, b = 1 + 0.3 * normal(d), 0.2 * normal(d)
    pos = torch.randint(-40, 1400, (T, len(pairs)), generator=gen, device="cuda", dtype=torch.int32)
    g = P.AxialRotary(d, pairs, adjacent=adjacent, norm=NORMS[norm], eps=eps).backward(dq, None, pos, q=q, q_weight=w, q_bias=b)
    ref = orc.Rotary(d, pairs, adjacent=adjacent, norm=NORMS[norm], eps=float(np.float32(eps)))
    args = np64(dq), np64(q), pos.cpu().numpy(), np64(w)
    want, limits = ref.backward(*args)[:3], bounds.rotary_backward(ref, *args)
    info = torch.finfo(dtype)
    limits = {"dx": limits[0], "weight": limits[1], "bias": limits[2]}
    got = {"dx": np64(g.dq), "weight": np64(g.q_weight), "bias": np64(g.q_bias)}
    assert not bounds.beyond(got, dict(zip(limits, want)), limits, (0.0 if dtype is FP32 else info.eps, info.tiny * info.eps / 2))


SHAPES = [(7, 5, 64, (16, 16)), (30, 3, 72, (18, 18)), (9, 16, 128, (16, 24, 24)), (40, 2, 100, (7, 11, 13)), (64, 2, 16, (4, 4))]


@pytest.mark.parametrize("size", (1e-12, 1.0, 1e12, 1e15, 1e17))
@pytest.mark.parametrize("norm", ("layer", "rms"))
@pytest.mark.parametrize("dtype", (FP32, BF16))
@pytest.mark.parametrize("shape", SHAPES)
def test_heads_of_large_and_of_small_values(shape, dtype, norm, size):
    """The gradient through the norm of a head is as large as 1 / its deviation, whatever that is."""
    check(*shape, dtype, norm, 1e-5 if size >= 1 else 1e-30, size)


@pytest.mark.parametrize("eps", (1e-5, 1e-27, 1e-37))
@pytest.mark.parametrize("norm", ("layer", "rms"))
@pytest.mark.parametrize("adjacent", (False, True))
@pytest.mark.parametrize("shape", SHAPES)
def test_heads_of_zeros_behind_a_tiny_eps(shape, adjacent, norm, eps):
    """Their gradient is 1 / sqrt(eps) times what comes in (less its mean); nothing comes of the product with the head itself."""
    check(*shape, FP32, norm, eps, 1.0, zeros=True, adjacent=adjacent)
