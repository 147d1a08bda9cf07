"""The C ABI's calls of the operators around the attention by their plain bindings: the same bits as the classes give; and calls that are a
process's first ones, made while a graph is captured."""

import subprocess
import sys

import pytest
import torch

import paper_2512_02541_b200 as P

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32


def normal(*shape, dtype=FP32, seed=0):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def test_rotary():
    T, hq, hk, d = 130, 5, 2, 64
    fused = normal(T, hq + 2 * hk, d, dtype=BF16)
    q, k, v = fused[:, :hq], fused[:, hq:hq + hk], fused[:, hq + hk:]
    w, b = normal(d, seed=1), normal(d, seed=2)
    pos = torch.arange(2 * T, device="cuda", dtype=torch.int32).view(T, 2)
    rot = P.AxialRotary(d, (16, 16), norm=P.AVGGT_NORM_LAYER)
    params = rot.params(T, hq, hk, BF16)
    want = rot(q, k, pos, v=v, q_weight=w, q_bias=b, k_weight=b)
    got = [torch.empty_like(t) for t in want]
    P.avggt_rotary(params, pos, q, k, v, w, b, b, None, *got)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    dq, dk, dv = (normal(*t.shape, dtype=BF16, seed=3 + i) for i, t in enumerate(want))
    g = rot.backward(dq, dk, pos, q=q, k=k, dv=dv, q_weight=w, q_bias=b, k_weight=b)
    out, sums = [torch.empty_like(t) for t in want], [torch.empty_like(w) for _ in range(3)]
    ws = torch.empty(P.avggt_rotary_workspace_bytes(params), dtype=torch.uint8, device="cuda")
    P.avggt_rotary_backward(params, pos, dq, dk, dv, q, k, w, b, *out, *sums, None, ws, ws.numel())
    assert all(torch.equal(x, y) for x, y in zip((*out, *sums), g))


def test_residual_norm():
    T, C = 70, 768
    x, y, w, gate, pw = normal(T, C), normal(T, C, dtype=BF16, seed=1), normal(C, seed=2), normal(C, seed=3), normal(C, seed=4)
    op = P.ResidualNorm(C, norm=P.AVGGT_NORM_RMS, post_norm=P.AVGGT_NORM_LAYER, residual_scale=0.5)
    params = P.AvggtResidualParams(T, 1, C, P.AVGGT_TYPE_FP32, P.AVGGT_TYPE_BF16, P.AVGGT_NORM_RMS, P.AVGGT_NORM_LAYER, 1e-5, 1e-5, 0.5, 0)
    want = op(x, y, weight=w, gate=gate, post_weight=pw)
    r, h = torch.empty_like(x), torch.empty_like(y)
    P.avggt_residual_norm(params, x, y, w, None, gate, pw, None, r, h)
    assert torch.equal(r, want[0]) and torch.equal(h, want[1])
    dh, dr = normal(T, C, dtype=BF16, seed=5), normal(T, C, seed=6)
    g = op.backward(dh, dr, r, y, weight=w, gate=gate, post_weight=pw)
    dx, dy, dw, dgate, dpw = torch.empty_like(r), torch.empty_like(y), *(torch.empty_like(w) for _ in range(3))
    ws = torch.empty(P.avggt_residual_workspace_bytes(params), dtype=torch.uint8, device="cuda")
    P.avggt_residual_norm_backward(params, dh, dr, r, y, w, gate, pw, None, dx, dy, dw, None, dgate, dpw, None, ws, ws.numel())
    assert all(torch.equal(a, b) for a, b in zip((dx, dy, dw, dgate, dpw), (g.dx, g.dy, g.weight, g.gate, g.post_weight)))


FIRST = """
import torch
import paper_2512_02541_b200 as P
x, y = torch.randn(9, 2048, device="cuda"), torch.randn(9, 2048, device="cuda")
w, pos = torch.ones(2048, device="cuda"), torch.arange(18, device="cuda", dtype=torch.int32).view(9, 2)
res, rot = P.ResidualNorm(2048), P.AxialRotary(64, (16, 16), norm=P.AVGGT_NORM_RMS)
heads, one = x.view(9, 32, 64), torch.ones(64, device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
def run():
    r, h = res(x, y, weight=w)
    g = res.backward(h, r, r, y, weight=w)
    Q, K, _ = rot(heads, None, pos, q_weight=one)
    return [r, h, *g[:3], Q, *rot.backward(Q, None, pos, q=heads, q_weight=one)[:4:3]]
with torch.cuda.graph(graph):
    got = run()
graph.replay()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, run()))
print("same")
"""


def test_first_calls_of_a_process_are_captured():
    """Kernels are loaded, and their shared memory is allowed, while the capture goes on."""
    done = subprocess.run([sys.executable, "-c", FIRST], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "same" in done.stdout, done.stderr[-2000:]
