"""The operators around the attention, called from several host threads at once, each on a stream of its own.  Arguments are packed once,
so that the threads are inside the library most of the time, where the interpreter lets them run side by side."""

import threading

import pytest
import torch

import paper_2512_02541_b200 as P
from paper_2512_02541_b200 import binding as B

pytestmark = pytest.mark.gpu

CALLS = 20000


def at_once(name, calls):
    """Calls the entry point ``name`` CALLS times with each list of arguments, each in a thread of its own, from a common start -> how many
    calls of each thread returned an error."""
    f, barrier, errors = B.packed_entry(name), threading.Barrier(len(calls)), [None] * len(calls)
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()

    def run(i):
        args = (*calls[i], streams[i].cuda_stream)
        f(*args)
        barrier.wait()
        errors[i] = sum(1 for _ in range(CALLS) if f(*args) != 0)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    return errors


def rows(t):
    return B.PACKED_ROWS.pack(t.data_ptr(), t.stride(0))


@pytest.mark.parametrize("sizes", [(1280, 2048), (2048, 1280, 1536, 1030), (4096, 2304, 4096, 2304)])
def test_forward_calls_of_one_kernel_with_different_shared_memory(sizes):
    """1,280 and 2,048 channels of 32 bits run the same kernel with pipelines of 64 and 96 KB."""
    calls, outputs = [], []
    for C in sizes:
        gen = torch.Generator(device="cuda").manual_seed(C)
        x, y, r, h = (torch.randn(4, C, generator=gen, device="cuda") for _ in range(4))
        params = B.PACKED_RESIDUAL.pack(4, 1, C, P.AVGGT_TYPE_FP32, P.AVGGT_TYPE_FP32, P.AVGGT_NORM_LAYER, P.AVGGT_NORM_NONE, 1e-5, 1e-5, 1.0, 0)
        calls.append((params, rows(x), rows(y), None, None, None, None, None, rows(r), rows(h)))
        outputs.append((x, y, (r, h), P.ResidualNorm(C)(x, y)))
    assert at_once("avggt_residual_norm", calls) == [0] * len(sizes)
    for _, _, got, want in outputs:
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("post", (P.AVGGT_NORM_NONE, P.AVGGT_NORM_RMS))
@pytest.mark.parametrize("sizes", [(1032, 2048), (2304, 4096, 2304, 4096)])
def test_backward_calls_of_one_kernel_with_different_shared_memory(sizes, post):
    """Pipelines of different depth, and behind a post norm the sums of 1,500 groups, which three groups do not need."""
    calls, outputs = [], []
    for i, C in enumerate(sizes):
        gen = torch.Generator(device="cuda").manual_seed(C)
        normal = lambda *s: torch.randn(s, generator=gen, device="cuda")
        T = 1500                                    # more groups than a wave of blocks, so that blocks take whole groups
        r, dr, dx = (normal(T, C) for _ in range(3))
        y, dh, dy = (normal(T, C).bfloat16() for _ in range(3))
        T = 3 if i % 2 else T
        r, dr, dx, y, dh, dy = (t[:T] for t in (r, dr, dx, y, dh, dy))
        gate, pw = normal(T, C), normal(C) if post else None
        op = P.ResidualNorm(C, post_norm=post, tokens_per_group=1)
        g = op.backward(dh, dr, r, y, gate=gate, post_weight=pw)
        fields = (T, 1, C, P.AVGGT_TYPE_FP32, P.AVGGT_TYPE_BF16, P.AVGGT_NORM_LAYER, post, 1e-5, 1e-5, 1.0, P.AVGGT_RESIDUAL_GATE_GROUPED)
        ws = torch.empty(P.avggt_residual_workspace_bytes(P.AvggtResidualParams(*fields)), dtype=torch.uint8, device="cuda")
        dgate, dpw = torch.empty_like(gate), torch.empty_like(pw) if post else None
        calls.append((B.PACKED_RESIDUAL.pack(*fields), rows(dh), rows(dr), rows(r), rows(y), None, gate.data_ptr(), pw.data_ptr() if post else None,
                      None, rows(dx), rows(dy), None, None, dgate.data_ptr(), dpw.data_ptr() if post else None, None, ws.data_ptr(), ws.numel()))
        outputs.append(((r, dr, y, dh, ws, gate, pw), (dx, dy, dgate) + ((dpw,) if post else ()), (g.dx, g.dy, g.gate, g.post_weight)))
    assert at_once("avggt_residual_norm_backward", calls) == [0] * len(sizes)
    for _, got, want in outputs:
        assert all(torch.equal(a, b) for a, b in zip(got, want))
