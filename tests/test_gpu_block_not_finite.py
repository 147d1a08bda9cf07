"""What becomes of infinities and NaN in the operators around the attention, as include/avggt.h has it."""

import pytest
import torch

import paper_2512_02541_b200 as P
import test_gpu_residual as residual
import test_gpu_rotary as rotary

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")
T, C = 41, 1001


def same(a, b):
    return torch.equal(torch.nan_to_num(a, nan=7.0), torch.nan_to_num(b, nan=7.0)) and torch.equal(torch.isnan(a), torch.isnan(b))


@pytest.mark.parametrize("value", (NAN, INF, -INF))
@pytest.mark.parametrize("channels", (64, 1001, 1024, 4100))
@pytest.mark.parametrize("norm", ("none", "layer", "rms"))
def test_residual_stream(norm, channels, value):
    pr = residual.Problem(T, channels, FP32, FP32, norm)
    want = [None if t is None else t.clone() for t in pr.forward()]
    g = pr.backward()
    row, at = 3, channels - 1
    pr.x[row, at] = value
    got, g2 = pr.forward(), pr.backward()
    others = torch.arange(T, device="cuda") != row
    # r: that channel alone
    hit = torch.zeros(channels, dtype=torch.bool, device="cuda")
    hit[at] = True
    assert torch.equal(got[0][others], want[0][others]) and torch.equal(got[0][row, ~hit], want[0][row, ~hit])
    assert not torch.isfinite(got[0][row, at])
    if norm == "none":
        assert got[1] is None and all(same(a, b) for a, b in zip(g, g2) if a is not None)       # gradients do not depend on r
        return
    assert torch.equal(got[1][others], want[1][others])
    if norm == "layer" or value != value:
        assert torch.isnan(got[1][row]).all()
    else:                                           # an infinite deviation
        assert torch.isnan(got[1][row, at]) and torch.equal(got[1][row, ~hit], pr.params["bias"][~hit])
    assert torch.equal(g2.dx[others], g.dx[others]) and torch.equal(g2.dy[others], g.dy[others])
    assert torch.isnan(g2.dx[row]).all() and torch.isnan(g2.dy[row]).all()
    assert torch.isnan(g2.gate).all() and torch.equal(g2.bias, g.bias) and torch.isnan(g2.weight[at])
    if norm == "rms" and value == value:
        assert torch.isfinite(g2.weight[~hit]).all()
    else:
        assert torch.isnan(g2.weight).all()


@pytest.mark.parametrize("value", (NAN, INF))
@pytest.mark.parametrize("post", ("layer", "rms"))
def test_branch(post, value):
    pr = residual.Problem(T, C, FP32, BF16, post=post)
    want, g = [t.clone() for t in pr.forward()], pr.backward()
    row, at = 7, 500
    pr.y[row, at] = value
    got, g2 = pr.forward(), pr.backward()
    others = torch.arange(T, device="cuda") != row
    assert all(torch.equal(a[others], b[others]) for a, b in zip(got, want))
    assert torch.isnan(got[1][row]).all() and torch.isnan(got[0][row, at])
    hit = torch.arange(C, device="cuda") == at
    if post == "layer" or value != value:
        assert torch.isnan(got[0][row]).all() and torch.isnan(g2.gate).all()
    else:
        finite = pr.x[row] + pr.params["gate"] * pr.params["post_bias"]
        assert ((got[0][row] - finite)[~hit].abs() <= 2 ** -22 * (1 + finite[~hit].abs() + pr.x[row][~hit].abs())).all()      # two roundings
        assert torch.isfinite(g2.gate[~hit]).all()
    assert torch.equal(g2.dx, g.dx) and torch.equal(g2.weight, g.weight) and torch.equal(g2.dy[others], g.dy[others])
    assert torch.isnan(g2.dy[row]).all() and torch.isnan(g2.gate[at])


def test_squares_beyond_32_bits():
    """As an infinite deviation; just below them the norm is as exact as ever."""
    pr = residual.Problem(4, 8192, FP32, FP32, "rms", gate="none")
    pr.y.zero_()
    pr.x.fill_(2.2e17)
    assert torch.equal(pr.forward()[1], pr.params["bias"].expand(4, 8192))
    pr.x.fill_(1.9e17)
    want = pr.params["weight"].double() + pr.params["bias"].double()
    size = pr.params["weight"].double().abs() + pr.params["bias"].double().abs()
    assert ((pr.forward()[1].double() - want).abs() <= 80 * 2.0 ** -24 * size).all()          # half of 70 of the sum, the root, two products


@pytest.mark.parametrize("value", (NAN, INF, -INF))
@pytest.mark.parametrize("adjacent", (False, True))
@pytest.mark.parametrize("d,pairs", [(64, (16, 16)), (72, (18, 10)), (6, (1, 1))])
@pytest.mark.parametrize("norm", ("none", "layer", "rms"))
def test_heads(norm, d, pairs, adjacent, value):
    pr = rotary.Problem(20, 3, 2, d, pairs, dtype=FP32, norm=norm, adjacent=adjacent)
    (a, b, axis, _), token, head = pr.orc.layout()[1 % len(pairs)], 5, 1
    pr.pos[token] = torch.tensor([3] * len(pairs), device="cuda")
    want, g = pr.forward()[0].clone(), pr.backward()
    pr.q[token, head, a] = value
    got, g2 = pr.forward()[0], pr.backward()
    keep = torch.ones(20, 3, dtype=torch.bool, device="cuda")
    keep[token, head] = False
    assert torch.equal(got[keep], want[keep]) and torch.equal(g2.dk, g.dk)
    assert norm == "none" or torch.equal(g2.k_weight, g.k_weight)
    pair = torch.zeros(d, dtype=torch.bool, device="cuda")
    pair[a] = pair[b] = True
    mine = got[token, head]
    if norm == "layer" or (norm == "rms" and value != value):
        assert torch.isnan(mine).all()
    elif norm == "rms":                             # the turned bias, and NaN in the pair
        zeros = pr.q.clone()
        zeros[token, head] = 0.0
        bias = pr.rot(zeros, pr.k, pr.pos, **pr.params())[0][token, head]
        assert torch.isnan(mine[pair]).all() and torch.equal(mine[~pair], bias[~pair])
    else:
        assert not torch.isfinite(mine[pair]).any() and torch.equal(mine[~pair], want[token, head][~pair])
        assert value != value or torch.isinf(mine[pair]).all()          # neither its cosine nor its sine is 0
        assert torch.equal(g2.dq, g.dq)
        return
    assert torch.equal(g2.dq[keep], g.dq[keep]) and torch.isnan(g2.dq[token, head]).all() and torch.isnan(g2.q_weight[a])
    assert torch.equal(g2.q_bias, g.q_bias)


def test_elements_that_are_not_turned_are_a_pair_too():
    """Without a norm, at position 0 and behind the last block, the element beside an infinity is NaN."""
    pr = rotary.Problem(4, 1, 1, 16, (4, 2), dtype=FP32, norm="none")
    pr.pos.zero_()
    pr.q[0, 0, 0], pr.q[1, 0, 12] = INF, INF
    Q = pr.forward()[0]
    for token, at, beside in ((0, 0, 4), (1, 12, 14)):
        assert torch.isinf(Q[token, 0, at]) and torch.isnan(Q[token, 0, beside])
        rest = [i for i in range(16) if i not in (at, beside)]
        assert torch.equal(Q[token, 0, rest], pr.q[token, 0, rest])
