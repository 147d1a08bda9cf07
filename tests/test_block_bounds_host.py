"""The bounds that the residual stream and its gradients are held to on the GPU, tried on the CPU: exact gradients, rounded as the library rounds
them, pass, and results with a mistake that a kernel can make do not, at the sizes where they are used."""

import dataclasses

import numpy as np
import pytest

from oracle import block_bounds as bounds
from oracle import block_oracle as orc

BF16 = (2.0 ** -7, 2.0 ** -134)
FP32 = (0.0, 2.0 ** -150)


def bf16(x):
    """To nearest even."""
    bits = np.asarray(x, np.float32).view(np.uint32)
    return ((bits + 0x7fff + ((bits >> 16) & 1)) & np.uint32(0xffff0000)).view(np.float32).astype(np.float64)


class Case:
    """bf16 rows; parameters of every kind that the norms allow, one row or one for each group."""

    def __init__(self, T, C, norm, post, per_group):
        rng = np.random.default_rng(T + C)
        normal = lambda *s: rng.standard_normal(s)
        self.op = orc.Residual(norm, 1e-5, post, 1e-5, 1.0, per_group is not None, per_group or 1)
        rows = (C,) if per_group is None else (-(-T // per_group), C)
        self.params = dict(weight=normal(*rows) if norm else None, bias=normal(*rows) if norm else None, gate=normal(*rows),
                           post_weight=1 + 0.2 * normal(C) if post else None, post_bias=0.2 * normal(C) if post else None)
        self.dh, self.dr, self.r, self.y = (bf16(normal(T, C)) for _ in range(4))
        if not norm:
            self.dh = None
        self.limits = bounds.residual_backward(self.op, self.dh, self.dr, self.r, self.y, **self.params)
        self.want = self.gradients()

    def gradients(self, op=None, rows=None):
        s = slice(None) if rows is None else rows
        dh = None if self.dh is None else self.dh[s]
        return (op or self.op).backward(dh, self.dr[s], self.r[s], self.y[s], **self.params)[0]

    def rejected(self, got):
        """The names whose error is beyond its bound."""
        got = {n: bf16(t) if n in ("dx", "dy") else np.float32(t).astype(np.float64) for n, t in got.items()}
        return set(bounds.beyond(got, self.want, self.limits, BF16, BF16))


SIZES = [(900, 1024, 1, 1, 300), (1500, 400, 1, 0, 500), (400, 1024, 2, 1, 1), (300, 1024, 1, 1, None), (50, 512, 1, 1, None), (2000, 500, 1, 0, None),
         (1374, 1024, 1, 0, None), (700, 250, 1, 0, None), (700, 2056, 1, 2, None), (30, 8192, 1, 1, None), (9, 4100, 2, 0, None), (26, 96, 0, 2, 5)]


@pytest.mark.parametrize("T,C,norm,post,per_group", SIZES)
def test_mistakes_are_beyond_the_bounds(T, C, norm, post, per_group, monkeypatch):
    case = Case(T, C, norm, post, per_group)
    assert not case.rejected(case.want)
    sums = [n for n in case.want if n not in ("dx", "dy")]
    every = set(case.want)
    assert case.rejected({n: 0.9 * t for n, t in case.want.items()}) == every
    assert case.rejected({n: np.zeros_like(t) for n, t in case.want.items()}) == every
    # the last token left out of the sums, and of the rows
    lost = case.gradients(rows=slice(0, T - 1))
    assert case.rejected({**case.want, **{n: lost[n] for n in sums}}) == set(sums)
    got = {**case.want, "dx": case.want["dx"].copy(), "dy": case.want["dy"].copy()}
    got["dx"][-1], got["dy"][-1] = got["dx"][0], got["dy"][0]
    assert case.rejected(got) == {"dx", "dy"}
    # a term of the norm's gradient left out: of the one in front of the next branch, and of the one behind the last
    back = orc.standardise_back
    parts = {"projection": lambda g, xhat, rstd, kind: g * rstd if kind == orc.RMS else (g - g.mean(-1, keepdims=True)) * rstd,
             "mean": lambda g, xhat, rstd, kind: (g - xhat * (g * xhat).mean(-1, keepdims=True)) * rstd}
    for part, wrong in parts.items():
        for which, kind, name in (("r", norm, "dx"), ("y", post, "dy")):
            if kind == orc.NONE or (part == "mean" and kind != orc.LAYER):
                continue
            of = bounds.Standard(case.r if which == "r" else case.y, kind, 1e-5).rstd
            monkeypatch.setattr(orc, "standardise_back", lambda g, xhat, rstd, k: (wrong if k == kind and np.array_equal(rstd, of) else back)(g, xhat, rstd, k))
            got = case.gradients()
            monkeypatch.setattr(orc, "standardise_back", back)
            assert name in case.rejected(got), (part, which)


@pytest.mark.parametrize("T,C,norm,post,per_group", SIZES)
def test_mistakes_of_the_forward_call_are_beyond_the_bounds(T, C, norm, post, per_group):
    case = Case(T, C, norm, post, per_group)
    x, y, op = case.r, case.y, case.op
    want = dict(zip("rh", op.forward(x, y, **case.params)))
    limits = bounds.residual_forward(op, x, y, **case.params)
    want = {n: want[n] for n in limits}
    rejected = lambda got: set(bounds.beyond({n: bf16(t) for n, t in got.items()}, want, limits, BF16, BF16))
    assert not rejected(want)
    assert rejected({n: 0.99 * t for n, t in want.items()}) == set(want)
    for wrong in (dict(norm=3 - norm), dict(post=3 - post), dict(scale=0.99), dict(post_eps=1e-2)):
        if wrong.get("norm") == 3 or not post and ("post" in wrong or "post_eps" in wrong):
            continue
        got = dict(zip("rh", dataclasses.replace(op, **wrong).forward(x, y, **case.params)))
        # 1e-2 beside a variance of about 1 moves a value by 5e-3 of it, more than half a step of the type
        names = {"h"} if "norm" in wrong else set(want) if "post" in wrong else {"r"}
        assert rejected({n: got[n] for n in want}) >= names, wrong
    for name in case.params:
        if case.params[name] is not None:
            short = {**case.params, name: np.roll(case.params[name], 1, -1)}
            assert rejected({n: t for n, t in zip("rh", op.forward(x, y, **short)) if n in want}) >= ({"h"} if name in ("weight", "bias") else {"r"}), name


def test_bounds_hold_for_the_formulas_in_32_bits():
    """The formulas in 32-bit numpy, sums in any order, are within them."""
    f32 = np.float32
    for norm, post in ((1, 0), (2, 1), (1, 2)):
        case = Case(60, 640, norm, post, None)
        p = {n: None if t is None else f32(t) for n, t in case.params.items()}
        case.params = {n: None if t is None else t.astype(np.float64) for n, t in p.items()}
        case.limits, case.want = bounds.residual_backward(case.op, case.dh, case.dr, case.r, case.y, **case.params), case.gradients()
        mean = lambda t: t.mean(-1, keepdims=True, dtype=f32)

        def standard(x, kind):
            x = f32(x)
            x = x - mean(x) if kind == orc.LAYER else x
            rstd = 1 / np.sqrt(mean(x * x) + f32(1e-5))
            return x * rstd, rstd

        def back(g, xhat, rstd, kind):
            out = g - xhat * mean(g * xhat)
            return (out - mean(g) if kind == orc.LAYER else out) * rstd

        dh, dr = f32(case.dh), f32(case.dr)
        xhat, rstd = standard(case.r, norm)
        d = dr + back(dh * p["weight"], xhat, rstd, norm)
        got = dict(weight=(dh * xhat).sum(0), bias=dh.sum(0), dx=d)
        y, y_rstd = standard(case.y, post) if post else (f32(case.y), None)
        e = d * p["gate"]
        got["gate"] = (d * (y * p["post_weight"] + p["post_bias"] if post else y)).sum(0)
        if post:
            got["post_weight"], got["post_bias"] = (e * y).sum(0), e.sum(0)
            e = back(e * p["post_weight"], y, y_rstd, post)
        got["dy"] = e
        assert not bounds.beyond({n: t.astype(np.float64) for n, t in got.items()}, case.want, case.limits, FP32, FP32)
