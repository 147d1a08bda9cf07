"""How far 32-bit arithmetic may be from the statements of block_oracle.py, element by element, from the sizes that the rows
themselves have: no largest value of an array stands in for its values, so that a lost row or term is not within a bound.

U = 2^-24 is the largest relative error of one operation.  Counted to first order in U:
  a sum over a row's channels    at most 16 terms in a row in a thread, five steps over its warp's lanes and 16 warps: with the errors of
                                 the terms themselves fewer than ROW = 70 errors of the sum of absolute terms
  a sum over tokens              rows of a segment, then a 32nd part of the segments, then five steps: CHAIN = 140 for up to 4000 tokens
                                 (thread blocks take at least one and, at that many tokens, at most 28 rows each)
  a sum over a group's tokens    rows of a segment, then the group's segments one behind the other, which are no more together than the
                                 group has tokens and one, and the factors behind them: its tokens and 8
A result is rounded to its type once, by at most half a step of its value (`half_step`), or of the type's smallest value.
"""

import numpy as np

from . import block_oracle as orc

U = 2.0 ** -24
ROW, CHAIN = 70, 140

mean = lambda t: t.mean(-1, keepdims=True)
rms = lambda t: np.sqrt(mean(t * t))


class Standard:
    """Standardised values ``xhat`` of rows, their reciprocal deviation, and what each may be off by."""

    def __init__(self, x, norm, eps):
        x = np.asarray(x, np.float64)
        self.norm = norm
        self.xhat, self.rstd = orc.standardise(x, norm, eps)
        if norm == orc.NONE:
            self.err, self.rel = np.zeros_like(x), np.zeros_like(self.rstd)
            return
        off = ROW * U * mean(np.abs(x)) if norm == orc.LAYER else np.zeros_like(self.rstd)      # of the mean
        c = np.abs(x - mean(x)) if norm == orc.LAYER else np.abs(x)
        self.apart = off + U * c                                                                # of the values less the mean
        variance = 2 * rms(c) * off + off ** 2 + (ROW + 3) * U * mean(c * c)
        self.rel = variance * self.rstd ** 2 / 2 + 4 * U                                        # of rstd, relative
        self.err = self.rstd * self.apart * (1 + self.rel) + np.abs(self.xhat) * (self.rel + U)

    def back(self, g, g_err):
        """-> what the gradient of the values may be off by, from the gradient g of the standardised ones, off by g_err."""
        if self.norm == orc.NONE:
            return g_err
        xhat, a = np.abs(self.xhat), np.abs(g)
        m, m_err = mean(g * self.xhat), ROW * U * mean(a * xhat) + mean(g_err * xhat + a * self.err)
        m_err = m_err + np.abs(m) * (self.rel + 3 * U)
        s, s_err = (mean(g), ROW * U * mean(a) + mean(g_err)) if self.norm == orc.LAYER else (0.0, 0.0)
        u = g - s - self.xhat * m
        u_err = g_err + s_err + xhat * m_err + np.abs(m) * self.err + 4 * U * (a + np.abs(s) + xhat * np.abs(m))
        return self.rstd * u_err + self.rstd * np.abs(u) * (self.rel + 2 * U)


def residual_forward(op, x, y, weight=None, bias=None, gate=None, post_weight=None, post_bias=None):
    """-> what r and h of ``op`` (block_oracle.Residual) may be off by in front of their rounding."""
    n = x.shape[0]
    rows = lambda t, fallback: np.abs(op.rows(t, n, fallback))
    r = op.forward(x, y, weight, bias, gate, post_weight, post_bias)[0]
    sy = Standard(y, op.post, op.post_eps)
    g, pw, pb = rows(gate, 1.0), rows(post_weight, 1.0), rows(post_bias, 0.0)
    r_err = g * (pw * sy.err + 5 * U * (pw * np.abs(sy.xhat) + pb)) + U * np.abs(op.scale * np.asarray(x, np.float64)) + U * np.abs(r)
    if op.norm == orc.NONE:
        return {"r": r_err}
    st = Standard(r, op.norm, op.eps)
    moved = st.rstd * (r_err + (mean(r_err) if op.norm == orc.LAYER else 0.0) + np.abs(st.xhat) * mean(r_err * np.abs(st.xhat)))
    a = np.abs(op.factor(weight, n))
    return {"r": r_err, "h": a * (st.err + moved) + 4 * U * (a * np.abs(st.xhat) + rows(bias, 0.0))}


def residual_backward(op, dh, dr, r, y, weight=None, bias=None, gate=None, post_weight=None, post_bias=None):
    """-> of each gradient that ``op`` (block_oracle.Residual) gives: {name: what it may be off by in front of its rounding}."""
    n = (dr if dr is not None else r).shape[0]
    bounds = {}
    per_token = lambda t, fallback: np.abs(op.rows(t, n, fallback))

    def summed(terms, errors, like):
        chain = CHAIN if like.ndim == 1 else min(op.per_group, n) + 8
        return op.summed(errors, like) + chain * U * op.summed(np.abs(terms), like)

    d, d_err = (0.0, 0.0) if dr is None else (np.asarray(dr, np.float64), 0.0)
    if dh is not None:
        dh = np.asarray(dh, np.float64)
        st = Standard(r, op.norm, op.eps)
        if weight is not None:
            bounds["weight"] = summed(dh * st.xhat, np.abs(dh) * st.err, np.asarray(weight))
        if bias is not None:
            bounds["bias"] = summed(dh, np.zeros_like(dh), np.asarray(bias))
        g = dh * op.factor(weight, n)
        through = orc.standardise_back(g, st.xhat, st.rstd, op.norm)
        d_err = st.back(g, 2 * U * np.abs(g)) + U * (np.abs(through) + np.abs(d))
        d = d + through
    bounds["dx"] = np.abs(op.scale) * (d_err + 2 * U * np.abs(d))
    if y is None:
        return bounds
    sy = Standard(y, op.post, op.post_eps)
    a, yhat = np.abs(d), np.abs(sy.xhat)
    s_err, n_err = d_err * yhat + a * sy.err + U * a * yhat, d_err + U * a          # of the terms of the two sums
    pw, pb = (np.abs(op.rows(t, n, f)) for t, f in ((post_weight, 1.0), (post_bias, 0.0)))
    if gate is not None:
        like = np.asarray(gate)
        bounds["gate"] = summed(d * sy.xhat * pw, s_err * pw + 3 * U * a * yhat * pw, like) + summed(d * pb, n_err * pb + 3 * U * a * pb, like)
    g = per_token(gate, 1.0)
    if post_weight is not None:
        bounds["post_weight"] = summed(d * sy.xhat * g, s_err * g + 3 * U * a * yhat * g, np.asarray(post_weight))
    if post_bias is not None:
        bounds["post_bias"] = summed(d * g, n_err * g + 3 * U * a * g, np.asarray(post_bias))
    e = d * op.rows(gate, n, 1.0) * op.rows(post_weight, n, 1.0)
    bounds["dy"] = sy.back(e, d_err * g * pw + 3 * U * np.abs(e))
    return bounds


def rotary_backward(op, dout, x, positions, weight=None):
    """-> what dx, dweight and dbias of ``op`` (block_oracle.Rotary) may be off by; dx in front of its rounding.  A cosine or sine is off by
    fewer than 4 U: the last bit of an angle in half turns (pi 2^-25) and the function's own two."""
    dout = np.asarray(dout, np.float64)
    size = np.abs(dout)
    for a, b, _, _ in op.layout():
        size[..., a] = size[..., b] = np.abs(dout[..., a]) + np.abs(dout[..., b])
    e, e_err = op.turn(dout, positions, back=True), 8 * U * size
    if op.norm == orc.NONE:
        return e_err, None, None
    st = Standard(x, op.norm, op.eps)
    w = 1.0 if weight is None else np.asarray(weight, np.float64)
    summed = lambda terms, errors: errors.sum((0, 1)) + CHAIN * U * np.abs(terms).sum((0, 1))
    dx = st.back(e * w, e_err * np.abs(w) + U * np.abs(e * w))
    return dx, summed(e * st.xhat, e_err * np.abs(st.xhat) + np.abs(e) * st.err), summed(e, e_err)


def half_step(want, step, smallest):
    """What rounding to a type of that step (eps) and smallest value may move a value by."""
    return step / 2 * np.abs(want) * (1 + 2.0 ** -8) + smallest


def beyond(got, want, bounds, residual=(0.0, 0.0), branch=(0.0, 0.0)):
    """-> {name: largest error / bound} of the results whose error passes its bound somewhere, or is not a number.  got, want: {name:
    array}; residual, branch: (eps, smallest value) of the types of r and dx and of h and dy."""
    out = {}
    for name, bound in bounds.items():
        step = residual if name in ("r", "dx") else branch if name in ("h", "dy") else (0.0, 2.0 ** -150)
        with np.errstate(over="ignore"):
            ratio = np.abs(got[name] - want[name]) / (bound + half_step(want[name], *step))
        if not (ratio <= 1).all():
            out[name] = float(ratio.max())
    return out
