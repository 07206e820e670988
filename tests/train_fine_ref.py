"""Bounds of the gated block's arithmetic that count what h, dg and du lose on their
way and no more: fp16 gradients go on times powers of two, and up to 16 rows every
number goes on as two."""
import math

import torch

from tests import train_ref as R

TWO_ROWS = 16


def _norms(t):
    return float(t.double().square().sum(1).max().sqrt()) if t.numel() else 0.0


def _most(t):
    return 0.0 if t is None else float(t.double().abs().max())


def largest(dy, x, w, b, name):
    """What |dg| and |du|, and |h|, cannot exceed: the sizes of rows and weights by the
    Cauchy-Schwarz inequality, |act'| <= 1.13, |act(g)| <= |g| or 1."""
    dh = _norms(dy) * math.sqrt(float(w[2].double().abs().amax(1).square().sum()))
    u = _norms(x) * _norms(w[1]) + _most(b[1])
    a = 1.0 if name == "sigmoid" else _norms(x) * _norms(w[0]) + _most(b[0])
    return dh * max(1.13 * u, a), a * u


def floor_of(most, kind):
    """The step of the smallest numbers: the type's own, over the power of two that
    brings `most` above half of 62384 (and never below 1)."""
    tiny = R.TINY[kind]
    return min(tiny, tiny * 2.01 * most / 62384.0) if kind == torch.float16 else tiny


def kept(v, bound, kind, floor, two):
    """The bound of a number that goes on in 16 bits, or in two such numbers, the second
    of which is what rounding left of the first."""
    step = R.HALF_STEP[kind]
    return bound + (step * step if two else step) * (v.abs() + bound) + floor


def gated(x, w, b, name, two=None):
    kind = x.dtype
    two = x.shape[0] <= TWO_ROWS if two is None else two
    g, u, eu, a, e_a, _, _ = R._front(x, w, b, name)
    h = a * u
    eh = kept(h, a.abs() * eu + u.abs() * e_a + e_a * eu + 2 * R.U * h.abs(), kind, R.TINY[kind],
              two)
    wd = w[2].double()
    y = h @ wd.t()
    e = eh @ wd.abs().t() + (2 * h.shape[1] + 2) * 2 * R.U * ((h.abs() + eh) @ wd.abs().t())
    if b[2] is not None:
        y = y + b[2].double()
        e = e + 2 * R.U * b[2].double().abs()
    return y, e


def gated_backward(dy, x, w, b, name, two=None):
    """(value, bound) of dx, dw_gate, dw_up and dw_down."""
    kind = x.dtype
    two = x.shape[0] <= TWO_ROWS if two is None else two
    top_grad, top_h = largest(dy, x, w, b, name)
    g, u, eu, a, e_a, slope, e_s = R._front(x, w, b, name)
    x, dy = x.double(), dy.double()
    wg, wu, wd = (v.double() for v in w)
    m, hid = g.shape
    h = a * u
    eh = kept(h, a.abs() * eu + u.abs() * e_a + e_a * eu + 2 * R.U * h.abs(), kind,
              floor_of(top_h, kind), two)
    dh = dy @ wd
    edh = (dy.shape[1] + 2) * 2 * R.U * (dy.abs() @ wd.abs())
    dh_ = dh.abs() + edh
    dg, du = dh * u * slope, dh * a
    at = floor_of(top_grad, kind)
    edg = kept(dg, edh * (u * slope).abs() + dh_ * (slope.abs() * eu + (u.abs() + eu) * e_s) +
               4 * R.U * dg.abs(), kind, at, two)
    edu = kept(du, edh * a.abs() + dh_ * e_a + 4 * R.U * du.abs(), kind, at, two)
    size = (dg.abs() + edg) @ wg.abs() + (du.abs() + edu) @ wu.abs()
    out = [(dg @ wg + du @ wu,
            edg @ wg.abs() + edu @ wu.abs() + (4 * hid + 2) * 2 * R.U * size)]
    for left, el, right, er in ((dg, edg, x, 0 * x), (du, edu, x, 0 * x), (dy, 0 * dy, h, eh)):
        e = el.t() @ (right.abs() + er) + left.abs().t() @ er
        out.append((left.t() @ right,
                    e + (2 * m + 2) * 2 * R.U * ((left.abs() + el).t() @ (right.abs() + er))))
    return out


def relative(got, want):
    return float((got.double() - want).norm() / want.norm())


def share(want, kind, two):
    """The relative error, over a whole table of random numbers, of what the arithmetic
    allows: rounding the result, and beside it (squares add up) rounding each number on
    its way by up to half a step, 1 / sqrt(3) of that on average.  In two numbers the
    latter is nothing next to the former; fp32 sums leave 1e-5 at most."""
    alone = relative(want.to(kind), want)
    return (1.02 * alone if two else 1.1 * math.hypot(alone, R.HALF_STEP[kind] / math.sqrt(3.0))) + 1e-5
