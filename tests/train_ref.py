"""Plain 64-bit forms of the training operators, with the error bounds of the
kernels' arithmetic (shared by their tests).

u = 2^-24 is half a step of fp32.  A sum of n fp32 numbers in any order is off by
at most n u times the sum of their absolute values; where a kernel adds in a tree,
its depth stands for n."""
import math

import torch

U = 2.0 ** -24
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def stored(y, bound, kind):
    """The bound after the one rounding to the output type."""
    return bound + HALF_STEP[kind] * (y.abs() + bound) + TINY[kind]


def within(got, want, bound, kind=None):
    """Whether got (of type kind, its own if None) is as near as it has to be."""
    limit = stored(want, bound, kind or got.dtype)
    off = (got.double() - want).abs()
    worst = float((off / limit).max()) if off.numel() else 0.0
    assert bool((off <= limit).all()), f"{worst:.3g} times the bound"
    return worst


# ------------------------------------------------------------ layer norm ---
# A row is added by lanes of up to 32 values each, then over 64 lanes and 8 waves:
# a depth of 32 + 6 + 8.
DEPTH = 46


def _stats(x, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    var = (d * d).mean(1, keepdim=True)
    r = 1.0 / (var + eps).sqrt()
    e_mean = (DEPTH + 2) * U * x.abs().mean(1, keepdim=True)
    # the deviations are off by a common e_mean and half a step each; the common
    # part adds only its square to the variance
    e_d = U * d.abs() + e_mean
    e_var = (DEPTH + 5) * U * var + e_mean ** 2 + 2 * U * e_mean * d.abs().mean(1, keepdim=True)
    e_r = 0.5 * e_var * r * r * (1 + e_var * r * r) + 4 * U  # relative
    e_xh = r * e_d + d.abs() * r * (e_r + 2 * U)
    return d * r, r, e_xh, e_r


def layer_norm(x, gamma, beta, eps):
    xh, r, e_xh, _ = _stats(x, eps)
    gamma, beta = gamma.double(), beta.double()
    y = xh * gamma + beta
    return y, gamma.abs() * e_xh + 3 * U * ((xh * gamma).abs() + beta.abs())


def layer_norm_backward(dy, x, gamma, eps):
    """((dx, bound), (dgamma, bound), (dbeta, bound))"""
    xh, r, e_xh, e_r = _stats(x, eps)
    dy = dy.double()
    g = dy * gamma.double()
    n = x.shape[1]
    m0, m1 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    e0 = (DEPTH + 3) * U * g.abs().mean(1, keepdim=True)
    e1 = (DEPTH + 4) * U * (g * xh).abs().mean(1, keepdim=True) + \
        (g.abs() * e_xh).mean(1, keepdim=True)
    dx = r * (g - m0 - xh * m1)
    e_dx = r * (e0 + xh.abs() * e1 + e_xh * (m1.abs() + e1) +
                5 * U * (g.abs() + m0.abs() + (xh * m1).abs())) + dx.abs() * (e_r + U)
    # down the rows: at least 512 sequences, then up to 1024 / 16 + 16 + 8 more
    depth = x.shape[0] / 512 + 100
    dgamma, dbeta = (dy * xh).sum(0), dy.sum(0)
    return ((dx, e_dx),
            (dgamma, depth * U * (dy * xh).abs().sum(0) + (dy.abs() * e_xh).sum(0)),
            (dbeta, depth * U * dy.abs().sum(0)))


# ---------------------------------------------------------- gated block ---

def act(name, g):
    """(act(g), its derivative, the kernel's error in either for an exact g)."""
    if name == "relu":
        return g.clamp(min=0), (g > 0).double(), torch.zeros_like(g)
    if name == "gelu":
        phi = torch.special.ndtr(g)
        # Phi's error is half of 1.5e-7, times |g|; some eight roundings besides
        return (g * phi, phi + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi),
                (1 + g.abs()) * (0.8e-7 + 12 * U))
    s = torch.sigmoid(g)
    # exp's argument is off by |g| u, and its own error, the sum's and the
    # reciprocal's are some four roundings
    e = (g.abs().clamp(max=90) + 8) * U
    if name == "sigmoid":
        return s, s * (1 - s), 4 * e
    return g * s, s * (1 + g * (1 - s)), (1 + g.abs()) * 4 * e


def _mm(a, b):
    return torch.matmul(a, b)


def _half(x, bound, kind):
    """The bound of what is rounded to 16 bits on its way."""
    return bound + HALF_STEP[kind] * (x.abs() + bound) + TINY[kind]


def _front(x, w, b, name):
    wg, wu = w[0].double(), w[1].double()
    x = x.double()
    bg, bu = (0.0 if v is None else v.double() for v in (b[0], b[1]))
    k = x.shape[1]
    out = []
    for wt, bias in ((wg, bg), (wu, bu)):
        v = _mm(x, wt.t()) + bias
        size = _mm(x.abs(), wt.abs().t()) + (bias.abs() if torch.is_tensor(bias) else 0.0)
        out += [v, (k + 2) * 2 * U * size]
    g, eg, u, eu = out
    a, slope, ea = act(name, g)
    # |act'| <= 1.13, |act''| <= 1
    e_a = 1.13 * eg + ea
    e_s = eg + ea
    if name == "relu":
        e_s = (g.abs() <= eg).double()
    return g, u, eu, a, e_a, slope, e_s


def gated(x, w, b, name):
    kind = x.dtype
    g, u, eu, a, e_a, _, _ = _front(x, w, b, name)
    h = a * u
    eh = _half(h, a.abs() * eu + u.abs() * e_a + e_a * eu + 2 * U * h.abs(), kind)
    wd = w[2].double()
    y = _mm(h, wd.t())
    n = h.shape[1]
    e = _mm(eh, wd.abs().t()) + (n + 2) * 2 * U * _mm(h.abs() + eh, wd.abs().t())
    if b[2] is not None:
        y = y + b[2].double()
        e = e + 2 * U * b[2].double().abs()
    return y, e


def gated_backward(dy, x, w, b, name):
    """(value, bound) of dx, dw_gate, dw_up, dw_down and of the biases' gradients."""
    kind = x.dtype
    g, u, eu, a, e_a, slope, e_s = _front(x, w, b, name)
    x, dy = x.double(), dy.double()
    wg, wu, wd = (v.double() for v in w)
    m, hid = g.shape
    h = a * u
    eh = _half(h, a.abs() * eu + u.abs() * e_a + e_a * eu + 2 * U * h.abs(), kind)
    dh = _mm(dy, wd)
    edh = (dy.shape[1] + 2) * 2 * U * _mm(dy.abs(), wd.abs())
    dh_ = dh.abs() + edh
    dg, du = dh * u * slope, dh * a
    edg0 = edh * (u * slope).abs() + dh_ * (slope.abs() * eu + (u.abs() + eu) * e_s) + \
        4 * U * dg.abs()
    edu0 = edh * a.abs() + dh_ * e_a + 4 * U * du.abs()
    edg, edu = _half(dg, edg0, kind), _half(du, edu0, kind)
    dx = _mm(dg, wg) + _mm(du, wu)
    size = _mm(dg.abs() + edg, wg.abs()) + _mm(du.abs() + edu, wu.abs())
    out = [(dx, _mm(edg, wg.abs()) + _mm(edu, wu.abs()) + (2 * hid + 2) * 2 * U * size)]
    for left, eleft, right, eright in ((dg, edg, x, 0 * x), (du, edu, x, 0 * x), (dy, 0 * dy, h, eh)):
        v = _mm(left.t(), right)
        e = _mm(eleft.t(), right.abs() + eright) + _mm(left.abs().t(), eright)
        out.append((v, e + (m + 2) * 2 * U * _mm((left.abs() + eleft).t(), right.abs() + eright)))
    # sums of dg and du before they are rounded
    for v, e in ((dg, edg0), (du, edu0), (dy, 0 * dy)):
        out.append((v.sum(0), e.sum(0) + (m + 2) * U * (v.abs() + e).sum(0)))
    return out
