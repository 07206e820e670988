"""The bounds of train_fine_ref: they cover what the kernels' roundings leave, and
nothing that drops the second of two numbers, or takes it from the first."""
import pytest
import torch

from tests import train_fine_ref as F
from tests import train_ref as R

KINDS = {"bf16": torch.bfloat16, "f16": torch.float16}
# Short fp32 sums, which have little to lose, and many results of each kind, some of
# which nearly cancel and show what the first number's rounding left: y and dWd, dx, dWg
# and dWu.
CASES = [(16, 8, 16, 600), (5, 12, 8, 900), (1, 16, 24, 2000), (16, 40, 8, 2), (9, 32, 16, 4),
         (16, 9, 300, 10)]
NAMES = ("y", "dx", "dw_gate", "dw_up", "dw_down")


def case(m, k, h, n, kind, device="cpu"):
    g = torch.Generator().manual_seed(m + k + h + n)

    def rand(*shape, by=1.0):
        return (torch.randn(*shape, generator=g) * by).to(kind).to(device)

    w = [rand(h, k, by=k ** -0.5), rand(h, k, by=k ** -0.5), rand(n, h, by=h ** -0.5)]
    return rand(m, k), w, [None] * 3, rand(m, n)


def wanted(x, w, b, dy, act):
    return [F.gated(x, w, b, act), *F.gated_backward(dy, x, w, b, act)]


def simulated(x, w, dy, act, rest):
    """The block in 64 bits, with the kernels' roundings of h, dg and du: `rest` times what
    the first of two numbers left goes on as the second."""
    kind = x.dtype

    def sent(v):
        hi = v.to(kind).double()
        return hi + rest * (v - hi).to(kind).double()

    wg, wu, wd = (t.double() for t in w)
    x, dy = x.double(), dy.double()
    g, u = x @ wg.t(), x @ wu.t()
    a, slope, _ = R.act(act, g)
    dh = dy @ wd
    h, dg, du = sent(a * u), sent(dh * u * slope), sent(dh * a)
    return [v.to(kind) for v in (h @ wd.t(), dg @ wg + du @ wu, dg.t() @ x, du.t() @ x, dy.t() @ h)]


def _worst(have, want):
    v, e = want
    return float(((have.double() - v).abs() / R.stored(v, e, have.dtype)).max())


@pytest.mark.parametrize("kind", KINDS)
def test_two_numbers_are_told_from_one(kind):
    caught = {rest: set() for rest in (0.0, -1.0)}
    for size in CASES:
        x, w, b, dy = case(*size, KINDS[kind])
        want = wanted(x, w, b, dy, "silu")
        for name, have, v in zip(NAMES, simulated(x, w, dy, "silu", 1.0), want):
            assert _worst(have, v) <= 1.0, (size, name)
        for rest in caught:
            for name, have, v in zip(NAMES, simulated(x, w, dy, "silu", rest), want):
                if _worst(have, v) > 1.0:
                    caught[rest].add(name)
    assert caught[0.0] == caught[-1.0] == set(NAMES)


@pytest.mark.parametrize("act", ["silu", "gelu", "sigmoid", "relu"])
def test_the_largest_numbers_are_bounded(act):
    for m, k, h, n in ((1, 1, 1, 1), (7, 5, 3, 4), (50, 40, 30, 20)):
        for by in (1e-3, 1.0, 30.0):
            x, w, b, dy = case(m, k, h, n, torch.float16)
            x, b = (x * by).half(), [0.3 * torch.ones(v).half() for v in (h, h, n)]
            g = x.double() @ w[0].double().t() + b[0].double()
            u = x.double() @ w[1].double().t() + b[1].double()
            a, slope, _ = R.act(act, g)
            dh = dy.double() @ w[2].double()
            top_grad, top_h = F.largest(dy, x, w, b, act)
            assert float((a * u).abs().max()) <= top_h * (1 + 1e-12)
            assert float((dh * u * slope).abs().max()) <= top_grad * (1 + 1e-12)
            assert float((dh * a).abs().max()) <= top_grad * (1 + 1e-12)


def test_rounding_alone_is_what_share_counts():
    """A product of rounded random numbers stays within the share of its rounding."""
    g = torch.Generator().manual_seed(3)
    left, right = (torch.randn(400, 300, dtype=torch.float64, generator=g) for _ in range(2))
    for kind in KINDS.values():
        want = left @ right.t()
        have = (left.to(kind).double() @ right.t()).to(kind)
        assert F.relative(have, want) <= F.share(want, kind, False)
        assert F.relative(want.to(kind), want) <= F.share(want, kind, True)
        assert F.relative(have, want) > F.share(want, kind, True)
