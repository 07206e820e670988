"""The training operators' plain forms against differences of the forward pass."""
import pytest
import torch

from tests import train_ref as R


def _rand(*shape, seed):
    return torch.randn(*shape, dtype=torch.float64, generator=torch.Generator().manual_seed(seed))


def _slope(f, leaf, way, step=1e-5):
    return (f(leaf + step * way) - f(leaf - step * way)) / (2 * step)


def test_layer_norm_gradient_is_the_slope():
    x, dy, gamma, beta = (_rand(*s, seed=i) for i, s in enumerate([(6, 11), (6, 11), (11,), (11,)]))
    (dx, _), (dg, _), (db, _) = R.layer_norm_backward(dy, x, gamma, 1e-5)
    loss = lambda x, g, b: float((R.layer_norm(x, g, b, 1e-5)[0] * dy).sum())
    for i, (leaf, grad) in enumerate(((x, dx), (gamma, dg), (beta, db))):
        way = _rand(*leaf.shape, seed=9 + i)
        args = [x, gamma, beta]

        def f(v):
            args[i] = v
            return loss(*args)

        # the loss is a few units: steps of 1e-5 leave 1e-10 of curvature and 1e-10 of rounding
        assert abs(_slope(f, leaf, way) - float((grad * way).sum())) < 1e-7


@pytest.mark.parametrize("name", ["silu", "gelu", "sigmoid", "relu"])
def test_gated_gradient_is_the_slope(name, monkeypatch):
    for table in (R.HALF_STEP, R.TINY):
        monkeypatch.setitem(table, torch.float64, 0.0)
    shapes = [(7, 5), (9, 5), (9, 5), (4, 9), (9,), (9,), (4,)]
    leaves = [_rand(*s, seed=i) for i, s in enumerate(shapes)]
    dy = _rand(7, 4, seed=20)
    grads = [v for v, _ in R.gated_backward(dy, leaves[0], leaves[1:4], leaves[4:], name)]
    for i, (leaf, grad) in enumerate(zip(leaves, grads)):
        way = _rand(*leaf.shape, seed=30 + i)

        def f(v):
            at = leaves[:i] + [v] + leaves[i + 1:]
            return float((R.gated(at[0], at[1:4], at[4:], name)[0] * dy).sum())

        want = float((grad * way).sum())
        assert abs(_slope(f, leaf, way) - want) < 1e-6 * max(1.0, abs(want))
