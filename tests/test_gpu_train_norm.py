"""Layer norm and its gradients on the GPU against their 64-bit forms."""
import pytest
import torch

from tests import train_ref as R

pytestmark = pytest.mark.gpu
KINDS = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def G():
    from paper_2402_09633_amd import gnn
    return gnn


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _table(t, pitch):
    """t in a table of wider rows."""
    if pitch is None:
        return t
    wide = torch.full((t.shape[0], pitch), 7.0, dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def _inputs(n, k, kind, seed, shift=0.3, pitch=None):
    g = _gen(seed)
    x = (torch.randn(n, k, device="cuda", generator=g) + shift).to(kind)
    dy = torch.randn(n, k, device="cuda", generator=g).to(kind)
    gamma = 1 + 0.2 * torch.randn(k, device="cuda", generator=g)
    beta = 0.1 * torch.randn(k, device="cuda", generator=g)
    return _table(x, pitch), _table(dy, pitch), gamma, beta


def _check(G, x, dy, gamma, beta, eps=1e-5):
    y, mean, rstd = G.layer_norm(x, gamma, beta, eps, save=True)
    want, bound = R.layer_norm(x, gamma, beta, eps)
    R.within(y, want, bound)
    got = G.layer_norm_backward(dy, x, gamma, mean, rstd)
    for have, (v, e) in zip(got, R.layer_norm_backward(dy, x, gamma, eps)):
        R.within(have, v, e)
    return y, got


WIDTHS = [1, 2, 3, 7, 8, 9, 16, 31, 64, 65, 128, 200, 391, 512, 513, 1000, 1024, 1025, 2047, 2048,
          2049, 4096, 4099, 8192, 10001, 16383, 16384]


@pytest.mark.parametrize("k", WIDTHS)
@pytest.mark.parametrize("kind", KINDS)
def test_widths(G, k, kind):
    for n in (1, 3, 130):
        _check(G, *_inputs(n, k, KINDS[kind], k + n))


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 255, 1000, 4097, 70_001])
def test_rows(G, n):
    for k, kind in ((24, torch.float32), (128, torch.bfloat16), (391, torch.float16)):
        _check(G, *_inputs(n, k, kind, n))


def test_many_rows(G):
    _check(G, *_inputs(1_000_513, 64, torch.float32, 1))
    _check(G, *_inputs(9_000, 2_056, torch.bfloat16, 1))


def test_tables_beyond_4_gib(G):
    m, k, piece = 1_200_000, 2048, 100_000
    g = _gen(2)
    x = torch.empty(m, k, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    dy = torch.empty(m, k, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    gamma, beta = torch.ones(k, device="cuda"), torch.zeros(k, device="cuda")
    y, mean, rstd = G.layer_norm(x, gamma, beta, save=True)
    dx, dgamma, dbeta = G.layer_norm_backward(dy, x, gamma, mean, rstd)
    sums = [[0.0, 0.0], [0.0, 0.0]]
    for at in range(0, m, piece):
        rows = slice(at, at + piece)
        want = R.layer_norm_backward(dy[rows], x[rows], gamma, 1e-5)
        if at in (0, m - piece):
            R.within(y[rows], *R.layer_norm(x[rows], gamma, beta, 1e-5))
            R.within(dx[rows], *want[0])
        for s, (v, e) in zip(sums, want[1:]):
            s[0], s[1] = s[0] + v, s[1] + e
    # a sequence of the whole has at most m / 512 + 100 numbers, twelve times a piece's
    for have, (v, e) in zip((dgamma, dbeta), sums):
        R.within(have, v, m / piece * e)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("k,pitch", [(8, 9), (128, 133), (391, 396), (512, 520), (2050, 2051)])
def test_strides(G, kind, k, pitch):
    x, dy, gamma, beta = _inputs(77, k, KINDS[kind], 3, pitch=pitch)
    x, dy = x[1:], dy[1:]
    y, got = _check(G, x, dy, gamma, beta)
    whole = torch.full((76, pitch), 5.0, dtype=x.dtype, device="cuda")
    assert torch.equal(G.layer_norm(x, gamma, beta, out=whole[:, :k]), y)
    _, mean, rstd = G.layer_norm(x, gamma, beta, save=True)
    assert (whole[:, k:] == 5).all()
    whole.fill_(5.0)
    G.layer_norm_backward(dy, x, gamma, mean, rstd, out=whole[:, :k])
    assert torch.equal(whole[:, :k], got[0]) and (whole[:, k:] == 5).all()


def test_a_large_mean_costs_no_digits(G):
    x, dy, gamma, beta = _inputs(50, 300, torch.float32, 4, shift=3000.0)
    _check(G, x, dy, gamma, beta)


def test_rows_without_spread_and_small_eps(G):
    x, dy, gamma, beta = _inputs(40, 96, torch.float32, 5)
    x[::2] = 0.25  # the mean is exact, the deviations are zero
    y, (dx, _, _) = _check(G, x, dy, gamma, beta, 1e-3)
    assert torch.equal(y[::2], beta.expand(20, -1))
    x[1::2] *= 1e-3
    _check(G, x, dy, gamma, beta, 1e-6)


@pytest.mark.parametrize("k", [40, 128, 3000])
def test_bad_rows_keep_to_themselves(G, k):
    x, dy, gamma, beta = _inputs(33, k, torch.float32, 6)
    y, (dx, _, _) = _check(G, x, dy, gamma, beta)
    x[4, 3], x[9, k - 1], x[20, 0] = float("nan"), float("inf"), -float("inf")
    y2, mean, rstd = G.layer_norm(x, gamma, beta, save=True)
    dx2 = G.layer_norm_backward(dy, x, gamma, mean, rstd)[0]
    good = torch.ones(33, dtype=torch.bool, device="cuda")
    good[[4, 9, 20]] = False
    for a, b in ((y, y2), (dx, dx2)):
        assert torch.equal(a[good], b[good])
        assert b[~good].isnan().any(1).all()


def test_in_place(G):
    x, dy, gamma, beta = _inputs(300, 130, torch.bfloat16, 7)
    y, mean, rstd = G.layer_norm(x, gamma, beta, save=True)
    dx = G.layer_norm_backward(dy, x, gamma, mean, rstd)[0]
    keep = x.clone()
    assert G.layer_norm(keep, gamma, beta, out=keep) is keep and torch.equal(keep, y)
    keep = dy.clone()
    assert torch.equal(G.layer_norm_backward(keep, x, gamma, mean, rstd, out=keep)[0], dx)
    assert torch.equal(keep, dx)


def test_no_rows(G):
    x, dy, gamma, beta = _inputs(0, 12, torch.float32, 8)
    y, mean, rstd = G.layer_norm(x, gamma, beta, save=True)
    dx, dgamma, dbeta = G.layer_norm_backward(dy, x, gamma, mean, rstd)
    assert y.shape == dx.shape == (0, 12) and mean.shape == (0,)
    assert (dgamma == 0).all() and (dbeta == 0).all() and dgamma.shape == (12,)


def test_same_bits_every_time(G):
    a = _inputs(50_000, 131, torch.float16, 9)
    first = _check(G, *a)
    again = _check(G, *a)
    assert all(torch.equal(p, q) for p, q in zip((first[0], *first[1]), (again[0], *again[1])))
