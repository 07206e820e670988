"""fp16 gradients of the gated block where upstream gradients or rows are small, or
large: what fp16 cannot hold of h, dg and du is not lost."""
import pytest
import torch

from tests import train_fine_ref as F
from tests import train_ref as R
from tests.test_gpu_train_gated import ACTS, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    from paper_2402_09633_amd import gnn
    return gnn


def _scaled(m, k, h, n, seed, x_by, dy_by, kind=torch.float16, bias=False):
    x, w, b, _ = make(m, k, h, n, torch.float32, seed, bias=bias)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    dy = torch.randn(m, n, device="cuda", generator=g)
    return ((x * x_by).to(kind), [t.to(kind) for t in w],
            [None if t is None else (t * x_by).to(kind) for t in b], (dy * dy_by).to(kind))


def _held(have, v, e):
    """have is within e of v where fp16 reaches (65504 is its last number, from 65520 on
    everything is rounded to infinity), and infinite beyond."""
    fits = v.abs() + e < 65504
    R.within(have[fits], v[fits], e[fits])
    beyond = v.abs() - e > 65520
    assert have[beyond].isinf().all() and (have[beyond] * v[beyond] > 0).all()
    return bool(fits.all())


def _check(G, x, w, b, dy, act):
    biases = None if b[0] is None else b
    got = G.gated_backward(dy, x, *w, biases=biases, activation=act)
    want = F.gated_backward(dy, x, w, b, act)
    two = x.shape[0] <= F.TWO_ROWS
    fit = [_held(have, v, e) for have, (v, e) in zip(got, want)]
    if act != "sigmoid" and float(x.abs().max()) > 1e-3:
        for have, (v, _), all_fit in zip(got, want, fit):
            if not all_fit:
                continue
            off, limit = F.relative(have, v), F.share(v, x.dtype, two)
            assert off <= limit, f"{off:.3g} of the whole, {limit:.3g} allowed"
    for have, (v, e) in zip(got[4:], R.gated_backward(dy, x, w, b, act)[4:]):
        if have is not None:
            R.within(have, v, e)


# Few rows, every tile for more, narrow rows in many tiles, odd widths.
SHAPES = [(1, 64, 512, 256), (8, 64, 4096, 256), (16, 37, 75, 29), (17, 256, 512, 256),
          (300, 64, 4096, 256), (4096, 256, 512, 256), (1000, 391, 131, 259),
          (9000, 136, 264, 72), (33_003, 128, 256, 128), (33_000, 40, 31, 33)]


@pytest.mark.parametrize("m,k,h,n", SHAPES)
@pytest.mark.parametrize("x_by,dy_by", [(1.0, 1.0), (1.0, 1e-2), (1.0, 1e-4), (1.0, 1e-5),
                                        (1e-2, 1.0), (1e-2, 1e-3), (1e-3, 1e-2), (30.0, 1e-5),
                                        (1.0, 1000.0)])
def test_small_and_large(G, m, k, h, n, x_by, dy_by):
    _check(G, *_scaled(m, k, h, n, m + k, x_by, dy_by), "silu")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m,k,h,n", [(12, 64, 512, 96), (700, 128, 256, 128), (33_001, 64, 96, 64)])
def test_activations_of_small_gradients(G, act, m, k, h, n):
    _check(G, *_scaled(m, k, h, n, 5, 1.0, 1e-5, bias=True), act)


def test_rows_of_very_different_sizes(G):
    """Gradients of most rows far below those of a few."""
    x, w, b, dy = _scaled(2000, 128, 256, 128, 6, 1.0, 1.0)
    dy[torch.arange(2000, device="cuda") % 50 != 0] *= 2.0 ** -12
    got = G.gated_backward(dy, x, *w)
    for have, (v, e) in zip(got, F.gated_backward(dy, x, w, b, "silu")):
        R.within(have, v, e)


@pytest.mark.parametrize("act", ["relu", "silu"])
@pytest.mark.parametrize("m", [3, 40, 33_000])
def test_the_largest_numbers_stay_numbers(G, m, act):
    """One element each, so that the bounds are met: nothing that fp16 holds becomes
    infinite, and nothing that it cannot hold is made a number."""
    for wu, wg, wd, by in ((200.0, 1.0, 60.0, 2.0 ** -12), (0.5, 8.0, 1000.0, 2.0 ** -9),
                           (2.0 ** -10, 2.0 ** -9, 2.0 ** -8, 2.0 ** -14), (30.0, 3.0, 2.0, 8.0)):
        t = lambda v: torch.full((1, 1), v, dtype=torch.float16, device="cuda")
        x = torch.linspace(0.25, 16.0, m, device="cuda").half()[:, None].contiguous()
        dy = torch.full((m, 1), by, device="cuda").half()
        w = [t(wg), t(wu), t(wd)]
        got = G.gated_backward(dy, x, *w, activation=act)
        want = F.gated_backward(dy, x, w, [None] * 3, act)
        for have, (v, e) in zip(got, want):
            _held(have, v, e)


@pytest.mark.parametrize("m", [9, 300, 33_000])
def test_bad_numbers_do_not_set_the_range(G, m):
    x, w, b, dy = _scaled(m, 64, 96, 32, 7, 1.0, 1e-5)
    good = torch.ones(m, dtype=torch.bool, device="cuda")
    good[[2, m - 1]] = False
    clean = F.gated_backward(dy[good], x[good], w, b, "silu", two=m <= 16)[0]
    x[2, 5], dy[m - 1, 3] = float("nan"), float("inf")
    dx = G.gated_backward(dy, x, *w)[0]
    R.within(dx[good], *clean)
    assert dx[2].isnan().all() and not dx[m - 1].isfinite().any()


def test_zero_gradients(G):
    x, w, b, dy = _scaled(200, 64, 96, 32, 8, 1.0, 1.0)
    for t in G.gated_backward(torch.zeros_like(dy), x, *w)[:4]:
        assert (t == 0).all()
    for t in G.gated_backward(dy, torch.zeros_like(x), *w)[1:4]:
        assert (t == 0).all()


def test_the_range_is_found_again_in_a_replay(G):
    """A captured call takes its powers of two from the numbers of each replay."""
    sizes = ((9, 64, 96, 32), (300, 64, 96, 40), (300, 37, 75, 29), (33_000, 64, 96, 32))
    held = [_scaled(*s, 9, 1.0, 1.0) for s in sizes]
    for x, w, b, dy in held:
        G.gated_backward(dy, x, *w)
    torch.cuda.synchronize()
    graphs, outs, pool = [], [], torch.cuda.graph_pool_handle()
    for x, w, b, dy in held:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=pool):
            outs.append(G.gated_backward(dy, x, *w)[:4])
        graphs.append(g)
    for turn, (x_by, dy_by) in enumerate(((1.0, 1e-5), (30.0, 1.0), (1e-2, 1e-3), (1.0, 1.0))):
        for s, (x, w, b, dy), g, out in zip(sizes, held, graphs, outs):
            fresh = _scaled(*s, 10 + turn, x_by, dy_by)
            for t, v in zip([x, *w, dy], [fresh[0], *fresh[1], fresh[3]]):
                t.copy_(v)
            g.replay()
            got = [t.clone() for t in out]
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got, G.gated_backward(dy, x, *w)[:4]))
            for have, (v, e) in zip(got, F.gated_backward(dy, x, w, b, "silu")):
                _held(have, v, e)
