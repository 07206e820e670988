"""Up to 16 rows the gated block's h, dg and du go on in two 16-bit numbers:
test_train_fine_ref.py shows that these bounds tell them from one."""
import pytest
import torch

from tests import train_fine_ref as F
from tests import train_ref as R
from tests.test_gpu_train_gated import ACTS, make
from tests.test_train_fine_ref import CASES, KINDS, NAMES, case, wanted

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    from paper_2402_09633_amd import gnn
    return gnn


def _check(G, x, w, b, dy, act):
    biases = None if b[0] is None else b
    got = [G.gated(x, *w, biases=biases, activation=act),
           *G.gated_backward(dy, x, *w, biases=biases, activation=act)[:4]]
    want = [F.gated(x, w, b, act), *F.gated_backward(dy, x, w, b, act)]
    for name, have, (v, e) in zip(NAMES, got, want):
        assert R.within(have, v, e) <= 1.0, name


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("size", CASES, ids=str)
def test_both_numbers_count(G, size, act, kind):
    x, w, b, dy = case(*size, KINDS[kind], "cuda")
    _check(G, x, w, b, dy, act)


# One row to the most that have two numbers, whole blocks of the products and their ends.
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("m", [1, 2, 7, 15, 16])
@pytest.mark.parametrize("k,h,n", [(64, 64, 64), (37, 75, 29), (1, 1, 1), (130, 129, 257),
                                   (24, 1031, 40), (264, 72, 520)])
def test_sizes(G, m, k, h, n, kind):
    x, w, b, dy = make(m, k, h, n, KINDS[kind], m + h)
    _check(G, x, w, b, dy, "silu")


def test_the_error_is_that_of_rounding_the_result(G):
    """Over whole tables, as one product of many results shows it."""
    for kind in KINDS.values():
        for m, k, h, n in ((2, 36, 114, 4386), (16, 64, 512, 256), (1, 512, 2048, 512)):
            x, w, b, dy = make(m, k, h, n, kind, 3, bias=False)
            got = [G.gated(x, *w), *G.gated_backward(dy, x, *w)[:4]]
            for name, have, (v, _) in zip(NAMES, got, wanted(x, w, b, dy, "silu")):
                assert F.relative(have, v) <= F.share(v, kind, True), name
