"""How the training operators take their arguments."""
import pytest
import torch

from tests.test_gpu_train_gated import make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    from paper_2402_09633_amd import gnn
    return gnn


@pytest.mark.parametrize("stream", [None, 0])
def test_biases_may_come_from_an_iterator(G, stream):
    x, w, b, dy = make(20, 32, 24, 40, torch.bfloat16, 1)
    for some in (b, [b[0], None, None], [None, b[1], b[2]]):
        want = G.gated_backward(dy, x, *w, biases=some)
        got = G.gated_backward(dy, x, *w, biases=iter(some), stream=stream)
        torch.cuda.synchronize()
        assert len(got) == len(want) == 7
        for p, q in zip(got, want):
            assert (p is None and q is None) or torch.equal(p, q)
        y = G.gated(x, *w, biases=iter(some), stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(y, G.gated(x, *w, biases=some))
