"""How the training operators take their arguments."""
import warnings

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


def test_no_graph_is_recorded_in_silence(G):
    """x + gated(layer_norm(x)) would go back through x alone."""
    x, w, b, _ = make(20, 32, 24, 32, torch.bfloat16, 1)
    gamma, beta = torch.ones(32, device="cuda"), torch.zeros(32, device="cuda")
    calls = {"layer_norm": ([x, gamma, beta], lambda a: G.layer_norm(*a)),
             "gated": ([x, *w, *b], lambda a: G.gated(*a[:4], biases=a[4:]))}
    for name, (args, call) in calls.items():
        for i, leaf in enumerate(args):
            some = [t.clone().requires_grad_() if t is leaf else t for t in args]
            with pytest.warns(UserWarning, match=f"{name} records no autograd graph.*{name}_backward"):
                assert not call(some).requires_grad
            with warnings.catch_warnings():
                warnings.simplefilter("error")
                with torch.no_grad():
                    call(some)
                call([t.detach() for t in some])
