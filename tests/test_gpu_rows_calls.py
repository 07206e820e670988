"""How the row operators are called on the GPU: dims, streams and errors."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    from paper_2402_09633_amd import gnn
    return gnn


def test_dims_of_one_network_reused_for_the_next(G):
    rng = np.random.default_rng(1)
    dims = G.make_mlp_dims([6, 16, 4], 1, G.GNN_BF16)
    w = rng.normal(size=G.gnn_mlp_weight_count(dims)).astype(np.float32)
    first = G.Mlp(w, dims)
    x = torch.as_tensor(rng.normal(size=(50, 6)).astype(np.float32)).cuda()
    y = first(x)
    dims.widths[0], dims.widths[2], dims.n_layers, dims.widths[3] = 5, 8, 3, 2
    second = G.Mlp(rng.normal(size=G.gnn_mlp_weight_count(dims)).astype(np.float32), dims)
    assert torch.equal(first(x), y)
    assert second(x[:, :5]).shape == (50, 2)
