"""Refusals and sizes of the training operators that need no GPU."""
import numpy as np
import pytest


@pytest.fixture(scope="module")
def G():
    from paper_2402_09633_amd import gnn
    return gnn


# Arguments are checked before any device call: the addresses below are never read.
X, Y, W = 1 << 20, 2 << 20, 4 << 20


@pytest.mark.parametrize("norm", [X, X + 12, Y, Y + 28])
def test_clip_refuses_a_norm_inside_a_tensor(G, norm):
    t = np.zeros(2, G._GRAD)
    t[0], t[1] = (X, X, 4, 0, 0), (X + 4096, Y, 8, 0, 0)
    assert G.lib.gnn_clip_grads(t.ctypes.data, 2, 1.0, norm, W, 1 << 30, None) == G.GNN_E_INVALID_ARG
    assert "overlap" in G.gnn_last_error()


@pytest.mark.parametrize("n,k", [(1, 16_384), (3, 7), (1000, 128), (8192, 8192), (1_000_000, 128),
                                 (1 << 28, 8)])
def test_layer_norm_scratch_is_what_is_used(G, n, k):
    """dgamma and dbeta of each of at most 1024 workgroups, and nothing beside them."""
    rows = 1 if k > 2048 else max(1, 64 // max(1, (k + 7) // 8)) * 4
    groups = min(-(-n // rows), 512 if k > 2048 else 1024)
    assert G.lib.gnn_layer_norm_workspace(n, k) <= groups * 2 * k * 4 + 256


@pytest.mark.parametrize("k,h,n", [(2048, 8192, 2048), (16, 16_384, 16), (128, 256, 128)])
def test_gated_scratch_of_few_rows(G, k, h, n):
    """h, dg and du in two 16-bit numbers each, the sums of dg and du over the rows of each
    of four waves, and one row of sums of dy in either place where they may be."""
    d = G.make_gated_dims(k, h, n)
    pad = 12 * 256
    for m in (0, 1, 16):
        assert G.lib.gnn_gated_workspace(d, m, 1, 1) <= m * h * 12 + 4 * 2 * h * 4 + 2 * n * 4 + pad
