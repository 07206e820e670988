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
