"""The binding of the row operators, as far as it needs no GPU."""
import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def G():
    from paper_2402_09633_amd import gnn
    return gnn


# Counts that the C calls take in 32 bits: their low bits alone would name
# another, smaller call.

def test_counts_past_32_bits_are_refused(G):
    big = (1 << 32) + 8
    for v in (big, 1 << 31, -big):
        with pytest.raises(ValueError, match="32-bit"):
            G.gnn_group_workspace(100, v)
        with pytest.raises(ValueError, match="32-bit"):
            G.gnn_group_rows(1 << 20, 100, v, 2 << 20, 3 << 20)
        with pytest.raises(ValueError, match="32-bit"):
            G.gnn_quantize_rows(1 << 20, G.GNN_FP32, 1 << 31, 1, v, 2 << 20, 1 << 31, 3 << 20)
        for kw in (dict(in_features=v), dict(out_features=v), dict(n_groups=v)):
            with pytest.raises(ValueError, match="32-bit"):
                G.make_linear_dims(**{**dict(in_features=8, out_features=8), **kw})
        with pytest.raises(ValueError, match="32-bit"):
            G.make_mlp_dims([3, v, 8])
        with pytest.raises(ValueError, match="32-bit"):
            G.make_mlp_dims([3, 8], n_groups=v)
    with pytest.raises(TypeError):
        G.make_linear_dims(8.0, 8)


def test_rows_wider_than_32_bits_are_refused(G):
    meta = torch.device("meta")
    for cols in (1 << 31, (1 << 32) + 8):
        x = torch.empty(1, cols, dtype=torch.bfloat16, device=meta)
        with pytest.raises(ValueError, match="at most"):
            G._rows("x", x, None, None, meta)
    x = torch.empty(2, (1 << 31) - 1, dtype=torch.bfloat16, device=meta)
    assert G._rows("x", x, None, None, meta)[1:] == (G.GNN_BF16, (1 << 31) - 1)


@pytest.mark.parametrize("kw,code", [
    (dict(in_features=0), "GNN_E_INVALID_ARG"), (dict(dtype=9), "GNN_E_INVALID_ARG"),
    (dict(in_features=16385), "GNN_E_UNSUPPORTED"), (dict(n_groups=4097), "GNN_E_UNSUPPORTED"),
    (dict(dtype=0), "GNN_E_UNSUPPORTED")])
def test_refused_layers_say_why(G, kw, code):
    d = G.make_linear_dims(**{**dict(in_features=8, out_features=8), **kw})
    with pytest.raises(G.GnnError) as e:
        G.gnn_linear_create(np.zeros(72, np.float32), d)
    assert e.value.code == getattr(G, code) == G.gnn_last_error_code()
    with pytest.raises(G.GnnError) as e:
        G.gnn_mlp_create(np.zeros(72, np.float32),
                         G.make_mlp_dims([d.in_features, 8], d.n_groups, d.dtype))
    assert e.value.code == getattr(G, code)


@pytest.mark.skipif(torch.cuda.device_count() > 0, reason="a GPU is visible")
def test_creating_without_a_device_says_so(G):
    with pytest.raises(G.GnnError) as e:
        G.gnn_linear_create(np.zeros(72, np.float32), G.make_linear_dims(8, 8))
    assert e.value.code == G.GNN_E_NO_DEVICE
    with pytest.raises(G.GnnError) as e:
        G.gnn_mlp_create(np.zeros(72, np.float32), G.make_mlp_dims([8, 8]))
    assert e.value.code == G.GNN_E_NO_DEVICE
