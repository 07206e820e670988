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


def _all_calls(G):
    """Every call with a stream argument, as a function of the stream alone."""
    rng = np.random.default_rng(1)
    x = torch.as_tensor(rng.normal(size=(300, 6)).astype(np.float32)).cuda()
    ids = torch.as_tensor(rng.integers(0, 3, 300).astype(np.int32)).cuda()
    ld, md = G.make_linear_dims(6, 4, 3), G.make_mlp_dims([6, 16, 4], 3, G.GNN_INT8)
    layer = G.Linear(rng.normal(size=G.gnn_linear_weight_count(ld)).astype(np.float32), ld)
    mlp = G.Mlp(rng.normal(size=G.gnn_mlp_weight_count(md)).astype(np.float32), md)
    off, order = G.group_rows(ids, 3)
    torch.cuda.synchronize()
    return [lambda s: G.quantize_rows(x, stream=s), lambda s: G.group_rows(ids, 3, stream=s),
            lambda s: (layer(x, offsets=off, order=order, stream=s),),
            lambda s: (mlp(x, ids, stream=s),)]


def test_streams_of_other_devices_are_refused(G):
    here = torch.cuda.Stream()

    class Elsewhere(torch.cuda.Stream):
        device = torch.device("cuda", 1 + torch.cuda.current_device())

    for call in _all_calls(G):
        with pytest.raises(ValueError, match="stream"):
            call(Elsewhere())
        call(here)
    torch.cuda.synchronize()


def test_streams_by_handle(G):
    side = torch.cuda.Stream()
    for call in _all_calls(G):
        want = call(None)
        torch.cuda.synchronize()
        for s in (side, side.cuda_stream, 0):  # 0: the default stream
            got = call(s)
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("kind", ["GNN_BF16", "GNN_INT8"])
@pytest.mark.parametrize("m,n", [(64, 300), (4000, 1100), (70_000, 40)])
def test_row_named_by_positions_of_two_groups(G, kind, m, n):
    """Every element of such a row is the one or the other group's."""
    rng = np.random.default_rng(1)
    k = 24
    d = G.make_linear_dims(k, n, 2, getattr(G, kind))
    layer = G.Linear(rng.normal(size=G.gnn_linear_weight_count(d)).astype(np.float32), d)
    x = torch.as_tensor(rng.normal(size=(m, k)).astype(np.float32)).cuda()
    half = m // 2
    off = torch.tensor([0, half, m], dtype=torch.int32, device="cuda")
    order = torch.arange(m, dtype=torch.int32, device="cuda")
    order[1:half:3] += half  # named by a position of group 0 and by their own of group 1
    y = layer(x, offsets=off, order=order, out=torch.full((m, n), 9.0, device="cuda"))
    first = layer(x, offsets=torch.tensor([0, m, m], dtype=torch.int32, device="cuda"))
    second = layer(x, offsets=torch.tensor([0, 0, m], dtype=torch.int32, device="cuda"))
    unnamed = torch.zeros(m, dtype=torch.bool, device="cuda")
    unnamed[1:half:3] = True
    twice = torch.roll(unnamed, half)
    assert (y[unnamed] == 9).all()
    assert ((y[twice] == first[twice]) | (y[twice] == second[twice])).all()
    once = ~(unnamed | twice)
    once[half:] = False
    assert torch.equal(y[once], first[once])
    once = ~(unnamed | twice)
    once[:half] = False
    assert torch.equal(y[once], second[once])
