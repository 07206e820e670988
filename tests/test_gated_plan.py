"""Which kernels a gated block's call takes: the GPU tests reach every tile that the rule
can choose (256 compute units)."""
import pytest

from tests.test_gpu_train_tiles import NARROW, TILES

CU = 256


@pytest.fixture(scope="module")
def G():
    from paper_2402_09633_amd import gnn
    return gnn


def plans(G, m, k, h, n):
    d = G.make_gated_dims(k, h, n)
    return G.gnn_debug_gated(d, CU, m), G.gnn_debug_gated(d, CU, m, backward=True)


@pytest.mark.parametrize("size,tiles,gate_up,down", TILES, ids=lambda v: str(v))
def test_the_calls_take_these_tiles(G, size, tiles, gate_up, down):
    f, b = plans(G, *size)
    assert f[0] == b[0] == 0
    assert (f[1], f[2], b[1], b[2]) == tiles
    assert (b[3], b[4] > 1) == gate_up and (b[5], b[6] > 1) == down


def test_every_tile_is_reached():
    for i in range(4):
        assert {t[1][i] for t in TILES} == {0, 1, 2, 3}
    for i in (2, 3):
        assert {t[i] for t in TILES} == {(t, parts) for t in range(4) for parts in (False, True)}


def test_narrow_and_few_rows(G):
    for size in NARROW:
        f, b = plans(G, *size)
        assert f[0] == b[0] == 2 and f[1:3] == b[1:3] == (-1, -1)
    assert {(k > 64, n > 64) for _, k, _, n in NARROW} == {(p, q) for p in (False, True)
                                                          for q in (False, True)}
    for m in (1, 16, 17, 64):
        f, b = plans(G, m, 96, 4096, 160)
        assert f[0] == 1 and b[0] == 0 and f[2] > 1
    assert plans(G, 65, 96, 4096, 160)[0][0] == 0


def test_debug_gated_refuses(G):
    d = G.make_gated_dims(8, 8, 8)
    for args in ((0, 10), (-1, 10), (256, 0), (256, -1)):
        with pytest.raises(G.GnnError):
            G.gnn_debug_gated(d, *args)
    for bad in (G.make_gated_dims(8, 20_000, 8), G.make_gated_dims(8, 8, 8, dtype=G.GNN_FP32)):
        with pytest.raises(G.GnnError):
            G.gnn_debug_gated(bad, 256, 10)
    assert G.lib.gnn_debug_gated(None, 256, 10, 0, None) == G.GNN_E_INVALID_ARG
    assert G.lib.gnn_debug_gated(d, 256, 10, 0, None) == G.GNN_E_INVALID_ARG
