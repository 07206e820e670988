"""Which kernel a linear layer's call takes: the selection's rules, and the kernels
that the GPU tests of the layers reach (256 compute units)."""
import pytest

from tests.test_gpu_rows_panels import CASES, ROWS

CU = 256


@pytest.fixture(scope="module")
def G():
    from paper_2402_09633_amd import gnn
    return gnn


def plan(G, kind, xt, m, k, n, g=1, y="f32", pitch=0, grouped=None):
    """(convert, tile, row blocks, waves, staging, split)."""
    types = {"f32": G.GNN_FP32, "bf16": G.GNN_BF16, "f16": G.GNN_F16, "i8": G.GNN_INT8}
    return G.gnn_debug_linear(G.make_linear_dims(k, n, g, types[kind]), CU, types[xt], m,
                              g > 1 if grouped is None else grouped, types[y], pitch)


def test_rows_are_converted_only_for_a_kernel_that_needs_it(G):
    """A pass over the rows is paid for where the tiles take the call (whose rows
    have the weights' type, in whole chunks of 16 bytes), or where the panels
    cannot: other 16-bit types, and rows too wide to be rounded while they are
    staged."""
    for kind in ("i8", "bf16", "f16"):
        for xt in ("f32", "bf16", "f16") + (("i8",) if kind == "i8" else ()):
            for m in (1, 300, 4100, 9000, 14001, 30000, 32767, 32768, 100000, 1000000):
                for k in (1, 64, 500, 512, 640, 896, 897, 960, 1000, 1024, 1025, 1152, 1153, 2048,
                          4096, 4097, 9000):
                    for n in (1, 32, 128, 129, 512, 1024, 1025, 1056, 2048, 4096):
                        convert, tile, rb, waves, staging, split = plan(G, kind, xt, m, k, n)
                        size = 1 if kind == "i8" else 2
                        if tile:
                            want = xt != kind or k * size % 16 != 0
                            assert tile in (2, 4) and rb == 0
                        else:
                            want = k > 4096 if kind == "i8" and xt != "i8" else \
                                xt not in ("f32", kind)
                            assert rb in (1, 2, 4) and waves in (4, 8)
                        assert convert == want, (kind, xt, m, k, n)


def test_debug_linear_refuses(G):
    d = G.make_linear_dims(8, 8, 1, G.GNN_BF16)
    for args in ((0, 0, 10), (256, 5, 10), (256, G.GNN_INT8, 10), (256, 0, 0), (256, 0, -1)):
        with pytest.raises(G.GnnError):
            G.gnn_debug_linear(d, *args)
    with pytest.raises(G.GnnError):
        G.gnn_debug_linear(d, 256, 0, 10, y_type=G.GNN_INT8)
    with pytest.raises(G.GnnError):
        G.gnn_debug_linear(G.make_linear_dims(8, 20000), 256, 0, 10)
    assert G.lib.gnn_debug_linear(None, 256, 0, 10, 0, 0, 8, None) == G.GNN_E_INVALID_ARG


# The calls that the GPU tests make for the tiles (test_linear_tiles and
# test_grouped_tiles of test_gpu_rows.py).
@pytest.mark.parametrize("kind,xt,m,k,n,g,tile", [
    ("bf16", "bf16", 4100, 640, 1100, 1, 2), ("bf16", "bf16", 4100, 643, 1100, 1, 2),
    ("f16", "f16", 14_001, 520, 1400, 1, 4), ("f16", "f32", 4100, 650, 1030, 1, 2),
    ("bf16", "f16", 4100, 520, 1027, 1, 2), ("i8", "bf16", 4100, 1000, 1100, 1, 2),
    ("i8", "f32", 14_001, 901, 1300, 1, 4), ("i8", "i8", 4100, 1040, 1100, 1, 2),
    ("i8", "i8", 4100, 1101, 1100, 1, 2), ("bf16", "bf16", 2000, 2056, 2100, 1, 2),
    ("i8", "bf16", 6000, 1032, 1100, 3, 2), ("i8", "bf16", 9000, 1001, 1064, 5, 2),
    ("i8", "bf16", 17_000, 904, 1100, 7, 4), ("bf16", "bf16", 6000, 1032, 1100, 3, 2),
    ("bf16", "bf16", 9000, 1001, 1064, 5, 2), ("f16", "f16", 17_000, 904, 1100, 7, 4)])
def test_tiles_take(G, kind, xt, m, k, n, g, tile):
    assert plan(G, kind, xt, m, k, n, g)[1] == tile


# The calls of test_gpu_rows_panels.py, and the ones that it compares them with.
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}x{c[1]}-{c[2]}")
@pytest.mark.parametrize("kind", ["i8", "bf16", "f16"])
def test_large_calls_take(G, kind, case):
    m, k, n, out, gap, g, want8, want16 = case
    want = want8 if kind == "i8" else want16
    for xt in ROWS[kind]:
        convert, tile, rb, waves, staging, split = plan(G, kind, xt, m, k, n, g, out, n + gap)
        if want is not None and len(want) == 2:
            assert (tile, rb, waves) == (0, *want), xt
        elif want is not None:
            assert (tile,) == want, xt
        if g == 1:  # calls of few rows run something else
            assert plan(G, kind, xt, 3000, k, n, g, out, n) != (convert, tile, rb, waves, staging, split)


def test_the_large_calls_reach_every_large_kernel(G):
    """Every panel of more than 32 rows, and both tiles, in every pair of weight
    and row types that they come in."""
    seen = set()
    for m, k, n, out, gap, g, _, _ in CASES:
        for kind, rows in ROWS.items():
            for xt in rows:
                convert, tile, rb, waves, staging, split = plan(G, kind, xt, m, k, n, g, out, n + gap)
                seen.add((kind, kind if convert else xt, tile, rb, waves))
    for kind, rows in ROWS.items():
        for xt in rows:
            for rb, waves in ((4, 8), (2, 8), (4, 4), (2, 4)):
                assert (kind, xt, 0, rb, waves) in seen, (kind, xt, rb, waves)
        assert (kind, kind, 4, 0, 0) in seen, kind
