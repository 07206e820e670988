"""Refusals of the row operators that need no GPU, and their plain forms."""
import ctypes

import numpy as np
import pytest

from tests import rows_ref as R


@pytest.fixture(scope="module")
def G():
    from paper_2402_09633_amd import gnn
    return gnn


@pytest.mark.parametrize("kw,code", [
    (dict(in_features=0), "positive"), (dict(out_features=-1), "positive"),
    (dict(in_features=16385), "supported"), (dict(out_features=20000), "supported"),
    (dict(n_groups=0), "positive"), (dict(n_groups=4097), "supported"),
    (dict(dtype=0), "GNN_BF16"), (dict(dtype=4), "unknown"), (dict(dtype=-1), "unknown")])
def test_linear_dims_refused(G, kw, code):
    d = G.make_linear_dims(**{**dict(in_features=8, out_features=8), **kw})
    assert G.gnn_linear_weight_count(d) == 0
    assert code in G.gnn_last_error()
    with pytest.raises(G.GnnError):
        G.gnn_linear_create(np.zeros(72, np.float32), d)


@pytest.mark.parametrize("widths,kw,text", [
    ([3, 0, 8], {}, "positive"), ([3, 5000, 8], {}, "hidden"), ([3, 64, 8], dict(ln_eps=0.0), "ln_eps"),
    ([3, 64, 8], dict(ln_eps=float("nan")), "ln_eps"), ([3, 64, 8], dict(dtype=0), "GNN_BF16"),
    ([3, 64, 8], dict(n_groups=0), "positive")])
def test_mlp_dims_refused(G, widths, kw, text):
    d = G.make_mlp_dims(widths, **kw)
    assert G.gnn_mlp_weight_count(d) == 0
    assert text in G.gnn_last_error()


def test_counts_and_struct_sizes(G):
    d = G.make_linear_dims(5, 7, 3, G.GNN_INT8)
    assert G.gnn_linear_weight_count(d) == 3 * (5 * 7 + 7)
    d.struct_size = 4
    assert G.gnn_linear_weight_count(d) == 0 and "struct_size" in G.gnn_last_error()
    m = G.make_mlp_dims([3, 16, 8], 2, G.GNN_BF16)
    assert G.gnn_mlp_weight_count(m) == 2 * (3 * 16 + 16 + 32 + 16 * 8 + 8)
    m.struct_size = 4
    assert G.gnn_mlp_weight_count(m) == 0 and "struct_size" in G.gnn_last_error()
    m = G.make_mlp_dims([3, 16, 8])
    m.n_layers = 9
    assert G.gnn_mlp_weight_count(m) == 0 and "n_layers" in G.gnn_last_error()
    with pytest.raises(ValueError):
        G.make_mlp_dims([3])
    with pytest.raises(ValueError):
        G.gnn_linear_create(np.zeros(5, np.float32), G.make_linear_dims(2, 2))


# Arguments are checked before any device call: the addresses below are never read.
X, Q, S = 1 << 20, 2 << 20, 3 << 20


@pytest.mark.parametrize("args,text", [
    ((X, 0, 8, -1, 8, Q, 8, S), "negative"), ((X, 3, 8, 4, 8, Q, 8, S), "float type"),
    ((X, 0, 8, 4, 0, Q, 8, S), "width"), ((None, 0, 8, 4, 8, Q, 8, S), "NULL"),
    ((X, 0, 7, 4, 8, Q, 8, S), "stride"), ((X, 0, 8, 4, 8, Q, 7, S), "stride"),
    ((X + 2, 0, 8, 4, 8, Q, 8, S), "aligned"), ((X + 1, 2, 8, 4, 8, Q, 8, S), "aligned"),
    ((X, 0, 8, 4, 8, Q, 8, None), "NULL"), ((X, 0, 8, 4, 8, None, 8, S), "NULL"),
    ((X, 0, 8, 4, 8, Q, 8, S + 2), "aligned"), ((X, 0, 1 << 40, 4, 8, Q, 8, S), "stride")])
def test_quantize_refuses(G, args, text):
    assert G.lib.gnn_quantize_rows(*args, None) == G.GNN_E_INVALID_ARG
    assert text in G.gnn_last_error()


def test_row_counts_refused(G):
    big = (1 << 30) + 1
    assert G.lib.gnn_quantize_rows(X, 0, 8, big, 8, Q, 8, S, None) == G.GNN_E_UNSUPPORTED
    assert G.lib.gnn_group_rows(X, big, 4, Q, S, None, 0, None) == G.GNN_E_UNSUPPORTED
    assert G.lib.gnn_quantize_rows(None, 0, 8, 0, 8, None, 8, None, None) == G.GNN_OK
    assert G.gnn_group_workspace(big, 4) == 0 and G.gnn_group_workspace(100, 0) == 0


@pytest.mark.parametrize("args,code,text", [
    ((X, 100, 0, Q, S, None, 0), -1, "n_groups"), ((X, 100, 4097, Q, S, None, 0), -6, "groups"),
    ((None, 100, 4, Q, S, None, 0), -1, "ids"), ((X, 100, 4, None, S, None, 0), -1, "offsets"),
    ((X, 100, 4, Q, None, None, 0), -1, "order"), ((X + 1, 100, 4, Q, S, None, 0), -1, "aligned"),
    ((X, 1 << 20, 4, Q, S, None, 0), -1, "workspace"),
    ((X, 1 << 20, 4, Q, S, 256, 16), -1, "workspace")])
def test_group_refuses(G, args, code, text):
    assert G.lib.gnn_group_rows(*args, None) == code
    assert text in G.gnn_last_error()


def test_null_handles(G):
    assert G.lib.gnn_linear_apply(None, X, 0, 8, None, 4, None, None, Q, 0, 8, None, 0, None) == -1
    assert G.lib.gnn_mlp_apply(None, X, 0, 8, None, 4, Q, 0, 8, None, 0, None) == -1
    assert G.gnn_linear_workspace(None, 0, 4) == 0 and G.gnn_mlp_workspace(None, 0, 4) == 0
    G.gnn_linear_destroy(None)
    G.gnn_mlp_destroy(None)
    d = G.make_linear_dims(2, 2)
    assert G.lib.gnn_linear_create(None, ctypes.byref(d)) is None
    m = G.make_mlp_dims([2, 2])
    assert G.lib.gnn_mlp_create(None, ctypes.byref(m)) is None


def test_binding_refuses_host_tensors(G):
    import torch
    with pytest.raises(ValueError):
        G.quantize_rows(torch.zeros(2, 2))
    with pytest.raises(ValueError):
        G.group_rows(torch.zeros(2, dtype=torch.int32), 2)


def test_plain_quantize_on_ties():
    # scale 1: 0.5 and 1.5 are ties, to even
    x = np.array([[127.0, 0.5, 1.5, -0.5, -2.5, np.float32(0.50000006)]], np.float32)
    q, s = R.quantize(x)
    assert s[0] == 1.0 and q.tolist() == [[127, 0, 2, 0, -2, 1]]
    q, s = R.quantize(np.array([[0.0, 0.0], [np.inf, 1.0], [1e-44, 0.0]], np.float32))
    assert s[0] == 0 and np.isnan(s[1]) and s[2] == 0 and not q.any()


def test_plain_group():
    off, order = R.group([2, 0, -1, 2, 5, 0], 3)
    assert off.tolist() == [0, 2, 2, 4] and order.tolist() == [1, 5, 0, 3, 2, 4]


@pytest.mark.parametrize("bits", [8, 11])
def test_16_bit_rounding_rule(bits):
    """The kernels round a 16-bit row to 8 bits by one multiply-add with a factor
    next to 127 / top, taken on the side that the rounding error of s = fl32(top /
    127) asks for (and both sides where s has none).  Over all mantissas of the
    largest value and of the others, and all exponents that do not round to 0, it
    must give the exact quotient's nearest whole number, ties to even."""
    lo, hi = 1 << (bits - 1), 1 << bits
    jx = np.arange(lo, hi, dtype=np.float64)
    xs = (jx[:, None] / 2.0 ** np.arange(10)).ravel()
    ties = 0
    for jm in range(lo, hi):
        top = np.float32(jm)
        s = np.float32(top / np.float32(127))
        d = float(s) * 127 - float(top)  # exact: 24 + 7 bits
        f = np.float32(np.float32(127) / top)
        e = float(f) * float(top) - 127.0
        below = np.nextafter(f, np.float32(0)) if e >= 0 else f
        above = np.nextafter(f, np.float32(np.inf)) if e <= 0 else f
        x = xs[xs <= jm]
        got = np.rint(x * float(below if d >= 0 else above))  # one rounding, as the fma's
        if d == 0:
            ties += 1
            got = np.rint(0.5 * (got + np.rint(x * float(above))))
        k = np.floor(x / float(s))
        r = 2 * (x - k * float(s))  # exact
        want = np.where(r > float(s), k + 1, np.where(r < float(s), k, k + k % 2))
        assert np.array_equal(got, want), jm
    assert ties > 0
