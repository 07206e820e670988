"""Refusals of the training operators that need no GPU."""
import ctypes

import numpy as np
import pytest


@pytest.fixture(scope="module")
def G():
    from paper_2402_09633_amd import gnn
    return gnn


# Arguments are checked before any device call: the addresses below are never read.
X, Y, V, W = 1 << 20, 2 << 20, 3 << 20, 4 << 20


@pytest.mark.parametrize("at,value,text", [
    (0, None, "NULL"), (0, X + 2, "aligned"), (1, 3, "float type"), (2, 7, "stride"),
    (2, 1 << 40, "stride"), (3, -1, "negative"), (4, 0, "positive"), (5, None, "NULL"),
    (6, V + 2, "aligned"), (7, 0.0, "eps"), (7, 1.5, "eps"), (8, None, "NULL"), (9, 7, "stride"),
    (10, None, "together"), (11, None, "together")])
def test_layer_norm_refuses(G, at, value, text):
    args = [X, 0, 8, 4, 8, V, V, 1e-5, Y, 8, W, W]
    args[at] = value
    assert G.lib.gnn_layer_norm(*args, None) == G.GNN_E_INVALID_ARG
    assert text in G.gnn_last_error()


@pytest.mark.parametrize("at,value,text", [
    (0, None, "NULL"), (1, 7, "stride"), (2, X + 1, "aligned"), (4, 9, "float type"),
    (5, -2, "negative"), (6, 0, "positive"), (7, None, "NULL"), (8, None, "NULL"), (9, W + 1, "aligned"),
    (10, None, "NULL"), (12, None, "NULL"), (13, None, "NULL"), (14, None, "workspace"),
    (14, W + 8, "256"), (15, 16, "workspace"), (15, -1, "workspace")])
def test_layer_norm_backward_refuses(G, at, value, text):
    args = [X, 8, X, 8, 0, 4, 8, V, V, V, Y, 8, W, W, W, 1 << 30]
    args[at] = value
    assert G.lib.gnn_layer_norm_backward(*args, None) == G.GNN_E_INVALID_ARG
    assert text in G.gnn_last_error()


def test_sizes_refused(G):
    big = (1 << 28) + 1
    assert G.lib.gnn_layer_norm(X, 0, 8, big, 8, V, V, 1e-5, Y, 8, W, W, None) == G.GNN_E_UNSUPPORTED
    assert G.lib.gnn_layer_norm(X, 0, 1 << 20, 1, 16385, V, V, 1e-5, Y, 1 << 20, W, W,
                                None) == G.GNN_E_UNSUPPORTED
    assert G.lib.gnn_layer_norm_workspace(big, 8) == 0
    assert G.lib.gnn_layer_norm_workspace(8, 16385) == 0
    assert G.lib.gnn_layer_norm(None, 0, 8, 0, 8, None, None, 1e-5, None, 8, None, None,
                                None) == G.GNN_OK


def _gated(G, **kw):
    d = G.make_gated_dims(8, 16, 8)
    w = G.gnn_gated_weights(ctypes.sizeof(G.gnn_gated_weights), W, W, W, None, None, None)
    for name, v in kw.items():
        setattr(d if hasattr(d, name) and name != "struct_size" else w, name, v)
    return d, w


@pytest.mark.parametrize("kw,code,text", [
    (dict(in_features=0), -1, "positive"), (dict(hidden=-3), -1, "positive"),
    (dict(out_features=16385), -6, "supported"), (dict(dtype=0), -6, "GNN_BF16"),
    (dict(dtype=3), -6, "GNN_BF16"), (dict(dtype=7), -1, "GNN_BF16"),
    (dict(activation=4), -1, "activation"), (dict(activation=-1), -1, "activation"),
    (dict(gate=None), -1, "gate is NULL"), (dict(down=None), -1, "down is NULL"),
    (dict(up=W + 1), -1, "aligned"), (dict(up_bias=W + 1), -1, "aligned"),
    (dict(struct_size=8), -1, "struct_size")])
def test_gated_refuses(G, kw, code, text):
    d, w = _gated(G, **kw)
    assert G.lib.gnn_gated(d, w, X, 8, 4, Y, 8, W, 1 << 30, None) == code
    assert text in G.gnn_last_error()
    _, dw = _gated(G, gate=V, up=V + 512, down=V + 1024)
    assert G.lib.gnn_gated_backward(d, w, X, 8, X, 8, 4, Y, 8, dw, W, 1 << 30, None) == code
    assert text in G.gnn_last_error()


@pytest.mark.parametrize("at,value,text", [
    (2, None, "NULL"), (2, X + 1, "aligned"), (3, 7, "stride"), (4, -1, "negative"),
    (5, None, "NULL"), (6, 7, "stride"), (7, None, "workspace"), (7, W + 128, "256"),
    (8, 100, "workspace")])
def test_gated_refuses_rows(G, at, value, text):
    args = [*_gated(G), X, 8, 4, Y, 8, W, 1 << 30]
    args[at] = value
    assert G.lib.gnn_gated(*args, None) == G.GNN_E_INVALID_ARG
    assert text in G.gnn_last_error()


def test_gated_scratch(G):
    d, w = _gated(G)
    big = (1 << 28) + 1
    assert G.lib.gnn_gated_workspace(d, big, 0, 1) == 0
    assert G.lib.gnn_gated_workspace(d, 0, 0, 1) == 0
    assert G.lib.gnn_gated_workspace(None, 5, 0, 1) == 0
    assert G.lib.gnn_gated(d, w, X, 8, big, Y, 8, W, 1, None) == G.GNN_E_UNSUPPORTED
    assert G.lib.gnn_gated(d, w, None, 8, 0, None, 8, None, 0, None) == G.GNN_OK
    # unaligned tables are copied first
    assert G.lib.gnn_gated_workspace(d, 1000, 0, 0) > G.lib.gnn_gated_workspace(d, 1000, 0, 1)
    assert G.lib.gnn_gated(d, w, X + 2, 8, 1000, Y, 8, W, G.lib.gnn_gated_workspace(d, 1000, 0, 1),
                           None) == G.GNN_E_INVALID_ARG
    d.struct_size = 4
    assert G.lib.gnn_gated_workspace(d, 5, 0, 1) == 0


def test_overlaps_are_refused(G):
    bad = G.GNN_E_INVALID_ARG
    d, w = _gated(G)
    args = [X, 0, 8, 4, 8, V, V, 1e-5, X, 16, W, W]
    assert G.lib.gnn_layer_norm(*args, None) == bad and "overlaps" in G.gnn_last_error()
    for dx, stride in ((X, 8), (Y, 16)):
        args = [Y, 8, X, 8, 0, 4, 8, V, V, V, dx, stride, W, W, W, 1 << 30]
        assert G.lib.gnn_layer_norm_backward(*args, None) == bad
        assert "overlaps" in G.gnn_last_error()
    assert G.lib.gnn_gated(d, w, X, 8, 4, X, 8, W, 1 << 30, None) == bad
    assert "overlaps" in G.gnn_last_error()
    apart = dict(gate=V, up=V + 512, down=V + 1024)
    for dx, kw in ((X, {}), (Y, {}), (X + 4096, dict(gate=W)), (X + 4096, dict(down=W)),
                   (X + 4096, dict(up=V)), (X + 4096, dict(down=V + 512))):
        _, dw = _gated(G, **{**apart, **kw})
        assert G.lib.gnn_gated_backward(d, w, Y, 8, X, 8, 4, dx, 8, dw, W, 1 << 30, None) == bad
        assert "overlap" in G.gnn_last_error()


def _list(G, *rows):
    t = np.zeros(len(rows), G._GRAD)
    for i, r in enumerate(rows):
        t[i] = (*r, 0)
    return t


@pytest.mark.parametrize("row,code,text", [
    ((X, X, 5, 3), -1, "float type"), ((X, X, -1, 0), -1, "negative"), ((0, X, 5, 0), -1, "NULL"),
    ((X, 0, 5, 0), -1, "NULL"), ((X + 2, X + 2, 5, 0), -1, "aligned"), ((X + 1, X, 5, 1), -1, "aligned"),
    ((X, X, (1 << 40) + 1, 0), -6, "2^40"), ((X, X, 1 << 39, 0), -6, "2^37"),
    ((X, X + 4, 5, 0), -1, "overlap")])
def test_clip_refuses(G, row, code, text):
    t = _list(G, (Y, Y, 4, 0), row)
    assert G.lib.gnn_clip_grads(t.ctypes.data, 2, 1.0, V, W, 1 << 30, None) == code
    assert text in G.gnn_last_error()
    if text != "overlap":
        assert G.lib.gnn_clip_workspace(t.ctypes.data, 2) == 0


def test_clip_refuses_the_rest(G):
    t = _list(G, (X, X, 4, 0))
    for args, text in (((None, 1, 1.0, V, W, 1 << 20), "NULL"), ((t.ctypes.data, -1, 1.0, V, W, 1 << 20), "count"),
                       ((t.ctypes.data, 1, 0.0, V, W, 1 << 20), "max_norm"),
                       ((t.ctypes.data, 1, 1.0, None, W, 1 << 20), "NULL"),
                       ((t.ctypes.data, 1, 1.0, V, None, 0), "workspace"),
                       ((t.ctypes.data, 1, 1.0, V, W + 4, 1 << 20), "256")):
        assert G.lib.gnn_clip_grads(*args, None) == G.GNN_E_INVALID_ARG
        assert text in G.gnn_last_error()


def test_counts_past_32_bits_are_refused(G):
    for kw in (dict(in_features=1 << 32), dict(hidden=1 << 31), dict(out_features=(1 << 32) + 8)):
        with pytest.raises(ValueError, match="32-bit"):
            G.make_gated_dims(**{**dict(in_features=8, hidden=8, out_features=8), **kw})
