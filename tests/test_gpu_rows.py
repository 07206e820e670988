"""Row operators on the GPU against their plain 64-bit forms: rows to 8 bits,
rows in group order, linear layers with one weight set per group, and networks
of them."""
import numpy as np
import pytest
import torch

from tests import rows_ref as R

pytestmark = pytest.mark.gpu
T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def G():
    from paper_2402_09633_amd import gnn
    return gnn


def _dtype(G, kind):
    return {"i8": G.GNN_INT8, "bf16": G.GNN_BF16, "f16": G.GNN_F16}[kind]


def _np(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _x(n, k, kind, seed, pitch=None, offset=0):
    """Rows in a wider table of NaN, so that what is read past a row shows."""
    rng = np.random.default_rng(seed)
    pitch = pitch or k
    t = torch.full((n * pitch + offset + 8,), float("nan"), dtype=T[kind], device="cuda")
    x = t[offset:offset + n * pitch].view(n, pitch)[:, :k]
    v = rng.normal(size=(n, k)) * np.exp(rng.normal(size=(n, 1)))
    x.copy_(torch.as_tensor(v))
    return x


# ------------------------------------------------------------ rows to 8 bits

@pytest.mark.parametrize("kind", R.FLOATS)
@pytest.mark.parametrize("n,k,pitch,offset", [
    (1, 1, 1, 0), (3, 7, 9, 1), (65, 8, 8, 0), (130, 64, 64, 0), (31, 65, 70, 3), (257, 128, 128, 0),
    (19, 509, 515, 5), (9, 513, 513, 1), (5, 1031, 1031, 0), (3, 2049, 2050, 1), (2, 4096, 4096, 0),
    (3, 4097, 4099, 1), (2, 16384, 16384, 0), (1000, 3, 3, 0)])
def test_quantize(G, kind, n, k, pitch, offset):
    print(f"quantize {kind} {n}x{k} pitch {pitch} offset {offset}", flush=True)
    x = _x(n, k, kind, n * 131 + k, pitch, offset)
    out = torch.full((n, k + 3), 99, dtype=torch.int8, device="cuda")
    q, s = G.quantize_rows(x, out=(out[:, 1:k + 1], torch.empty(n, device="cuda")))
    qr, sr = R.quantize(_np(x))
    assert np.array_equal(_np(s), sr)
    assert np.array_equal(_np(q), qr)
    assert (out[:, 0] == 99).all() and (out[:, k + 1:] == 99).all()


def test_quantize_ties_and_extremes(G):
    # every multiple of a half step of a scale that is a power of two, and of
    # scales that are not, in bf16 and fp32
    half = np.arange(-254, 255) / 2.0
    rows = [half * f for f in (1.0, 2.0 ** -20, 3.0, 127.0, 1.7, 2.0 ** 100, 2.0 ** -130)]
    x = torch.as_tensor(np.stack(rows), dtype=torch.float32, device="cuda")
    for t in (x, x.to(torch.bfloat16)):
        q, s = G.quantize_rows(t)
        qr, sr = R.quantize(_np(t))
        assert np.array_equal(_np(s), sr) and np.array_equal(_np(q), qr)
    y = torch.zeros(6, 20, device="cuda")
    y[1, 3] = float("inf")
    y[2, 19] = float("nan")
    y[3, :] = 1e-40
    y[4, 7] = -3.0e38
    y[5, 0] = -float("inf")
    q, s = G.quantize_rows(y)
    qr, sr = R.quantize(_np(y))
    assert np.array_equal(_np(s), sr, equal_nan=True) and np.array_equal(_np(q), qr)
    assert np.isnan(_np(s)[[1, 2, 5]]).all() and _np(s)[0] == 0 and _np(s)[3] == 0


def test_quantize_random_bits(G):
    rng = np.random.default_rng(3)
    bits = rng.integers(0, 1 << 32, size=(400, 96), dtype=np.uint32)
    x = bits.view(np.float32)
    x = np.where(np.isfinite(x), x, 0.0).astype(np.float32)
    q, s = G.quantize_rows(torch.as_tensor(x).cuda())
    qr, sr = R.quantize(x)
    assert np.array_equal(_np(s), sr) and np.array_equal(_np(q), qr)


# ------------------------------------------------------- rows in group order

@pytest.mark.parametrize("n,g", [(1, 1), (2, 5), (63, 2), (64, 3), (65, 64), (4095, 7), (4096, 4),
                                 (4097, 4), (10_000, 300), (70_001, 1), (50_003, 4096),
                                 (300_000, 16), (3_000_001, 5), (3000, 2000), (4096, 900),
                                 (8192, 899), (8193, 899), (2048, 3), (2049, 3), (1_200_000, 60)])
def test_group(G, n, g):
    print(f"group {n} rows {g} groups", flush=True)
    rng = np.random.default_rng(n + g)
    ids = rng.integers(-1, g + 1, size=n).astype(np.int32)
    ids[rng.random(n) < 0.01] = 2 ** 31 - 1
    ids[rng.random(n) < 0.01] = -2 ** 31
    off, order = G.group_rows(torch.as_tensor(ids).cuda(), g)
    offr, orderr = R.group(ids, g)
    assert np.array_equal(_np(off), offr) and np.array_equal(_np(order), orderr)


def test_group_one_value_and_empty(G):
    for v, g in ((0, 3), (2, 3), (7, 3)):
        ids = torch.full((9001,), v, dtype=torch.int32, device="cuda")
        off, order = G.group_rows(ids, g)
        offr, orderr = R.group(_np(ids), g)
        assert np.array_equal(_np(off), offr) and np.array_equal(_np(order), orderr)
    off, order = G.group_rows(torch.empty(0, dtype=torch.int32, device="cuda"), 4)
    assert _np(off).tolist() == [0] * 5 and order.numel() == 0


# --------------------------------------------------------------- linear layer

def _weights(g, n, k, seed):
    rng = np.random.default_rng(seed)
    return (rng.normal(size=(g, n, k)) / np.sqrt(k)).astype(np.float32), \
        rng.normal(size=(g, n)).astype(np.float32)


def _layer(G, w, b, kind):
    g, n, k = w.shape
    blob = np.concatenate([w.reshape(g, -1), b], axis=1)
    return G.Linear(blob.ravel(), G.make_linear_dims(k, n, g, _dtype(G, kind)))


def _held(a, kind):
    """fp32 values as a 16-bit layer holds them."""
    return a if kind == "i8" else _np(torch.as_tensor(a).to(T[kind]))


def _check(y, x, w, b, kind, out, what=""):
    ref, bound = R.linear(_held(x, kind), _held(w, kind), b, kind)
    lim = R.stored(ref, bound, out)
    err = np.abs(np.asarray(y, np.float64) - ref)
    assert err.shape == lim.shape
    worst = (err / lim).max() if err.size else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3f} of the bound"


SHAPES = [(1, 1, 1), (1, 512, 512), (3, 9, 33), (33, 31, 65), (64, 64, 32), (129, 128, 96),
          (200, 391, 259), (65, 513, 40), (70, 1025, 129), (40, 2050, 257), (17, 4096, 64),
          (300, 300, 520)]


@pytest.mark.parametrize("kind", ["i8", "bf16", "f16"])
@pytest.mark.parametrize("m,k,n", SHAPES)
def test_linear(G, kind, m, k, n):
    w, b = _weights(1, n, k, m + k + n)
    layer = _layer(G, w, b, kind)
    for xt in R.FLOATS:
        for out in R.FLOATS:
            print(f"linear {kind} {m}x{k}->{n} x {xt} y {out}", flush=True)
            x = _x(m, k, xt, m * k + n, k + 3, 1)
            table = torch.full((m, n + 5), 7.0, dtype=T[out], device="cuda")
            y = layer(x, out=table[:, 2:n + 2])
            _check(_np(y), _np(x), w[0], b[0], kind, out, f"{xt} {out}")
            assert (table[:, :2] == 7).all() and (table[:, n + 2:] == 7).all()


@pytest.mark.parametrize("kind", ["i8", "bf16", "f16"])
@pytest.mark.parametrize("m,k,n", [(3, 9000, 70), (140, 5001, 40), (1000, 4097, 300)])
def test_linear_wide_rows(G, kind, m, k, n):
    w, b = _weights(1, n, k, 5)
    layer = _layer(G, w, b, kind)
    for xt in (["f32", "bf16"] if kind == "i8" else ["f32", kind]):
        x = _x(m, k, xt, m, k + 1, 1)
        _check(_np(layer(x, out_dtype=torch.float32)), _np(x), w[0], b[0], kind, "f32", xt)


def test_linear_more_tiles_than_cus(G):
    # several row tiles per CU, the output split and not split
    for m, k, n in ((70_001, 40, 72), (9_000, 96, 1100)):
        w, b = _weights(1, n, k, 9)
        for kind in ("i8", "bf16"):
            x = _x(m, k, "bf16", 4)
            _check(_np(_layer(G, w, b, kind)(x)), _np(x), w[0], b[0], kind, "bf16")


# Sizes that the tiles for wide layers take: 128 and 256 rows to a tile, widths
# that are whole chunks of 16 bytes, and others, whose rows are copied first.
@pytest.mark.parametrize("kind,xt,m,k,n", [
    ("bf16", "bf16", 4100, 640, 1100), ("bf16", "bf16", 4100, 643, 1100),
    ("f16", "f16", 14_001, 520, 1400), ("f16", "f32", 4100, 650, 1030),
    ("bf16", "f16", 4100, 520, 1027), ("i8", "bf16", 4100, 1000, 1100),
    ("i8", "f32", 14_001, 901, 1300), ("i8", "i8", 4100, 1040, 1100),
    ("i8", "i8", 4100, 1101, 1100), ("bf16", "bf16", 2000, 2056, 2100)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_linear_tiles(G, kind, xt, m, k, n, out):
    print(f"tiles {kind} {m}x{k}->{n} x {xt} y {out}", flush=True)
    w, b = _weights(1, n, k, m + k)
    layer = _layer(G, w, b, kind)
    x = _x(m, k, "f32" if xt == "i8" else xt, k, k + 3, 1)
    scales = None
    xs = _np(x)
    if xt == "i8":
        table = torch.full((m * (k + 3) + 1,), 77, dtype=torch.int8, device="cuda")
        q = table[1:].view(m, k + 3)[:, :k]
        x, scales = G.quantize_rows(x, out=(q, torch.empty(m, device="cuda")))
    table = torch.full((m, n + 5), 7.0, dtype=T[out], device="cuda")
    y = layer(x, scales=scales, out=table[:, 2:n + 2])
    _check(_np(y), xs, w[0], b[0], kind, out, f"{xt} {out}")
    assert (table[:, :2] == 7).all() and (table[:, n + 2:] == 7).all()


@pytest.mark.parametrize("kind", ["i8", "bf16", "f16"])
@pytest.mark.parametrize("m,k,n,g,ordered", [(6000, 1032, 1100, 3, True), (9000, 1001, 1064, 5, False),
                                             (17_000, 904, 1100, 7, True)])
def test_grouped_tiles(G, kind, m, k, n, g, ordered):
    print(f"grouped tiles {kind} {m}x{k}->{n} {g} groups", flush=True)
    rng = np.random.default_rng(m)
    sizes = _sizes("ragged", g, m - 50, rng)
    w, b = _weights(g, n, k, g)
    x = _x(m, k, "bf16" if kind == "i8" else kind, g)
    off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32) + 20  # 20 rows before, 30 behind
    order = rng.permutation(m).astype(np.int32) if ordered else np.arange(m, dtype=np.int32)
    out = torch.full((m, n), 7.0, device="cuda")
    y = _np(_layer(G, w, b, kind)(x, offsets=torch.as_tensor(off).cuda(),
                                  order=torch.as_tensor(order).cuda() if ordered else None, out=out))
    xs = _np(x)
    for i in range(g):
        rows = order[off[i]:off[i + 1]][:400]  # enough of each group
        if len(rows):
            _check(y[rows], xs[rows], w[i], b[i], kind, "f32", f"group {i}")
    rest = np.concatenate([order[:off[0]], order[off[-1]:]])
    assert len(rest) == 50 and (y[rest] == 7.0).all()


@pytest.mark.parametrize("m,k", [(3000, 4096), (3000, 2100), (40, 16384)])
def test_linear_one_block_of_channels(G, m, k):
    w, b = _weights(1, 20, k, 1)
    for kind in ("i8", "bf16"):
        x = _x(m, k, "bf16", 4)
        _check(_np(_layer(G, w, b, kind)(x, out_dtype=torch.float32)), _np(x), w[0], b[0], kind,
               "f32")


@pytest.mark.parametrize("m,k,n", [(1, 64, 32), (77, 100, 50), (500, 387, 130), (3, 6001, 20),
                                   (2500, 1024, 640)])
def test_linear_given_8_bit_rows(G, m, k, n):
    w, b = _weights(1, n, k, 11)
    layer = _layer(G, w, b, "i8")
    x = _x(m, k, "f32", 12)
    table = torch.full((m, k + 3), 77, dtype=torch.int8, device="cuda")
    q, s = G.quantize_rows(x, out=(table[:, :k], torch.empty(m, device="cuda")))
    y = layer(q, scales=s)
    assert y.dtype == torch.float32
    _check(_np(y), _np(x), w[0], b[0], "i8", "f32")
    assert torch.equal(y, layer(x))  # rounded while staged, or before: the same values


def _sizes(kind, g, m, rng):
    if kind == "even":
        return np.full(g, m // g)
    if kind == "one":
        s = np.zeros(g, np.int64)
        s[g // 2] = m
        return s
    p = rng.exponential(size=g) * (rng.random(g) > 0.3)
    p[0] += 1e-3
    return rng.multinomial(m, p / p.sum())


@pytest.mark.parametrize("kind", ["i8", "bf16", "f16"])
@pytest.mark.parametrize("m,k,n,g,how", [
    (1, 16, 8, 3, "one"), (5, 40, 33, 9, "ragged"), (64, 64, 64, 64, "ragged"),
    (300, 130, 70, 4, "ragged"), (300, 96, 160, 5, "even"), (2000, 77, 129, 70, "ragged"),
    (513, 200, 64, 130, "one"), (40_000, 64, 96, 17, "ragged"), (1500, 1030, 65, 6, "ragged"),
    (4000, 520, 640, 3, "ragged"), (700, 33, 20, 1000, "ragged")])
@pytest.mark.parametrize("ordered", [False, True])
def test_grouped(G, kind, m, k, n, g, how, ordered):
    print(f"grouped {kind} {m}x{k}->{n} {g} groups {how} ordered {ordered}", flush=True)
    rng = np.random.default_rng(m + g)
    sizes = _sizes(how, g, m, rng)
    spare = m - int(sizes.sum())  # rows of no group
    w, b = _weights(g, n, k, g)
    layer = _layer(G, w, b, kind)
    xt = "f32" if kind == "i8" else kind
    x = _x(m, k, xt, g)
    off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    order = rng.permutation(m).astype(np.int32) if ordered else np.arange(m, dtype=np.int32)
    out = torch.full((m, n), 7.0, device="cuda")
    y = _np(layer(x, offsets=torch.as_tensor(off).cuda(),
                  order=torch.as_tensor(order).cuda() if ordered else None, out=out))
    xs = _np(x)
    for i in range(g):
        rows = order[off[i]:off[i + 1]]
        if len(rows):
            _check(y[rows], xs[rows], w[i], b[i], kind, "f32", f"group {i}")
    assert (y[order[off[-1]:]] == 7.0).all() and len(order[off[-1]:]) == spare


def test_rows_in_no_group_keep_their_values(G):
    w, b = _weights(3, 40, 24, 1)
    layer = _layer(G, w, b, "bf16")
    x = _x(500, 24, "bf16", 2)
    off = torch.tensor([100, 100, 230, 400], dtype=torch.int32, device="cuda")
    out = torch.full((500, 40), 3.0, device="cuda")
    y = _np(layer(x, offsets=off, out=out))
    assert (y[:100] == 3).all() and (y[400:] == 3).all()
    _check(y[100:230], _np(x)[100:230], w[1], b[1], "bf16", "f32")
    _check(y[230:400], _np(x)[230:400], w[2], b[2], "bf16", "f32")
    new = _np(layer(x, offsets=off, out_dtype=torch.float32))
    assert (new[:100] == 0).all() and (new[400:] == 0).all()
    assert np.array_equal(new[100:400], y[100:400])


def test_order_without_groups(G):
    w, b = _weights(1, 40, 24, 1)
    for kind in ("bf16", "i8"):
        x = _x(700, 24, "bf16", 2)
        order = torch.as_tensor(np.random.default_rng(1).permutation(700).astype(np.int32)).cuda()
        layer = _layer(G, w, b, kind)
        assert torch.equal(layer(x, order=order), layer(x))
        # a row named twice, with the same weights, has its one result; a row
        # that no position names keeps its value
        order[5] = order[6]
        out = torch.full((700, 40), 2.0, device="cuda")
        y = layer(x, order=order, out=out)
        named = torch.zeros(700, dtype=torch.bool, device="cuda")
        named[order.long()] = True
        assert torch.equal(y[named], layer(x, out_dtype=torch.float32)[named])
        assert int((~named).sum()) == 1 and (y[~named] == 2).all()


def test_one_group_by_its_offsets(G):
    w, b = _weights(1, 33, 24, 1)
    layer = _layer(G, w, b, "bf16")
    x = _x(300, 24, "bf16", 2)
    off = torch.tensor([37, 205], dtype=torch.int32, device="cuda")
    y = layer(x, offsets=off, out=torch.full((300, 33), 2.0, device="cuda"))
    assert (y[:37] == 2).all() and (y[205:] == 2).all()
    _check(_np(y)[37:205], _np(x)[37:205], w[0], b[0], "bf16", "f32")


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_every_row_its_own_group(G, kind):
    m = 500
    w, b = _weights(m, 9, 20, 1)
    x = _x(m, 20, "bf16", 2)
    off = torch.arange(m + 1, dtype=torch.int32, device="cuda")
    y = _np(_layer(G, w, b, kind)(x, offsets=off, out_dtype=torch.float32))
    for i in range(0, m, 7):
        _check(y[i:i + 1], _np(x)[i:i + 1], w[i], b[i], kind, "f32", f"row {i}")


@pytest.mark.parametrize("kind", ["i8", "bf16", "f16"])
def test_not_finite_rows_stay_alone(G, kind):
    w, b = _weights(1, 70, 50, 1)
    layer = _layer(G, w, b, kind)
    x = _x(100, 50, "f32", 2)
    clean = _np(layer(x))
    x[17, 49] = float("inf")
    x[40, 0] = float("nan")
    y = _np(layer(x))
    keep = np.ones(100, bool)
    keep[[17, 40]] = False
    assert np.array_equal(y[keep], clean[keep])
    assert not np.isfinite(y[17]).any() and np.isnan(y[40]).all()
    # a weight that is not finite: its channel alone
    w[0, 5, 3] = float("nan")
    y = _np(_layer(G, w, b, kind)(_x(100, 50, "f32", 2)))
    assert np.isnan(y[:, 5]).all() and np.array_equal(np.delete(y, 5, 1), np.delete(clean, 5, 1))


def test_zero_rows_and_zero_channels(G):
    w, b = _weights(1, 40, 30, 1)
    w[0, 7] = 0.0
    for kind in ("i8", "bf16"):
        x = _x(50, 30, "f32", 2)
        x[3] = 0.0
        y = _np(_layer(G, w, b, kind)(x))
        assert np.array_equal(y[3], b[0]) and (y[:, 7] == b[0, 7]).all()


def test_no_rows(G):
    w, b = _weights(2, 8, 4, 1)
    layer = _layer(G, w, b, "bf16")
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert layer(torch.empty(0, 4, device="cuda"), offsets=off).shape == (0, 8)
    y = layer(torch.ones(5, 4, device="cuda"), offsets=off, out=torch.full((5, 8), 2.0, device="cuda"))
    assert (y == 2).all()


def test_offsets_and_order_out_of_range_are_clamped(G):
    """Nonsense in, nonsense out; rows of sound positions are right and nothing
    outside the output is written."""
    w, b = _weights(4, 33, 20, 1)
    layer = _layer(G, w, b, "bf16")
    x = _x(100, 20, "bf16", 3)
    table = torch.full((102, 33), 5.0, device="cuda")
    for off in ([-5, 10, 400, 20, 1 << 30], [7, 3, -1, 90, 100], [200, 200, 200, 200, 200]):
        o = torch.tensor(off, dtype=torch.int32, device="cuda")
        layer(x, offsets=o, out=table[1:101])
        torch.cuda.synchronize()
        assert (table[0] == 5).all() and (table[101] == 5).all()
    order = torch.arange(100, dtype=torch.int32, device="cuda")
    order[50] = -7
    order[51] = 1 << 30
    off = torch.tensor([0, 50, 52, 52, 100], dtype=torch.int32, device="cuda")
    y = _np(layer(x, offsets=off, order=order, out=table[1:101]))
    assert (table[0] == 5).all() and (table[101] == 5).all()
    _check(y[1:50], _np(x)[1:50], w[0], b[0], "bf16", "f32")
    _check(y[52:99], _np(x)[52:99], w[3], b[3], "bf16", "f32")


def test_same_result_every_time_and_in_every_split(G):
    w, b = _weights(1, 300, 260, 1)
    for kind in ("i8", "bf16", "f16"):
        layer = _layer(G, w, b, kind)
        x = _x(5000, 260, "f32", 3)
        y = layer(x)
        assert all(torch.equal(y, layer(x)) for _ in range(3))
        if kind == "i8":  # exact sums: the same for any number of rows
            assert torch.equal(y[:7], layer(x[:7])) and torch.equal(y[100:1000], layer(x[100:1000]))


def test_layer_refusals(G):
    w, b = _weights(2, 8, 6, 1)
    layer = _layer(G, w, b, "bf16")
    x = torch.ones(5, 6, device="cuda")
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(G.GnnError, match="offsets"):
        layer(x)
    with pytest.raises(G.GnnError, match="INT8"):
        layer(x.to(torch.int8), offsets=off)
    with pytest.raises(G.GnnError, match="x_scales"):
        layer(x, scales=torch.ones(5, device="cuda"), offsets=off)
    with pytest.raises(ValueError, match="rows of 5"):
        layer(torch.ones(5, 5, device="cuda"), offsets=off)
    with pytest.raises(ValueError, match="contiguous"):
        layer(torch.ones(6, 5, device="cuda").t(), offsets=off)
    with pytest.raises(ValueError, match="overlap"):
        layer(x[:1].expand(5, 6), offsets=off)
    with pytest.raises(TypeError):
        layer(x, offsets=off.long())
    with pytest.raises(TypeError):
        layer(x, offsets=off[:2])
    with pytest.raises(TypeError):
        layer(x.double(), offsets=off)
    with pytest.raises(ValueError, match="4 rows"):
        layer(x, offsets=off, out=torch.ones(4, 8, device="cuda"))
    with pytest.raises(G.GnnError, match="y_type"):
        layer(x, offsets=off, out=torch.ones(5, 8, dtype=torch.int8, device="cuda"))
    i8 = _layer(G, w[:1], b[:1], "i8")
    with pytest.raises(G.GnnError, match="x_scales"):
        i8(x.to(torch.int8))
    wide = _layer(G, *_weights(1, 8, 5000, 1), "i8")
    need = G.gnn_linear_workspace(wide.handle, G.GNN_FP32, 5)
    assert need > 0 and G.gnn_linear_workspace(wide.handle, G.GNN_INT8, 5) == 0
    xw, y = torch.ones(5, 5000, device="cuda"), torch.full((5, 8), 9.0, device="cuda")
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    for p, nb in ((None, need), (ws, need - 1)):
        with pytest.raises(G.GnnError, match="workspace"):
            G.gnn_linear_apply(wide.handle, xw, G.GNN_FP32, 5000, None, 5, None, None, y,
                               G.GNN_FP32, 8, p, nb)
    torch.cuda.synchronize()
    assert (y == 9).all()


def test_streams_and_graphs(G):
    """Calls of one layer on two streams at once, and two captured graphs that
    replay in turn with eager work between, against the eager results."""
    w, b = _weights(3, 200, 5000, 1)
    layer = _layer(G, w, b, "i8")  # wide float rows: the call takes scratch
    mlp = _mlp(G, [24, 96, 64, 8], 3, "i8", 5)[0]
    rng = np.random.default_rng(1)
    data = []
    for m in (300, 700):
        ids = torch.as_tensor(rng.integers(0, 3, m).astype(np.int32)).cuda()
        data.append((_x(m, 5000, "f32", m), ids, _x(m, 24, "bf16", m + 1)))

    def step(x, ids, z, stream=None):
        off, order = G.group_rows(ids, 3, stream=stream)
        return (layer(x, offsets=off, order=order, stream=stream), mlp(z, ids, stream=stream))

    want = [step(*d) for d in data]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in data]
    for _ in range(3):
        got = [step(*d, stream=s) for d, s in zip(data, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for g, r in zip(got, want) for p, q in zip(g, r))
    graphs, outs = [], []
    for d in data:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(*d))
        graphs.append(g)
    for k in range(3):
        for o in outs:
            for t in o:
                t.zero_()
        for g, s in zip(graphs, streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for g, r in zip(outs, want) for p, q in zip(g, r)), k
        eager = step(*data[k % 2])
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(eager, want[k % 2]))


def test_long_table_offsets_pass_32_bits(G):
    # rows behind 2^32 elements of the table
    k, n, pitch = 8, 8, 1 << 16
    m = (1 << 16) + 40
    table = torch.empty(m * pitch, dtype=torch.int8, device="cuda")
    x = table.view(m, pitch)[:, :k]
    x.copy_(torch.randint(-127, 128, (m, k), device="cuda", dtype=torch.int8))
    w, b = _weights(1, n, k, 1)
    s = torch.ones(m, device="cuda")
    y = torch.empty(m * pitch, dtype=torch.bfloat16, device="cuda").view(m, pitch)[:, :n]
    _layer(G, w, b, "i8")(x, scales=s, out=y)
    wq, ws = R.quantize(w[0])
    part = (_np(x).astype(np.float64) @ wq.astype(np.float64).T) * ws.astype(np.float64)
    lim = R.stored(part + b[0], 4 * 2.0 ** -24 * (np.abs(part) + np.abs(b[0])), "bf16")
    assert (np.abs(_np(y) - (part + b[0])) <= lim).all()


# ------------------------------------------------------------------- networks

def _mlp(G, widths, g, kind, seed):
    rng = np.random.default_rng(seed)
    layers, blob = [], []
    for i in range(len(widths) - 1):
        w, b = _weights(g, widths[i + 1], widths[i], seed + i)
        ga = be = None
        if i + 2 < len(widths):
            ga = (1 + 0.2 * rng.normal(size=b.shape)).astype(np.float32)
            be = (0.3 * rng.normal(size=b.shape)).astype(np.float32)
        for j in range(g):
            blob += [w[j].ravel(), b[j]] + ([ga[j], be[j]] if ga is not None else [])
        layers.append((w, b, ga, be))
    m = G.Mlp(np.concatenate(blob), G.make_mlp_dims(widths, g, _dtype(G, kind)))
    return m, layers


def _mlp_ref(x, layers, j, kind, eps=1e-5):
    """(y, bound) of group j's network in 64 bits.  The first layer's rows are
    rounded as the layer does; what hidden layers hand on is not rounded here:
    that rounding (half a step) and the fp32 arithmetic go into the bound, which
    is carried through the layers.  LayerNorm of v with errors e: the centred
    values move by e_i + mean e at most, and 1 / deviation by the part that |e|
    has of the centred values' norm."""
    for i, (w, b, ga, be) in enumerate(layers):
        if i == 0:
            a, e = R.linear(_held(x, kind), _held(w[j], kind), b[j], kind)
        else:
            W = np.asarray(_held(w[j], kind), np.float64)
            if kind == "i8":
                q, s = R.quantize(w[j])
                W = q.astype(np.float64) * s.astype(np.float64)[:, None]
                e = e + (a.max(axis=1, keepdims=True) + e.max(axis=1, keepdims=True)) / 254 * \
                    (1 + 2.0 ** -20)
            else:
                e = e + R.HALF_STEP[kind] * (a + e) + R.TINY[kind]
            size = (a + e) @ np.abs(W).T + np.abs(b[j])
            e = e @ np.abs(W).T + (a.shape[1] + 4) * 2.0 ** -23 * size
            a = a @ W.T + b[j]
        if ga is None:
            return a, e
        c = a - a.mean(axis=1, keepdims=True)
        sd = np.sqrt((c * c).mean(axis=1, keepdims=True) + eps)
        part = np.sqrt((e * e).mean(axis=1, keepdims=True)) / sd
        assert part.max() < 0.5
        n = c / sd
        en = (e + e.mean(axis=1, keepdims=True)) / sd / (1 - part) + np.abs(n) * part / (1 - part)
        a = np.maximum(n * ga[j] + be[j], 0.0)
        e = en * np.abs(ga[j]) + a.shape[1] * 2.0 ** -23 * (np.abs(n * ga[j]) + np.abs(be[j]))


@pytest.mark.parametrize("kind", ["bf16", "f16", "i8"])
@pytest.mark.parametrize("m,widths,g", [(1, [3, 40, 8], 1), (333, [3, 256, 8], 4),
                                        (1000, [12, 130, 5], 9), (257, [70, 64, 72, 6], 3),
                                        (50, [5, 1030, 3], 2)])
def test_mlp_against_the_formula(G, kind, m, widths, g):
    print(f"mlp {kind} {m} rows {widths} {g} groups", flush=True)
    mlp, layers = _mlp(G, widths, g, kind, m)
    x = _x(m, widths[0], "f32", m, widths[0] + 2)
    ids = np.random.default_rng(m).integers(0, g, m).astype(np.int32)
    y = _np(mlp(x, torch.as_tensor(ids).cuda() if g > 1 else None))
    for j in range(g):
        rows = np.nonzero(ids == j)[0]
        if len(rows):
            ref, bound = _mlp_ref(_np(x)[rows], layers, j, kind)
            assert (np.abs(y[rows] - ref) <= R.stored(ref, bound, "f32")).all()


def test_grouped_mlp_equals_one_network_per_group(G):
    # sums of 8-bit products are exact: the same however rows are tiled
    kind, widths, g, m = "i8", [9, 200, 64, 7], 4, 3000
    mlp, layers = _mlp(G, widths, g, kind, 1)
    x = _x(m, widths[0], "bf16", 2)
    ids = np.random.default_rng(3).integers(-1, g + 1, m).astype(np.int32)
    out = torch.full((m, 7), 4.0, device="cuda")
    y = mlp(x, torch.as_tensor(ids).cuda(), out=out)
    for j in range(g):
        blob = []
        for w, b, ga, be in layers:
            blob += [w[j].ravel(), b[j]] + ([ga[j], be[j]] if ga is not None else [])
        one = G.Mlp(np.concatenate(blob), G.make_mlp_dims(widths, 1, _dtype(G, kind)))
        rows = torch.as_tensor(np.nonzero(ids == j)[0]).cuda()
        assert torch.equal(one(x[rows], out_dtype=torch.float32), y[rows])
    assert (_np(y)[(ids < 0) | (ids >= g)] == 4.0).all()


def test_mlp_with_wide_hidden_layers(G):
    # a hidden layer that the tiles take, with rows that have to be copied first
    widths, m = [20, 1101, 1100, 4], 4100
    x = _x(m, 20, "f32", 5)
    mlp, layers = _mlp(G, widths, 1, "bf16", 3)
    ref, bound = _mlp_ref(_np(x), layers, 0, "bf16")
    assert (np.abs(_np(mlp(x)) - ref) <= R.stored(ref, bound, "f32")).all()
    # sums of 8-bit products are exact: a small call, which the row panels take,
    # gives the same bits
    mlp, layers = _mlp(G, widths, 1, "i8", 3)
    assert torch.equal(mlp(x)[:300], mlp(x[:300]))


def test_one_layer_mlp_is_a_linear_layer(G):
    mlp, layers = _mlp(G, [50, 30], 1, "i8", 1)
    x = _x(400, 50, "f32", 2)
    assert torch.equal(mlp(x), _layer(G, layers[0][0], layers[0][1], "i8")(x))


def test_mlp_refusals(G):
    mlp, _ = _mlp(G, [6, 16, 4], 3, "bf16", 1)
    one, _ = _mlp(G, [6, 16, 4], 1, "bf16", 1)
    x, ids = torch.ones(5, 6, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda")
    with pytest.raises(G.GnnError, match="group_ids"):
        mlp(x)
    with pytest.raises(G.GnnError, match="group_ids"):
        one(x, ids)
    with pytest.raises(G.GnnError, match="x_type"):
        one(x.to(torch.int8))
    with pytest.raises(TypeError):
        mlp(x, ids[:4])
    with pytest.raises(TypeError):
        mlp(x, ids.long())
    with pytest.raises(ValueError):
        mlp(torch.ones(5, 7, device="cuda"), ids)
    assert one(x[:0]).shape == (0, 4) and mlp(x[:0], ids[:0]).shape == (0, 4)
    need = G.gnn_mlp_workspace(mlp.handle, G.GNN_FP32, 5)
    ws, y = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.full((5, 4), 9.0, device="cuda")
    with pytest.raises(G.GnnError, match="workspace"):
        G.gnn_mlp_apply(mlp.handle, x, G.GNN_FP32, 6, ids, 5, y, G.GNN_FP32, 4, ws, need - 1)
    torch.cuda.synchronize()
    assert (y == 9).all()
    G.gnn_mlp_apply(mlp.handle, x, G.GNN_FP32, 6, ids, 5, y, G.GNN_FP32, 4, ws, need)
    assert torch.equal(y, mlp(x, ids))


def test_wide_embedding_feeds_the_radius_search(G):
    """Hits of several regions through a wide 8-bit network and on to the pair
    search: the pairs are those of the network's own output."""
    mlp, _ = _mlp(G, [3, 320, 320, 8], 4, "i8", 7)
    rng = np.random.default_rng(8)
    x = torch.as_tensor(rng.normal(size=(2000, 3)).astype(np.float32)).cuda()
    ids = torch.as_tensor(rng.integers(0, 4, 2000).astype(np.int32)).cuda()
    z = mlp(x, ids)
    zz = _np(z).astype(np.float64)
    alld = ((zz[:, None, :] - zz[None, :, :]) ** 2).sum(axis=2)
    r2 = float(np.quantile(alld[np.triu_indices(2000, 1)], 0.002))
    pairs = _np(G.radius_graph(z, r2))
    d = ((zz[pairs[0]] - zz[pairs[1]]) ** 2).sum(axis=1)
    assert pairs.shape[1] > 0 and (d < r2 * (1 + 1e-6)).all()
    sure = np.count_nonzero(np.triu(alld < r2 * (1 - 1e-6), 1))
    maybe = np.count_nonzero(np.triu(alld < r2 * (1 + 1e-6), 1))
    assert sure <= pairs.shape[1] <= maybe
