"""Row operators on the GPU at the ends of their ranges: the smallest scales, the
widest rows and the most rows."""
import numpy as np
import pytest
import torch

from tests import rows_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    from paper_2402_09633_amd import gnn
    return gnn


def _next_to_halves(scale_bits, seed):
    """fp32 rows whose scales have the given binade (bits of the scale's exponent
    field), and whose values are the numbers to both sides of every half step:
    the quotients are as near to a half as they can be."""
    rng = np.random.default_rng(seed)
    m = rng.integers(1 << 23, 1 << 24, size=64, dtype=np.int64)
    m[:4] = [1 << 23, (1 << 23) + 1, (1 << 24) - 1, (1 << 24) - 2]
    unit = 2.0 ** (scale_bits - 150)  # an ulp of the scales
    tops = (127.0 * m * unit).astype(np.float32)
    s = (tops.astype(np.float64) / 127.0).astype(np.float32).astype(np.float64)
    h = np.concatenate([np.arange(0.5, 126.5), -np.arange(0.5, 126.5)])
    at = (h[None, :] * s[:, None]).astype(np.float32)
    x = np.concatenate([tops[:, None], at, np.nextafter(at, np.float32(np.inf)),
                        np.nextafter(at, np.float32(-np.inf))], axis=1).astype(np.float32)
    return x


@pytest.mark.parametrize("scale_bits", [1, 2, 3, 24, 25, 126, 127, 128, 200, 246, 247])
def test_quotients_next_to_a_half(G, scale_bits):
    # at scale_bits 1 (scales from 2^-126 to 2^-125) half an ulp of the scale is
    # below the smallest fp32 number
    x = _next_to_halves(scale_bits, scale_bits)
    assert np.isfinite(x).all()
    qr, sr = R.quantize(x)
    assert (sr > 0).all()
    q, s = G.quantize_rows(torch.as_tensor(x).cuda())
    assert np.array_equal(s.cpu().numpy(), sr)
    wrong = np.argwhere(q.cpu().numpy() != qr)
    assert len(wrong) == 0, f"{len(wrong)} of {x.size}, the first at {wrong[:1]}"


def test_layers_round_the_smallest_rows_and_weights_alike(G):
    # rows rounded while they are staged, and the weights' own rounding
    x = _next_to_halves(1, 5)
    k = x.shape[1]
    w = _next_to_halves(1, 6)[:40]
    unit = np.eye(k, dtype=np.float32)[:200]  # rows that pick single columns: q = 127, scale 1 / 127
    layer = G.Linear(np.concatenate([w.ravel(), np.zeros(len(w), np.float32)]),
                     G.make_linear_dims(k, len(w), 1, G.GNN_INT8))
    wq, ws = R.quantize(w)
    us = np.float32(1.0 / 127.0)
    want = (wq.T[:200].astype(np.float32) * 127 * ws[None, :]) * us
    got = layer(torch.as_tensor(unit).cuda()).cpu().numpy()
    # products of small numbers, the last of which may round to a subnormal one
    assert (np.abs(got - want) <= 2.0 ** -149 + 2.0 ** -23 * np.abs(want)).all()
    ones = np.zeros((64, k), np.float32)
    ones[:, :64] = np.eye(64)
    pick = G.Linear(np.concatenate([ones.ravel(), np.zeros(64, np.float32)]),
                    G.make_linear_dims(k, 64, 1, G.GNN_INT8))
    xq, xs = R.quantize(x)
    want = (xq[:, :64].astype(np.float32) * 127 * us) * xs[:, None]
    got = pick(torch.as_tensor(x).cuda()).cpu().numpy()
    assert (np.abs(got - want) <= 2.0 ** -149 + 2.0 ** -23 * np.abs(want)).all()


def test_smallest_scales_of_16_bit_rows(G):
    # bf16 rows with scales around 2^-126, below which a row counts as zero
    rng = np.random.default_rng(2)
    tops = torch.as_tensor(np.ldexp(rng.uniform(0.9, 2.2, 300), -119).astype(np.float32))
    x = torch.as_tensor(rng.uniform(-1, 1, (300, 200)).astype(np.float32)) * tops[:, None]
    x[:, 0] = tops
    x = x.to(torch.bfloat16)
    qr, sr = R.quantize(x.float().numpy())
    assert (sr == 0).any() and (sr > 0).any()
    q, s = G.quantize_rows(x.cuda())
    assert np.array_equal(s.cpu().numpy(), sr) and np.array_equal(q.cpu().numpy(), qr)


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("width", [(1 << 31) - 1, (1 << 31) - 2044])
def test_widest_row(G, kind, width):
    """A row of as many elements as a width can count: the step past its end is
    beyond 2^31."""
    print(f"widest row {width} {kind}", flush=True)
    x = torch.empty(width, dtype=kind, device="cuda")
    part = 1 << 27
    gen = torch.Generator(device="cuda").manual_seed(1)
    top = 0.0
    for i in range(0, width, part):
        n = min(part, width - i)
        x[i:i + n] = torch.randn(n, device="cuda", generator=gen)
        top = max(top, float(x[i:i + n].float().abs().max()))
    x[-1] = 3 * top
    out = torch.full((width + 8,), 99, dtype=torch.int8, device="cuda")
    s = torch.empty(1, device="cuda")
    G.quantize_rows(x.view(1, width), out=(out[:width].view(1, width), s))
    want = np.float32(float(x[-1].float()) / 127.0)
    assert s.item() == float(want)
    assert (out[width:] == 99).all() and out[width - 1] == 127
    for i in range(0, width, part):
        n = min(part, width - i)
        q = torch.round(x[i:i + n].double() / float(want)).to(torch.int8)
        assert torch.equal(out[i:i + n], q), i


@pytest.mark.parametrize("width,short", [(65, 0), (70, 15)])
def test_most_rows(G, width, short):
    """As many rows as a call takes, of a width at which a workgroup of 256 threads
    holds 16 rows: a workgroup for every 16 would be 2^32 threads in one launch."""
    n = (1 << 28) - short
    print(f"most rows {n} x {width}", flush=True)
    x = torch.empty(n, width, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    part = 1 << 23
    base = torch.randn(part, width, device="cuda", generator=gen).to(torch.bfloat16)
    for i in range(0, n, part):  # the same rows a few places on, and of another size
        m = min(part, n - i)
        x[i:i + m] = torch.roll(base, i // part, 0)[:m] * (1.0 + i // part)
    q, s = G.quantize_rows(x)
    for i in range(0, n, part):
        xd = x[i:i + part].double()
        want = (xd.abs().amax(1) / 127.0).float()
        assert torch.equal(s[i:i + part], want), i
        assert torch.equal(q[i:i + part], torch.round(xd / want.double()[:, None]).to(torch.int8)), i


def test_more_rows_than_are_taken_are_refused(G):
    x = torch.zeros((1 << 28) + 1, 1, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(G.GnnError, match="rows"):
        G.quantize_rows(x)


def test_most_rows_in_group_order(G):
    n, g = 1 << 28, 5
    print(f"most rows grouped {n}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(-1, g + 1, (n,), device="cuda", generator=gen, dtype=torch.int32)
    off, order = G.group_rows(ids, g)
    start = 0
    for j in [*range(g), None]:
        mine = (ids == j) if j is not None else (ids < 0) | (ids >= g)
        rows = torch.nonzero(mine).flatten().to(torch.int32)  # ascending
        assert off[0 if j == 0 else (g if j is None else j)].item() == start
        assert torch.equal(order[start:start + rows.numel()], rows), j
        start += rows.numel()
    assert start == n


@pytest.mark.parametrize("kind", ["GNN_BF16", "GNN_INT8"])
def test_most_rows_through_a_layer(G, kind):
    n, k, width = 1 << 28, 9, 7
    print(f"most rows through a layer {n} {kind}", flush=True)
    rng = np.random.default_rng(1)
    w = rng.normal(size=(2, width, k)).astype(np.float32)
    b = rng.normal(size=(2, width)).astype(np.float32)
    layer = G.Linear(np.concatenate([w.reshape(2, -1), b], 1).ravel(),
                     G.make_linear_dims(k, width, 2, getattr(G, kind)))
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(n, k, dtype=torch.bfloat16, device="cuda")
    part = 1 << 25
    for i in range(0, n, part):
        x[i:i + part] = torch.randn(part, k, device="cuda", generator=gen)
    cut = n - 77
    off = torch.tensor([3, cut, n - 2], dtype=torch.int32, device="cuda")
    y = layer(x, offsets=off, out=torch.full((n, width), 5.0, dtype=torch.bfloat16, device="cuda"))
    assert (y[:3] == 5).all() and (y[n - 2:] == 5).all()
    # the same rows in small calls: 8-bit sums are exact, and so few 16-bit
    # products are summed in one step
    for g, lo, hi in ((0, 3, 5000), (0, (1 << 27) - 3000, (1 << 27) + 3000),
                      (0, cut - 5000, cut), (1, cut, n - 2)):
        few = torch.tensor([0, hi - lo, hi - lo] if g == 0 else [0, 0, hi - lo],
                           dtype=torch.int32, device="cuda")
        assert torch.equal(y[lo:hi], layer(x[lo:hi], offsets=few)), (g, lo)
        ref, bound = R.linear(x[lo:hi].float().cpu().numpy(),
                              w[g] if kind == "GNN_INT8" else
                              torch.as_tensor(w[g]).to(torch.bfloat16).float().numpy(),
                              b[g], "i8" if kind == "GNN_INT8" else "bf16")
        err = np.abs(y[lo:hi].double().cpu().numpy() - ref)
        assert (err <= R.stored(ref, bound, "bf16")).all()


def test_most_rows_through_a_network(G):
    n, widths = 1 << 28, [4, 8, 3]
    print(f"most rows through a network {n}", flush=True)
    rng = np.random.default_rng(1)
    dims = G.make_mlp_dims(widths, 2, G.GNN_INT8)
    mlp = G.Mlp(rng.normal(size=G.gnn_mlp_weight_count(dims)).astype(np.float32), dims)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(n, widths[0], device="cuda", generator=gen)
    ids = torch.randint(-1, 2, (n,), device="cuda", generator=gen, dtype=torch.int32)
    y = mlp(x, ids)
    for lo, hi in ((0, 5000), ((1 << 27) - 3000, (1 << 27) + 3000), (n - 5000, n)):
        assert torch.equal(y[lo:hi], mlp(x[lo:hi], ids[lo:hi])), lo
        assert (y[lo:hi][ids[lo:hi] < 0] == 0).all() and y[lo:hi].isfinite().all()


@pytest.mark.parametrize("kind,unit", [("f16", 2.0 ** -24), ("bf16", 2.0 ** -133)])
@pytest.mark.parametrize("m,k,n", [(5, 64, 40), (4100, 640, 1100), (40_000, 64, 40)])
def test_subnormal_rows_and_weights_count(G, kind, unit, m, k, n):
    """Whole multiples of the smallest number of a 16-bit type, on either side: the
    sums are exact."""
    t = {"f16": torch.float16, "bf16": torch.bfloat16}[kind]
    rng = np.random.default_rng(1)
    small = (rng.integers(-60, 61, (n, k)) * unit).astype(np.float32)
    big = rng.integers(-8, 9, (m, k)).astype(np.float32)
    dims = G.make_linear_dims(k, n, 1, G.GNN_F16 if kind == "f16" else G.GNN_BF16)
    b = np.zeros(n, np.float32)
    layer = G.Linear(np.concatenate([small.ravel(), b]), dims)
    y = layer(torch.as_tensor(big).to(t).cuda(), out_dtype=torch.float32)
    assert np.array_equal(y.double().cpu().numpy(), big.astype(np.float64) @ small.astype(np.float64).T)
    few = rng.integers(-8, 9, (n, k)).astype(np.float32)
    layer = G.Linear(np.concatenate([few.ravel(), b]), dims)
    x = (rng.integers(-60, 61, (m, k)) * unit).astype(np.float32)
    y = layer(torch.as_tensor(x).to(t).cuda(), out_dtype=torch.float32)
    assert np.array_equal(y.double().cpu().numpy(), x.astype(np.float64) @ few.astype(np.float64).T)
    y = layer(torch.as_tensor(x).cuda(), out_dtype=torch.float32)  # rounded on the way
    assert np.array_equal(y.double().cpu().numpy(), x.astype(np.float64) @ few.astype(np.float64).T)
