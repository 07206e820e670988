"""The large calls of the linear layers on the GPU: row panels of 64 and 128 rows
with four and with eight waves, long output rows that do not start on whole
sectors, and the tiles for wide layers, each in every type that it takes.
test_rows_plan.py checks that the calls reach the kernels they are meant for."""
import numpy as np
import pytest
import torch

from tests import rows_ref as R

pytestmark = pytest.mark.gpu
T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ROWS = {"i8": ("f32", "bf16", "f16", "i8"), "bf16": ("bf16", "f32"), "f16": ("f16", "f32")}

# rows, row width, outputs, output type, gap behind an output row, groups, and for
# 8-bit and 16-bit weights (row blocks, waves), or (tile,)
CASES = [
    # one step of four: no weights are fetched again; 3 channel blocks for 8 waves
    # in the last round
    (70_001, 40, 300, "f32", 0, 1, (4, 8), (4, 8)),
    (40_000, 72, 300, "bf16", 0, 1, (2, 8), (2, 8)),
    # many rounds over the channels, the last one partial
    (66_001, 100, 1100, "bf16", 20, 1, (4, 8), (4, 8)),
    (33_000, 130, 1100, "f16", 4, 1, (2, 8), (2, 8)),
    # as wide as 128 and 64 rows to a panel get
    (66_000, 512, 256, "bf16", 0, 1, (4, 8), (2, 8)),
    (65_700, 1000, 160, "bf16", 0, 1, (2, 8), None),
    # four waves, and rows too wide for 128 to a panel beside three others
    (70_001, 100, 128, "f16", 0, 1, (4, 4), (4, 4)),
    (70_001, 333, 97, "bf16", 0, 1, (2, 4), (2, 4)),
    # groups, in an order and without one
    (70_001, 77, 200, "f32", 3, 5, (4, 8), (4, 8)),
    (50_000, 200, 333, "bf16", 3, 9, (2, 8), (2, 8)),
    # long output rows that do not start on 64 bytes: 64 rows to a panel
    (70_001, 64, 1537, "bf16", 0, 1, (2, 8), (2, 8)),
    (66_000, 40, 769, "f32", 0, 1, (2, 8), (2, 8)),
    (66_000, 40, 1000, "f16", 2, 3, (2, 8), (2, 8)),
    # 256 rows to a tile
    (14_001, 1101, 1300, "bf16", 1, 1, (4,), (4,)),
    (17_000, 1101, 1100, "f32", 0, 3, (4,), (4,)),
    (16_500, 1040, 1056, "f16", 0, 1, (4,), (4,)),
]


@pytest.fixture(scope="module")
def G():
    from paper_2402_09633_amd import gnn
    return gnn


def _sample(off, m, rng):
    """Positions to check: the ends, around the groups' borders, and some others."""
    at = [np.arange(0, 300), np.arange(m - 300, m), rng.integers(0, m, 400)]
    at += [np.arange(o - 70, o + 70) for o in off]
    at = np.unique(np.concatenate(at))
    return at[(at >= 0) & (at < m)]


@pytest.mark.parametrize("kind", ["i8", "bf16", "f16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}x{c[1]}-{c[2]}{c[3]}+{c[4]}g{c[5]}")
def test_large_calls(G, kind, case):
    m, k, n, out, gap, g, want8, want16 = case
    rng = np.random.default_rng(m + k + n)
    w = (rng.normal(size=(g, n, k)) / np.sqrt(k)).astype(np.float32)
    b = rng.normal(size=(g, n)).astype(np.float32)
    dtype = {"i8": G.GNN_INT8, "bf16": G.GNN_BF16, "f16": G.GNN_F16}[kind]
    layer = G.Linear(np.concatenate([w.reshape(g, -1), b], 1).ravel(),
                     G.make_linear_dims(k, n, g, dtype))
    held = w if kind == "i8" else torch.as_tensor(w).to(T[kind]).float().numpy()
    off = order = offsets = None
    ends = [0, m]
    if g > 1:  # uneven groups, one of them empty, and rows of no group at both ends
        ends = np.sort(rng.integers(20, m - 30, g + 1))
        ends[0], ends[1], ends[-1] = 20, ends[2], m - 30
        offsets = torch.as_tensor(ends.astype(np.int32)).cuda()
        if gap == 3:
            order = torch.randperm(m, device="cuda", generator=torch.Generator("cuda").manual_seed(m)
                                   ).to(torch.int32)
    for xt in ROWS[kind]:
        print(f"large {kind} {m}x{k}->{n} x {xt} y {out} {g} groups", flush=True)
        gen = torch.Generator(device="cuda").manual_seed(m + k)
        pitch = k + (3 if k % 2 else 0)
        table = torch.full((m * pitch + 1,), float("nan"), dtype=T.get(xt, torch.float32),
                           device="cuda")
        x = table[1:].view(m, pitch)[:, :k]
        x.copy_(torch.randn(m, k, device="cuda", generator=gen) *
                torch.rand(m, 1, device="cuda", generator=gen).add_(0.1))
        rows, scales = x, None
        if xt == "i8":
            rows, scales = G.quantize_rows(x)
        y = torch.full((m, n + gap), 7.0, dtype=T[out], device="cuda")
        layer(rows, scales=scales, offsets=offsets, order=order, out=y[:, :n])
        assert (y[:, n:] == 7).all()
        y = y[:, :n]
        at = _sample(ends, m, rng)
        idx = torch.as_tensor(at).cuda() if order is None else order[torch.as_tensor(at).cuda()].long()
        ys, xs = y[idx].double().cpu().numpy(), x[idx].float()
        xs = (xs if kind == "i8" else xs.to(T[kind]).float()).cpu().numpy()
        for j in range(g):
            mine = (at >= ends[j]) & (at < ends[j + 1])
            if mine.any():
                ref, bound = R.linear(xs[mine], held[j], b[j], kind)
                worst = (np.abs(ys[mine] - ref) / R.stored(ref, bound, out)).max()
                assert worst <= 1.0, f"{xt} group {j}: {worst:.3f} of the bound"
        rest = (at < ends[0]) | (at >= ends[-1])
        assert (ys[rest] == 7.0).all() and rest.sum() == (50 if g > 1 else 0)
        if kind == "i8" and g == 1:
            # exact sums: every row is the same in calls of few rows, which other
            # kernels take
            step = 3000
            for lo in range(0, m, step):
                few = layer(rows[lo:lo + step], scales=None if scales is None else
                            scales[lo:lo + step], out_dtype=T[out])
                assert torch.equal(y[lo:lo + step], few), (xt, lo)
