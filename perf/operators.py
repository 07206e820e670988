"""Performance cases of the row operators: products with 8-bit weights and
rows, products grouped by detector region, and the two steps that feed them
(rows to 8 bits, rows put in group order).

Rows are hits or edges.  ``run`` computes each operator either plainly in torch
(``own`` false) or through the public calls of ``paper_2402_09633_amd.gnn``.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # True: run() makes the library's calls

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "i8": 1}


# ------------------------------------------------------------------ cases ---

def _linear(name, rows, k, n, weights="i8", x="bf16", y="bf16", groups=1, ordered=False):
    return {"name": name, "op": "linear", "rows": rows, "in": k, "out": n, "weights": weights,
            "x": x, "y": y, "groups": groups, "ordered": ordered}


def listed():
    return [
        # A single row through one layer of a wide network: latency.
        _linear("i8_one_row", 1, 512, 512, x="f32", y="f32"),
        # A hidden layer of a wide embedding over all hits of a full event.
        _linear("i8_hits", 300_000, 512, 512),
        # The first layer of an edge MLP, [h_src; h_dst; e] at H = 128, over the
        # edges of a full event with the fp32 model's rows.
        _linear("i8_edges", 1_000_513, 384, 128, x="f32"),
        # A region of interest with raw features appended to its rows: odd
        # widths and row starts that are not aligned.
        _linear("i8_odd", 20_011, 391, 259, x="f16", y="f32"),
        # A large square layer, bound by the matrix cores.
        _linear("i8_large", 16_384, 4096, 4096),
        # Hits in input order, one weight set for each of four regions (barrel
        # and endcap, pixel and strip), sizes as uneven as a detector's.
        _linear("regions_hits", 300_000, 128, 128, "bf16", groups=4, ordered=True),
        # Edges in input order, one weight set for each pair of regions; some
        # pairs have no edge.
        _linear("regions_edges", 1_000_513, 384, 128, "f16", "f16", "f16", groups=16, ordered=True),
        # A handful of rows spread over many wide weight sets: the weights of the
        # groups in use have to be read.
        _linear("regions_few", 64, 1024, 1024, "bf16", groups=64),
        # Rows of all edges to 8 bits.
        {"name": "quantize_edges", "op": "quantize", "rows": 1_000_513, "in": 128, "x": "f32"},
        # Rows of an odd width out of a wider table.
        {"name": "quantize_odd", "op": "quantize", "rows": 4097, "in": 1031, "x": "bf16"},
        # Edges of a full event put in the order of their region pairs.
        {"name": "group_edges", "op": "group", "rows": 1_000_513, "groups": 16},
        # The hits of a small event put in the order of their regions.
        {"name": "group_small", "op": "group", "rows": 2_000, "groups": 4},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear"] * 6 + ["quantize", "group"])
    if op == "group":
        return {"op": op, "rows": _log_int(rng, 1, 1_000_000), "groups": _log_int(rng, 2, 256)}
    if op == "quantize":
        k = _log_int(rng, 8, 4096)
        return {"op": op, "rows": _log_int(rng, 1, min(1_000_000, 128_000_000 // k)), "in": k,
                "x": rng.choice(["f32", "bf16", "f16"])}
    groups = rng.choice([1, 1, _log_int(rng, 2, 64)])
    wide = 4096 if groups == 1 else 1024
    k, n = _log_int(rng, 8, wide), _log_int(rng, 8, wide)
    if rng.random() < 0.5:  # half the layers have widths that are multiples of 32
        k, n = -(-k // 32) * 32, -(-n // 32) * 32
    weights = rng.choice(["i8", "i8", "bf16", "f16"] if groups == 1 else ["i8", "bf16", "f16"])
    most = min(1_000_000, 16_384 * 4096 * 4096 // (k * n), 400_000_000 // (k + n))
    x = rng.choice(["f32", "bf16", "f16"]) if weights == "i8" else weights
    return _draw_linear(_log_int(rng, 1, most), k, n, weights, x,
                        rng.choice(["f32", "bf16", "f16"]), groups, rng)


def _draw_linear(rows, k, n, weights, x, y, groups, rng):
    c = _linear("", rows, k, n, weights, x, y, groups, groups > 1 and rng.random() < 0.5)
    del c["name"]
    return c


# ----------------------------------------------------------------- inputs ---

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _rows(rows, k, dtype, gen, pitch=None):
    """Rows as they leave a LayerNorm and ReLU, of a row-dependent size."""
    t = torch.randn(rows, k, device=DEV, generator=gen).add_(0.3).clamp_(min=0.0)
    t *= torch.rand(rows, 1, device=DEV, generator=gen).add_(0.25)
    if pitch is None or pitch == k:
        return t.to(dtype)
    table = torch.zeros(rows, pitch, dtype=dtype, device=DEV)
    table[:, :k] = t
    return table[:, :k]


def _sizes(rows, groups, seed):
    """Uneven group sizes that add up to `rows`; about one group in eight is empty."""
    rng = np.random.default_rng(seed)
    share = rng.exponential(1.0, groups) * (rng.random(groups) > 0.125)
    if not share.any():
        share[0] = 1.0
    return np.bincount(rng.choice(groups, rows, p=share / share.sum()),
                       minlength=groups).astype(np.int64)


def _ids(sizes, gen):
    ids = torch.repeat_interleave(torch.arange(len(sizes), device=DEV, dtype=torch.int32),
                                  torch.as_tensor(sizes, device=DEV))
    return ids[torch.randperm(ids.numel(), device=DEV, generator=gen)]


def prepare(case, seed):
    gen = _gen(seed)
    st = {"op": case["op"]}
    if case["op"] == "group":
        st["groups"] = case["groups"]
        st["ids"] = _ids(_sizes(case["rows"], case["groups"], seed), gen)
        if own:
            _own_group(st)
        return st
    if case["op"] == "quantize":
        k = case["in"]
        st["x"] = _rows(case["rows"], k, TYPES[case["x"]], gen, k + (5 if k % 2 else 0))
        if own:
            _own_quantize(st)
        return st
    m, k, n, g = case["rows"], case["in"], case["out"], case["groups"]
    st["x"] = _rows(m, k, TYPES[case["x"]], gen)
    st["y"], st["weights"] = TYPES[case["y"]], case["weights"]
    w = torch.randn(g, n, k, device=DEV, generator=gen) * (1.0 / math.sqrt(k))
    st["b"] = torch.randn(g, n, device=DEV, generator=gen) * 0.1
    st["sizes"] = _sizes(m, g, seed).tolist() if g > 1 else [m]
    st["offsets"] = st["order"] = None
    if g > 1:
        ends = np.concatenate([[0], np.cumsum(st["sizes"])]).astype(np.int32)
        st["offsets"] = torch.as_tensor(ends, device=DEV)
        if case["ordered"]:  # rows in input order, as their group ids come
            st["order"] = torch.argsort(_ids(st["sizes"], gen), stable=True).to(torch.int32)
    # The weights as the layer holds them: 16-bit numbers, or whole numbers of
    # 8 bits with one scale for each output channel.
    if case["weights"] == "i8":
        st["ws"] = _scale(w)
        st["w"] = torch.round(w.double() / st["ws"].double()[:, :, None]).float()
    else:
        st["w"] = w.to(TYPES[case["weights"]]).float()
    if own:
        _own_linear(st, case, w)
    return st


def _own_group(st):
    from paper_2402_09633_amd import gnn as G
    st["call"] = G


def _own_quantize(st):
    from paper_2402_09633_amd import gnn as G
    st["call"] = G


def _own_linear(st, case, w):
    from paper_2402_09633_amd import gnn as G
    dtype = {"i8": G.GNN_INT8, "bf16": G.GNN_BF16, "f16": G.GNN_F16}[case["weights"]]
    blob = torch.cat([w.flatten(1), st["b"]], 1).flatten().cpu().numpy()
    st["layer"] = G.Linear(blob, G.make_linear_dims(case["in"], case["out"], case["groups"], dtype))
    st["out"] = torch.zeros(case["rows"], case["out"], dtype=st["y"], device=DEV)


# ------------------------------------------------------------------ a pass ---

def _scale(x):
    """The fp32 number nearest to a 127th of each row's largest absolute value.
    In 64 bits: 16-bit rows often hold values half way between two steps, and
    the last bit of the scale then says which way they go."""
    return (x.abs().amax(-1).double() / 127.0).float()


def _quantize(x):
    """Whole numbers in -127..127 and the scale of each row."""
    x = x.float()
    s = _scale(x)[:, None]
    q = torch.round(x.double() / s.clamp(min=2.0 ** -126).double())  # a quotient next to a half
    return q.float(), s


def _product(x, w, ws, b):
    """Rows of one group through one weight set, in fp32."""
    if ws is None:
        return x.float() @ w.t() + b
    q, s = _quantize(x)
    return (q @ w.t()) * s * ws + b


def run(state):
    op = state["op"]
    if op == "group":
        ids, groups = state["ids"], state["groups"]
        if own:
            return state["call"].group_rows(ids, groups)
        ends = torch.cumsum(torch.bincount(ids, minlength=groups), 0)
        offsets = torch.nn.functional.pad(ends, (1, 0))
        return offsets.to(torch.int32), torch.argsort(ids, stable=True).to(torch.int32)
    if op == "quantize":
        if own:
            return state["call"].quantize_rows(state["x"])
        q, s = _quantize(state["x"])
        return q.to(torch.int8), s.flatten()
    x, order = state["x"], state["order"]
    if own:
        return state["layer"](x, offsets=state["offsets"], order=order, out=state["out"])
    if state["offsets"] is None:
        ws = state["ws"][0] if "ws" in state else None
        return _product(x, state["w"][0], ws, state["b"][0]).to(state["y"])
    parts = torch.split(x if order is None else x[order.long()], state["sizes"])
    scales = state["ws"] if "ws" in state else [None] * len(parts)
    y = torch.cat([_product(p, w, ws, b) for p, w, ws, b
                   in zip(parts, state["w"], scales, state["b"])]).to(state["y"])
    if order is None:
        return y
    back = torch.empty_like(y)
    back[order.long()] = y
    return back


# -------------------------------------------------------- work and answers ---

def work(case):
    m = case["rows"]
    if case["op"] == "group":
        return {"bytes": 8 * m + 4 * (case["groups"] + 1), "flops": 0}
    if case["op"] == "quantize":
        return {"bytes": m * case["in"] * (SIZE[case["x"]] + 1) + 4 * m, "flops": 2 * m * case["in"]}
    k, n, g = case["in"], case["out"], case["groups"]
    # weight sets that have to be read: with sizes as _sizes draws them, the
    # groups that are expected to have a row
    used = 1 if g == 1 else max(1, round(0.875 * g * m / (m + 0.875 * g)))
    nbytes = m * k * SIZE[case["x"]] + m * n * SIZE[case["y"]]
    nbytes += used * n * (k * SIZE[case["weights"]] + 4)
    if case["weights"] == "i8":
        nbytes += 4 * used * n
    if g > 1:
        nbytes += 4 * (g + 1) + (4 * m if case["ordered"] else 0)
    return {"bytes": nbytes, "flops": 2 * m * n * k}


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "group":
        return None
    x = st["x"].to(torch.float64)
    if case["op"] == "quantize":
        top = torch.maximum(x.max(dim=1).values, -x.min(dim=1).values)
        scale = (top / 127).to(torch.float32)  # a row's scale is an fp32 number
        steps = x / scale.double().clamp(min=2.0 ** -126).unsqueeze(1)
        return torch.round(steps).to(torch.int8), scale.double()
    group_of = torch.zeros(case["rows"], dtype=torch.long, device=DEV)
    if case["groups"] > 1:
        place = torch.arange(case["rows"], device=DEV)
        at = place if st["order"] is None else st["order"].long()
        group_of[at] = torch.searchsorted(st["offsets"].long(), place, right=True) - 1
    if case["weights"] == "i8":
        top = torch.maximum(x.max(dim=1).values, -x.min(dim=1).values)
        scale = (top / 127).to(torch.float32).double().unsqueeze(1)
        x = torch.round(x / scale.clamp(min=2.0 ** -126)) * scale
    y = torch.empty(case["rows"], case["out"], dtype=torch.float64, device=DEV)
    for g in range(case["groups"]):
        weight = st["w"][g].double()
        if case["weights"] == "i8":
            weight = weight * st["ws"][g].double().unsqueeze(1)
        mine = torch.nonzero(group_of == g).flatten()
        y[mine] = torch.addmm(st["b"][g].double(), x[mine], weight.t())
    return y
