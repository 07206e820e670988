"""Performance cases of the operators that networks are trained with: layer norm
and its gradients, the gated feed-forward block and its gradients, and the
gradients' global norm with clipping.

Rows are hits or edges.  ``run`` computes each operator either plainly in torch
(``own`` false) or through the public calls of ``paper_2402_09633_amd.gnn``.
"""
from __future__ import annotations

import math

import torch

own = False  # True: run() makes the library's calls

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
MAX_NORM = 1.0


# ------------------------------------------------------------------ cases ---

def _norm(name, rows, width, kind, train):
    return {"name": name, "op": "norm", "rows": rows, "width": width, "type": kind, "train": train}


def _gated(name, rows, k, hidden, n, kind, train, act="silu", bias=False):
    return {"name": name, "op": "gated", "rows": rows, "in": k, "hidden": hidden, "out": n,
            "type": kind, "train": train, "act": act, "bias": bias}


def _clip(name, blocks, width, hidden, kind):
    return {"name": name, "op": "clip", "blocks": blocks, "width": width, "hidden": hidden,
            "type": kind}


def listed():
    return [
        # A single row of a wide network on its way to an answer: latency.
        _norm("norm_one_row", 1, 512, "f32", False),
        # A training step's norm over all edges of a full event at H = 128.
        _norm("norm_edges_train", 1_000_513, 128, "f32", True),
        # A region of interest with raw features appended to its rows: an odd
        # width and row starts that are not aligned.
        _norm("norm_odd_train", 20_011, 391, "f16", True),
        # Very wide rows, a batch of a training step.
        _norm("norm_wide_train", 8_192, 8_192, "bf16", True),
        # A single row through a wide block: the weights have to be read.
        _gated("gated_one_row", 1, 2048, 8192, 2048, "bf16", False),
        # The requests of one moment of a service, a row each.
        _gated("gated_batch", 48, 2048, 8192, 2048, "f16", False),
        # All hits of a full event through a block of an embedding.
        _gated("gated_hits", 300_000, 128, 512, 128, "bf16", False, "gelu", True),
        # A training step over all edges of a full event.
        _gated("gated_edges_train", 1_000_513, 128, 256, 128, "bf16", True, "silu", True),
        # A training step of a region of interest, every width odd.
        _gated("gated_odd_train", 4_097, 391, 1031, 259, "f16", True, "gelu", True),
        # A training step of a wide block, bound by the matrix cores.
        _gated("gated_large_train", 8_192, 2048, 8192, 2048, "bf16", True),
        # The gradients of a small network: few values in many tensors.
        _clip("clip_small", 4, 64, 128, "f32"),
        # The gradients of a large network, 16 and 32 bits side by side.
        _clip("clip_large", 24, 1024, 4096, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm"] * 3 + ["gated"] * 5 + ["clip"] * 2)
    train = rng.random() < 0.6
    if op == "norm":
        width = _log_int(rng, 8, 16_384)
        case = _norm("", _log_int(rng, 1, min(1_000_000, 60_000_000 // width)), width,
                     rng.choice(["f32", "bf16", "f16"]), train)
    elif op == "clip":
        width, hidden = _log_int(rng, 16, 1024), _log_int(rng, 16, 4096)
        case = _clip("", _log_int(rng, 1, 24), width, hidden, rng.choice(["f32", "bf16", "f16"]))
    else:
        k, hidden, n = (_log_int(rng, 8, 8192) for _ in range(3))
        if rng.random() < 0.5:  # half the blocks have widths that are multiples of 32
            k, hidden, n = (-(-v // 32) * 32 for v in (k, hidden, n))
        most = min(1_000_000, 8_192 * 2048 * 8192 // (hidden * max(k, n)),
                   128_000_000 // (hidden + k + n))
        case = _gated("", _log_int(rng, 1, max(1, most)), k, hidden, n, rng.choice(["bf16", "f16"]),
                      train, rng.choice(["silu", "silu", "gelu", "sigmoid"]),
                      rng.random() < 0.5)
    del case["name"]
    return case


# ----------------------------------------------------------------- inputs ---

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(gen, *shape):
    return torch.randn(*shape, device=DEV, generator=gen)


def _rows(gen, rows, width, dtype, shift=0.0):
    """Rows of a row-dependent size; odd widths lie in a wider table."""
    t = _randn(gen, rows, width) * torch.rand(rows, 1, device=DEV, generator=gen).add_(0.25)
    t += shift
    if width % 2 == 0:
        return t.to(dtype)
    table = torch.zeros(rows, width + 5, dtype=dtype, device=DEV)
    table[:, :width] = t
    return table[:, :width]


def _tensors(case):
    """(shape, type) of the parameters of `blocks` gated blocks with a layer norm each."""
    w, h, kind = case["width"], case["hidden"], TYPES[case["type"]]
    block = [((h, w), kind), ((h, w), kind), ((w, h), kind), ((h,), kind), ((h,), kind),
             ((w,), kind), ((w,), torch.float32), ((w,), torch.float32)]
    return block * case["blocks"]


def prepare(case, seed):
    gen = _gen(seed)
    st = {"op": case["op"]}
    if case["op"] == "norm":
        m, n, kind = case["rows"], case["width"], TYPES[case["type"]]
        st["train"] = case["train"]
        st["x"] = _rows(gen, m, n, kind, 0.3)
        st["gamma"] = 1.0 + 0.2 * _randn(gen, n)
        st["beta"] = 0.1 * _randn(gen, n)
        if st["train"]:
            st["dy"] = _rows(gen, m, n, kind)
    elif case["op"] == "gated":
        m, kind = case["rows"], TYPES[case["type"]]
        k, h, n = case["in"], case["hidden"], case["out"]
        st.update(train=case["train"], act=case["act"], bias=case["bias"])
        st["x"] = _rows(gen, m, k, kind)
        st["wg"] = (_randn(gen, h, k) / math.sqrt(k)).to(kind)
        st["wu"] = (_randn(gen, h, k) / math.sqrt(k)).to(kind)
        st["wd"] = (_randn(gen, n, h) / math.sqrt(h)).to(kind)
        st["bg"], st["bu"], st["bd"] = ((0.1 * _randn(gen, v)).to(kind) if case["bias"] else None
                                        for v in (h, h, n))
        if st["train"]:
            st["dy"] = _rows(gen, m, n, kind)
    else:
        sizes = [math.prod(shape) for shape, _ in _tensors(case)]
        st["grads"] = []
        for (shape, kind), n in zip(_tensors(case), sizes):
            size = 10.0 ** (-1.0 - 2.0 * torch.rand(1, device=DEV, generator=gen))
            st["grads"].append((_randn(gen, *shape) * size).to(kind))
        # Clipped, they lie side by side, as an optimiser or an all-reduce takes them.
        st["flat"] = {str(k): torch.zeros(sum(n for (_, kk), n in zip(_tensors(case), sizes)
                                              if kk == k), dtype=k, device=DEV)
                      for k in {kk for _, kk in _tensors(case)}}
        at = dict.fromkeys(st["flat"], 0)
        st["clipped"] = []
        for g in st["grads"]:
            k = str(g.dtype)
            st["clipped"].append(st["flat"][k][at[k]:at[k] + g.numel()].view(g.shape))
            at[k] += g.numel()
    return st


# ------------------------------------------------------------------ a pass ---

def _plain_norm(st):
    x = st["x"].float()
    mean = x.mean(1, keepdim=True)
    centred = x - mean
    rstd = torch.rsqrt((centred * centred).mean(1, keepdim=True) + EPS)
    xhat = centred * rstd
    kind = st["x"].dtype
    y = (xhat * st["gamma"] + st["beta"]).to(kind)
    if not st["train"]:
        return y
    dy = st["dy"].float()
    g = dy * st["gamma"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return y, dx.to(kind), (dy * xhat).sum(0), dy.sum(0)


def _act(name, g):
    """The activation and its derivative."""
    if name == "gelu":
        phi = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * phi, phi + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    s = 1.0 / (1.0 + torch.exp(-g))
    if name == "sigmoid":
        return s, s * (1.0 - s)
    return g * s, s * (1.0 + g * (1.0 - s))


def _plain_gated(st):
    kind = st["x"].dtype
    x, wg, wu, wd = (st[k].float() for k in ("x", "wg", "wu", "wd"))
    g, u = x @ wg.t(), x @ wu.t()
    if st["bias"]:
        g, u = g + st["bg"].float(), u + st["bu"].float()
    a, slope = _act(st["act"], g)
    h = a * u
    y = h @ wd.t()
    if st["bias"]:
        y = y + st["bd"].float()
    if not st["train"]:
        return y.to(kind)
    dy = st["dy"].float()
    dh = dy @ wd
    dg, du = dh * u * slope, dh * a
    grads = [dg @ wg + du @ wu, dg.t() @ x, du.t() @ x, dy.t() @ h]
    if st["bias"]:
        grads += [dg.sum(0), du.sum(0), dy.sum(0)]
    return (y.to(kind), *(v.to(kind) for v in grads))


def _plain_clip(st):
    squares = [g.float().square().sum(dtype=torch.float64) for g in st["grads"]]
    norm = torch.stack(squares).sum().sqrt().float()
    scale = torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)
    for g, out in zip(st["grads"], st["clipped"]):
        out.copy_(g.float() * scale)
    return norm, st["flat"]


def _own_pass(st):
    from paper_2402_09633_amd import gnn as G
    if st["op"] == "clip":
        return G.clip_grads(st["grads"], MAX_NORM, out=st["clipped"]), st["flat"]
    if st["op"] == "norm":
        if not st["train"]:
            return G.layer_norm(st["x"], st["gamma"], st["beta"], EPS)
        y, mean, rstd = G.layer_norm(st["x"], st["gamma"], st["beta"], EPS, save=True)
        return y, *G.layer_norm_backward(st["dy"], st["x"], st["gamma"], mean, rstd)
    w = (st["wg"], st["wu"], st["wd"])
    b = (st["bg"], st["bu"], st["bd"]) if st["bias"] else None
    y = G.gated(st["x"], *w, biases=b, activation=st["act"])
    if not st["train"]:
        return y
    grads = G.gated_backward(st["dy"], st["x"], *w, biases=b, activation=st["act"])
    return y, *(grads if st["bias"] else grads[:4])


def run(state):
    if own:
        return _own_pass(state)
    return {"norm": _plain_norm, "gated": _plain_gated, "clip": _plain_clip}[state["op"]](state)


# -------------------------------------------------------- work and answers ---

def work(case):
    if case["op"] == "clip":
        n = [(math.prod(shape), 4 if kind == torch.float32 else 2) for shape, kind in _tensors(case)]
        return {"bytes": 2 * sum(c * s for c, s in n) + 4, "flops": 3 * sum(c for c, _ in n)}
    s = SIZE[case["type"]]
    if case["op"] == "norm":
        m, n = case["rows"], case["width"]
        if case["train"]:  # x and dy, y and dx, gamma and beta and their gradients
            return {"bytes": 4 * m * n * s + 16 * n, "flops": 20 * m * n}
        return {"bytes": 2 * m * n * s + 8 * n, "flops": 8 * m * n}
    m, k, h, n = case["rows"], case["in"], case["hidden"], case["out"]
    weights = 2 * h * k + h * n + (2 * h + n if case["bias"] else 0)
    if not case["train"]:
        return {"bytes": s * (m * (k + n) + weights), "flops": 2 * m * h * (2 * k + n)}
    # every product of the forward pass has two in the backward pass
    return {"bytes": s * (2 * m * (k + n) + 2 * weights), "flops": 6 * m * h * (2 * k + n)}


def _with_grad(*tensors):
    return [t.double().requires_grad_() for t in tensors]


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "clip":
        total = torch.cat([g.double().flatten().square().sum()[None] for g in st["grads"]]).sum()
        norm = total ** 0.5
        factor = min(1.0, MAX_NORM / (float(norm) + 1e-6))
        flat = {k: torch.cat([g.double().flatten() for g in st["grads"] if str(g.dtype) == k])
                .mul_(factor) for k in st["flat"]}
        return norm, flat
    # gradients by automatic differentiation of the definition
    if case["op"] == "norm":
        leaves = _with_grad(st["x"], st["gamma"], st["beta"])
        x, gamma, beta = leaves
        var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
        y = gamma * ((x - mean) / (var + EPS).sqrt()) + beta
    else:
        names = ["x", "wg", "wu", "wd"] + (["bg", "bu", "bd"] if case["bias"] else [])
        leaves = _with_grad(*(st[k] for k in names))
        x, wg, wu, wd = leaves[:4]
        bg, bu, bd = leaves[4:] if case["bias"] else (0.0, 0.0, 0.0)
        gate, up = torch.matmul(x, wg.t()) + bg, torch.matmul(x, wu.t()) + bu
        if case["act"] == "silu":
            gate = gate * torch.sigmoid(gate)
        elif case["act"] == "sigmoid":
            gate = torch.sigmoid(gate)
        else:
            gate = gate * torch.special.ndtr(gate)
        y = torch.matmul(gate * up, wd.t()) + bd
    if not case["train"]:
        return y.detach()
    return y.detach(), *torch.autograd.grad(y, leaves, st["dy"].double())
