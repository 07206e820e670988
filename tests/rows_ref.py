"""Plain 64-bit forms of the row operators, with the error bounds of the
kernels' arithmetic (shared by their tests)."""
import numpy as np

FLOATS = ("f32", "bf16", "f16")
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # relative, largest
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}    # smallest number


def quantize(x):
    """(q, scale) of rows of fp32 values, from the definition."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore"):
        s = (np.abs(x).max(axis=1) / 127.0).astype(np.float32)
    bad = ~np.isfinite(x).all(axis=1)
    s[bad] = np.nan
    s[s < np.float32(2.0 ** -126)] = 0.0
    inv = np.where(bad | (s == 0), 1.0, s.astype(np.float64))
    q = np.rint(np.where((bad | (s == 0))[:, None], 0.0, x) / inv[:, None])
    return q.astype(np.int8), s


def group(ids, G):
    """(offsets, order): stable by group, rows of no group last."""
    ids = np.asarray(ids, np.int64)
    key = np.where((ids >= 0) & (ids < G), ids, G)
    counts = np.bincount(key, minlength=G + 1)[:G]
    return (np.concatenate([[0], np.cumsum(counts)]).astype(np.int32),
            np.argsort(key, kind="stable").astype(np.int32))


def linear(x, w, b, kind):
    """(y, bound): rows x [m][K] (fp32 values; rounded already where the weights
    have 16 bits) through w [N][K] (as the layer holds it in 16 bits; fp32 for
    kind "i8"), and how far the kernel's fp32 value may be.

    i8: the sum is exact; its conversion, the scales' product, the product with
    it and the bias add one rounding each.  16 bits: products are exact in fp32
    and every one of the K sums and the bias' rounds a partial sum that is no
    larger than the sum of the absolute values, by a last place at most."""
    b = np.asarray(b, np.float64)
    if kind == "i8":
        q, s = quantize(x)
        wq, ws = quantize(w)
        part = (q.astype(np.float64) @ wq.astype(np.float64).T) * s.astype(np.float64)[:, None] * \
            ws.astype(np.float64)[None, :]
        return part + b, 4 * 2.0 ** -24 * (np.abs(part) + np.abs(b))
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    size = np.abs(x) @ np.abs(w).T + np.abs(b)
    return x @ w.T + b, (x.shape[1] + 2) * 2.0 ** -23 * size


def stored(y, bound, out):
    """The bound after the one rounding to the output type."""
    return bound + HALF_STEP[out] * (np.abs(y) + bound) + TINY[out]
