"""Plain 64-bit definitions of the single integer layers: the projection with low-rank adapters and the norms
before and after a block with its gate and residual scale. NumPy and Python integers only."""
import math

import numpy as np

LIM24 = 1 << 23


def rq(a, m, s):
    """floor((a m + 2^(30+s)) / 2^(31+s))"""
    s = np.asarray(s, dtype=np.int64)
    return (np.asarray(a, dtype=np.int64) * np.asarray(m, dtype=np.int64) + (np.int64(1) << (30 + s))) >> (31 + s)


def product(a, b):
    """a @ b.T of small integers, exact: float64 holds sums below 2^53."""
    return (a.astype(np.float64) @ b.astype(np.float64).T).astype(np.int64)


def slots_of_rows(rows, seg_start, seg_adapter):
    """Adapter of each row, -1 for none, -2 for rows in no request."""
    slot = np.full(rows, -2, dtype=np.int64)
    for q, a in enumerate(seg_adapter):
        slot[seg_start[q]:seg_start[q + 1]] = a
    return slot


def projection(layer, x, adapters=(), seg_start=None, seg_adapter=None, y=None):
    """y [rows, c_out] int64; rows in no request keep y's values."""
    w = np.asarray(layer["w"]).reshape(layer["c_out"], layer["c_in"])
    acc = product(x, w) + layer["bias"].astype(np.int64)
    slot = np.full(x.shape[0], -1) if seg_start is None or len(seg_adapter) == 0 else slots_of_rows(x.shape[0], seg_start, seg_adapter)
    for a in np.unique(slot):
        if a < 0 or adapters[a] is None:
            continue
        ad, at = adapters[a], np.nonzero(slot == a)[0]
        h = np.clip(rq(product(x[at], ad["down"]), ad["m0"], ad["s"]), -128, 127)
        acc[at] += product(h, ad["up"])
    v = rq(acc, layer["m0"], layer["s"])
    if layer["relu"]:
        v = np.maximum(v, 0)
    if layer["clamp"] is not None:
        v = np.clip(v, *layer["clamp"])
    if y is not None:
        v = np.where((slot == -2)[:, None], y, v)
    return v


def normed_row(v, kind, eps):
    """One row, in Python integers."""
    v = [min(max(int(e), -LIM24), LIM24 - 1) for e in v]
    C = len(v)
    if kind == "centred":
        mean = (2 * sum(v) + C) // (2 * C)
        v = [e - mean for e in v]
    D, t = sum(e * e for e in v) + eps, 0
    while D << t < 1 << 60:
        t += 2
    rho = ((1 << 61) - 1) // math.isqrt(D << t)
    sh = 39 - t // 2
    return [(e * rho + (1 << (sh - 1))) >> sh for e in v]


def normed(v, kind, eps):
    return np.array([normed_row(row, kind, eps) for row in v], dtype=np.int64).reshape(v.shape)


def clip24(v):
    return np.clip(np.asarray(v, dtype=np.int64), -LIM24, LIM24 - 1)


def norm_step(desc, r, b=None, gate=None):
    """(r', n) of rows [rows, c], int64; None where the description has no such part."""
    out = n = None
    r = np.asarray(r, dtype=np.int64)
    if b is not None:
        post = desc["post"]
        a = normed(b, post["norm"], desc["eps"]) if post["norm"] else clip24(b)
        if gate is not None:
            a = a * gate.astype(np.int64)
        r = out = np.clip(clip24(r) + rq(a, post["mult"], post["shift"]), *desc["res_range"])
    if desc.get("pre"):
        pre = desc["pre"]
        n = np.clip(rq(normed(r, pre["norm"], desc["eps"]), pre["mult"], pre["shift"]) + pre["bias"], *pre["clamp"])
    return out, n
