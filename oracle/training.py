"""Plain forms of the training operators for tests: AdamW, the 8-bit moments,
the gradient norm, and the mixture-of-experts router, with numpy in 64 bits.

``adamw32`` states the same update with every operation rounded to float32 in
the order that the C header gives, so that moments can be compared bit for bit.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 256
WEYL_M = (0x9E3779B9, 0xBB67AE85)
WEYL_V = (0x6A09E667, 0x9E3779B9)


# ---- AdamW ----------------------------------------------------------------------------------

def adamw64(p, m, v, g, *, lr, b1, b2, eps, wd, t, factor=1.0):
    """One step in 64 bits: (p, m, v)."""
    p, m, v, g = (np.asarray(x, dtype=np.float64) for x in (p, m, v, g))
    g = g * factor
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    d = np.sqrt(v / (1 - b2**t)) + eps
    return p * (1 - lr * wd) - lr * (m / (1 - b1**t)) / d, m, v


def adamw32(m, v, g, *, b1, b2, factor=None):
    """The moments of one step, every operation rounded to float32: (m, v)."""
    f = np.float32
    m, v, g = (np.asarray(x, dtype=f) for x in (m, v, g))
    with np.errstate(over="ignore", invalid="ignore"):
        if factor is not None:
            g = g * f(factor)
        return f(b1) * m + f(1 - b1) * g, f(b2) * v + f(1 - b2) * (g * g)


def dither(n, t, weyl):
    i = np.arange(n, dtype=np.uint64)
    return ((i * np.uint64(weyl[0]) + np.uint64(t * weyl[1] % 2**32)) % np.uint64(2**32) >> np.uint64(12)).astype(np.int64)


def encode(x, t, *, signed):
    """8-bit codes of one tensor's moment and every block's top step: (uint8[n], int64[blocks])."""
    x = np.ascontiguousarray(x, dtype=np.float32)
    n, span = x.size, 127 if signed else 255
    bits = x.view(np.uint32).astype(np.int64) & 0x7FFFFFFF
    step = np.minimum(bits + dither(n, t, WEYL_M if signed else WEYL_V) >> 20, 2039)      # of finite values
    blocks = -(-n // BLOCK)
    padded = np.zeros(blocks * BLOCK, dtype=np.int64)
    padded[:n] = step
    top = padded.reshape(blocks, BLOCK).max(axis=1)
    base = np.repeat(np.maximum(top, span) - span, BLOCK)[:n]
    code = np.clip(step - base, 0, span)
    if signed:
        code |= np.where((code > 0) & np.signbit(x), 128, 0)
    else:
        code = np.where((x != 0) & (code == 0), 1, code)
    return code.astype(np.uint8), top


def decode(code, top, *, signed):
    span = 127 if signed else 255
    size = code.astype(np.int64) & span
    base = np.repeat(np.maximum(top, span) - span, BLOCK)[:code.size]
    x = np.where(size > 0, size + base << 20, 0).astype(np.uint32).view(np.float32)
    return np.where(code > span, -x, x).astype(np.float32)


def norm(grads, max_norm):
    """(norm, factor) of a list of gradients."""
    total = math.sqrt(math.fsum(float(x) * float(x) for g in grads for x in np.asarray(g, dtype=np.float64).ravel()))
    return total, max_norm / total if total > max_norm else 1.0


# ---- the router ---------------------------------------------------------------------------------

def route64(x, k, off, weights, *, valid=None, renormalise=False):
    """Forward pass in 64 bits: a dict like RouterOutputs, with ``p`` and ``counted``."""
    x = np.asarray(x, dtype=np.float64)
    T, E = x.shape
    K = len(off) - 1
    on = np.ones(T, dtype=bool) if valid is None else np.asarray(valid, dtype=bool)
    counted = on & (x > -np.inf).any(axis=1)
    mx = np.where(counted, x.max(axis=1, initial=-np.inf), 0.0)
    with np.errstate(invalid="ignore", over="ignore"):
        ex = np.where(counted[:, None], np.exp(x - mx[:, None]), 0.0)
    total = ex.sum(axis=1)
    p = ex / np.where(counted, total, 1.0)[:, None]
    lse = np.where(counted, mx + np.log(np.where(counted, total, 1.0)), 0.0)
    idx = np.argsort(-x, axis=1, kind="stable")[:, :k]
    some = (np.take_along_axis(x, idx, axis=1) > -np.inf) & counted[:, None]
    gate = np.where(some, np.take_along_axis(p, idx, axis=1), 0.0)
    idx = np.where(some, idx, -1)
    if renormalise:
        sums = gate.sum(axis=1, keepdims=True)
        gate = gate / np.where(sums > 0, sums, 1.0)
    counts = np.zeros((K, E), dtype=np.int64)
    share, load, prob, z = np.zeros(K), np.zeros(E), np.zeros(E), 0.0
    for d in range(K):
        s = slice(off[d], off[d + 1])
        chosen = idx[s][counted[s]]
        counts[d] = np.bincount(chosen[chosen >= 0], minlength=E)
        n = int(counted[s].sum())
        if n:
            share[d] = 1.0 / n
            load += weights[d] * share[d] / k * counts[d]
            prob += weights[d] * share[d] * p[s].sum(axis=0)
            z += weights[d] * share[d] * (lse[s] ** 2).sum()
    return {"idx": idx, "gate": gate, "lse": lse, "counts": counts, "load": load, "share": share,
            "loss": np.array([E * (load * prob).sum(), z]), "p": p, "counted": counted}


def route_back64(f, off, weights, d_gate, d_loss, *, renormalise=False):
    """Gradient of the logits in 64 bits from route64's dict, and the sum of its terms' sizes."""
    p, idx, gate = f["p"], f["idx"], f["gate"]
    T, E = p.shape
    K = len(off) - 1
    scale = np.repeat(np.asarray(weights, dtype=np.float64) * f["share"], np.diff(off))[:, None]
    a, b = (0.0, 0.0) if d_loss is None else (float(y) for y in d_loss)
    mean = (p * f["load"]).sum(axis=1, keepdims=True)
    dx = scale * p * (a * E * (f["load"] - mean) + 2 * b * f["lse"][:, None])
    size = scale * p * (abs(a) * E * (f["load"] + mean) + 2 * abs(b) * np.abs(f["lse"])[:, None])
    if d_gate is not None:
        h = np.where(idx >= 0, gate * np.asarray(d_gate, dtype=np.float64), 0.0)
        part, parts = h.sum(axis=1, keepdims=True), np.abs(h).sum(axis=1, keepdims=True)
        rows = np.arange(T)[:, None]
        to = np.where(idx >= 0, idx, E)                       # a place of no expert
        def put(y):
            out = np.zeros((T, E + 1))
            np.add.at(out, (rows, to), y)
            return out[:, :E]
        if renormalise:
            dx, size = dx + put(h - gate * part), size + put(np.abs(h) + gate * parts)
        else:
            dx, size = dx + put(h) - p * part, size + put(np.abs(h)) + p * parts
    on = f["counted"][:, None]
    return np.where(on, dx, 0.0), np.where(on, size, 0.0)
