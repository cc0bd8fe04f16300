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
