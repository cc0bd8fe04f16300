"""Plain forms of the operators between tokens and logits for tests, with numpy in 64 bits."""
from __future__ import annotations

import numpy as np


# ---- tokens sorted by expert --------------------------------------------------------------

def order(idx, experts, off):
    """(pos, src, bounds) of choices idx [T, k]; an index outside the experts is missing."""
    T, k = idx.shape
    K = len(off) - 1
    flat = idx.reshape(-1).astype(np.int64)
    there = (flat >= 0) & (flat < experts)
    device = np.repeat(np.arange(K), np.diff(off) * k)
    rows = [i for i in np.argsort(np.where(there, flat * K + device, experts * K), kind="stable") if there[i]]
    pos, src = np.full(T * k, -1), np.full(T * k, -1)
    pos[rows], src[: len(rows)] = np.arange(len(rows)), rows
    cell = np.bincount((flat * K + device)[there], minlength=experts * K)
    return pos.reshape(T, k).astype(np.int32), src.astype(np.int32), np.concatenate([[0], np.cumsum(cell)]).astype(np.int32)


def combine(rows, gate, pos):
    """(sums [T, dim], sums of the products' magnitudes)."""
    on = (pos >= 0)[:, :, None]
    part = np.where(on, rows.astype(np.float64)[np.maximum(pos, 0)] * np.where(on, gate[:, :, None], 0.0), 0.0)
    return part.sum(axis=1), np.abs(part).sum(axis=1)
