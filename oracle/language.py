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


# ---- embedding ------------------------------------------------------------------------------

def embed(ids, weight, scale):
    there = (ids >= 0) & (ids < len(weight))
    return np.where(there[:, None], weight.astype(np.float64)[np.where(there, ids, 0)] * scale, 0.0)


def embed_gradients(ids, d_out, vocab, scale, off):
    """(gradients [devices, vocab, dim], sums of the terms' magnitudes)."""
    K = len(off) - 1
    total = np.zeros((K, vocab, d_out.shape[1]))
    size = np.zeros_like(total)
    for d in range(K):
        for t in range(off[d], off[d + 1]):
            if 0 <= ids[t] < vocab:
                total[d, ids[t]] += scale * d_out[t]
                size[d, ids[t]] += abs(scale) * np.abs(d_out[t])
    return total, size


# ---- layer norm -------------------------------------------------------------------------------

def layer_norm(x, weight, bias, eps):
    """(y, mean, rstd, h)."""
    x = x.astype(np.float64)
    mean = x.mean(axis=1, keepdims=True)
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(axis=1, keepdims=True) + eps)
    h = (x - mean) * rstd
    return h * weight + (0.0 if bias is None else bias), mean[:, 0], rstd[:, 0], h


def layer_norm_gradients(h, rstd, weight, d_y, off):
    """(d_x, d_weight [devices, dim], d_bias)."""
    w = d_y * weight
    d_x = rstd[:, None] * (w - w.mean(axis=1, keepdims=True) - h * (w * h).mean(axis=1, keepdims=True))
    cut = list(zip(off, off[1:]))
    return d_x, np.stack([(d_y * h)[a:b].sum(axis=0) for a, b in cut]), np.stack([d_y[a:b].sum(axis=0) for a, b in cut])


# ---- cross entropy of a linear layer --------------------------------------------------------------

def cross_entropy(x, weight, target, off, weights):
    """(logits, nll, lse, device_loss, share, loss); rows of other targets are not counted."""
    z = x.astype(np.float64) @ weight.astype(np.float64).T
    on = (target >= 0) & (target < len(weight))
    top = z.max(axis=1)
    with np.errstate(invalid="ignore"):
        lse = np.where(on, top + np.log(np.exp(z - top[:, None]).sum(axis=1)), 0.0)
    nll = np.where(on, lse - z[np.arange(len(z)), np.where(on, target, 0)], 0.0)
    rows = np.array([on[a:b].sum() for a, b in zip(off, off[1:])])
    share = np.where(rows > 0, 1.0 / np.maximum(rows, 1), 0.0)
    each = np.array([nll[a:b].sum() for a, b in zip(off, off[1:])]) * share
    return z, nll, lse, each, share, float((each * weights).sum())


def cross_entropy_gradients(x, weight, target, off, z, lse, scale):
    """(G, d_x, d_weight [devices, vocab, dim]) with scale [devices] = weight * share."""
    on = (target >= 0) & (target < len(weight))
    g = np.exp(z - lse[:, None])
    g[np.arange(len(z))[on], target[on]] -= 1.0
    g = np.where(on[:, None], g * np.repeat(scale, np.diff(off))[:, None], 0.0)
    x = np.where(on[:, None], x, 0.0)
    return g, g @ weight, np.stack([g[a:b].T @ x[a:b] for a, b in zip(off, off[1:])])
