"""What the tests of the operators between tokens and logits share."""
from __future__ import annotations

import numpy as np

U = 2.0**-24                                    # half a step of float32
HALF = {"f32": 2.0**-24, "bf16": 2.0**-8}      # and of an output's type
FILL = 7.0


def bounds(T, K, rng):
    """Uneven devices, some of them empty."""
    cut = np.sort(rng.integers(0, T + 1, K - 1)) if K > 1 else np.zeros(0, dtype=np.int64)
    return [0] + [int(c) for c in cut] + [T]


def dtype(torch, kind):
    return torch.bfloat16 if kind == "bf16" else torch.float32


def tensor(torch, dev, a, kind, pad=0):
    """The array as a [rows, dim] tensor; with `pad` its rows lie dim + pad apart, from an
    address that is aligned to the elements only, with other values between them."""
    x = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(dev).to(dtype(torch, kind))
    if not pad:
        return x
    n, d = x.shape
    buf = torch.full((n * (d + pad) + pad,), FILL, dtype=x.dtype, device=dev)[pad:].view(n, d + pad)
    buf[:, :d] = x
    return buf[:, :d]


def space(torch, dev, n, d, kind, pad=0):
    """Room for an output in the same form, full of FILL."""
    return tensor(torch, dev, np.full((n, d), FILL), kind, pad)


def around(x):
    """The values between the rows of a padded tensor."""
    base = x._base
    return np.concatenate([base[: x.storage_offset()].float().cpu().numpy(),
                           base[x.storage_offset():].view(x.shape[0], x.stride(0))[:, x.shape[1]:].float().cpu().numpy().reshape(-1)])


def host(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


def near(got, want, room, kind="f32", what=""):
    """Every value of `got` within `room` before its rounding to the type, and that rounding."""
    room = np.broadcast_to(np.asarray(room, dtype=np.float64), want.shape)
    limit = room + (np.abs(want) + room) * HALF[kind] + 2.0**-149
    off = np.abs(host(got).reshape(want.shape) - want)
    bad = ~(off <= limit)
    assert not bad.any(), (what, int(bad.sum()), float(np.nanmax(off[bad] / limit[bad])) if bad.any() else 0.0)
