"""The router over the whole range of finite logits: row maxima of both signs
from 1e5 to 1e38, and finite values of large size in place of -infinity as
masks, against the formulas in 64 bits.

Bounds. U is the unit roundoff. An exponential's argument of size s carries at
most 4 s U of relative error (difference, constant, product, result), and
beyond s = 104 the exponential is below the smallest float; sums and quotients
add at most 48 U as everywhere in these tests. lse is the row's maximum plus a
logarithm: 2 U relative to it, whatever its size. An exponential below 2^-126
may become zero."""
import math

import numpy as np
import pytest

from _gpu_common import log, torch_dev
from oracle import training as ot

pytestmark = pytest.mark.gpu
U = 2.0**-24
NEAR = U * (48 + 4 * 104)
FLT_MAX = float(np.finfo(np.float32).max)
SIZES = [1e5, 2.0**20 - 1.0, 2.0**20, 2.0**20 + 1.0, 1e7, 1e9, 1.5e9, 4e9, 5e9, 1e10, 1e12, 1e20, 9e29, 1e30, 1e38]


@pytest.fixture(scope="module")
def sc():
    import paper_2301_08897_amd as sc
    return sc


def rows_of(b, E, rng):
    """Rows whose values are of size b: equal, a few steps of a float apart,
    spread by half, and masks of that size among ordinary values."""
    out = []
    for sign in (1.0, -1.0):
        step = float(np.spacing(np.float32(b)))
        out += [np.full((4, E), sign * b), sign * b + step * rng.integers(-3, 4, (8, E)), sign * b * (1 + 0.5 * rng.random((4, E))),
                np.where(rng.random((8, E)) < 0.5, sign * b, rng.normal(0, 1.5, (8, E)))]
    x = np.concatenate(out + [rng.normal(0, 1.5, (8, E))])
    return x[rng.permutation(len(x))].astype(np.float32)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("shape", [(1, 1), (3, 2), (8, 2), (16, 16), (31, 5), (60, 4), (64, 8), (100, 8), (200, 8), (256, 2), (500, 3), (1000, 16)],
                         ids=str)
def test_every_size(sc, shape, bf16):
    torch, dev = torch_dev()
    E, k = shape
    log(f"router range {shape} bf16={bf16}")
    for b in SIZES:
        rng = np.random.default_rng(int(math.log2(b) * 1000) + E)
        x = torch.from_numpy(rows_of(b, E, rng)).to(dev)
        x = x.to(torch.bfloat16) if bf16 else x
        T, host = x.shape[0], x.float().cpu().numpy()
        assert np.isfinite(host).all()
        off, w = [0, T // 3, T], np.array([0.25, 0.75], dtype=np.float32)
        dg, dl = rng.normal(0, 1.0, (T, k)).astype(np.float32), np.array([0.7, -0.3], dtype=np.float32)
        for renormalise in (False, True):
            r = sc.Router(T, E, k, devices=2, renormalise=renormalise)
            f = r.forward(x, tok_off=off, weights=w)
            got = {n: getattr(f, n).cpu().numpy().astype(np.float64) for n in ("idx", "gate", "lse", "counts", "load", "loss")}
            want = ot.route64(host, k, off, w.astype(np.float64), renormalise=renormalise)
            assert np.array_equal(got["idx"], want["idx"]) and np.array_equal(got["counts"], want["counts"]), b
            assert np.all(np.abs(got["gate"] - want["gate"]) <= NEAR * want["gate"] + 1e-37), b
            assert np.all(np.abs(got["lse"] - want["lse"]) <= NEAR + 2 * U * np.abs(want["lse"])), b
            assert np.all(np.abs(got["load"] - want["load"]) <= 2 * U * want["load"]), b
            assert abs(got["loss"][0] - want["loss"][0]) <= (NEAR + 300 * U) * want["loss"][0], b
            if want["loss"][1] > FLT_MAX:
                assert got["loss"][1] == math.inf, b
            else:                               # 2 |lse| d <= d (1 + lse^2)
                assert abs(got["loss"][1] - want["loss"][1]) <= (4 * NEAR + 8 * U) * (1 + want["loss"][1]), b
            dx = r.backward(x, f, torch.from_numpy(dg).to(dev), torch.from_numpy(dl).to(dev)).float().cpu().numpy().astype(np.float64)
            ref, size = ot.route_back64(want, off, w, dg, dl, renormalise=renormalise)
            # lse may be off by 8 where its neighbours are that far apart: exponentials of e^8 times their size become zero
            lost = 2.0**-126 * math.exp(8.0) * (2 * 0.7 * E + 2 * 0.3 * np.abs(want["lse"]).max() + 5 * k)
            tol = (4 * NEAR + 64 * U) * size + (2.0**-8 * np.abs(ref) if bf16 else 0.0) + lost
            assert np.all(np.abs(dx - ref) <= tol), (b, float((np.abs(dx - ref) / tol).max()))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("b", [1e9, 5e9, 1e10, 1e20, 9e29])
def test_padding_filled_with_large_values(sc, b, bf16):
    """Rows filled with one large value of either sign change nothing but the sums
    that they belong to, and their own gates are even."""
    torch, dev = torch_dev()
    T, E, k = 300, 64, 4
    x = torch.from_numpy(np.random.default_rng(5).normal(0, 1.5, (T, E)).astype(np.float32)).to(dev)
    x = x.to(torch.bfloat16) if bf16 else x
    r, q = sc.Router(T, E, k), sc.Router(T, E, k)
    f = r.forward(x)
    y = x.clone()
    y[::7], y[3::7] = -b, b
    rest = torch.ones(T, dtype=torch.bool, device=dev)
    rest[::7] = rest[3::7] = False
    g = q.forward(y)
    for n in ("idx", "gate", "lse"):
        assert torch.equal(getattr(f, n)[rest], getattr(g, n)[rest]), n
    assert torch.equal(g.idx[~rest], torch.arange(k, dtype=torch.int32, device=dev).expand(int((~rest).sum()), k))
    assert bool(((g.gate[~rest] * E - 1).abs() <= 48 * U).all())
    assert int(g.counts.sum()) == T * k and abs(float(g.load.sum()) - 1) <= 70 * U and math.isfinite(float(g.loss[0]))
    dx, dy = r.backward(x, f, torch.ones(T, k, device=dev)), q.backward(y, g, torch.ones(T, k, device=dev))
    assert torch.equal(dx[rest], dy[rest]) and bool(torch.isfinite(dy).all())
