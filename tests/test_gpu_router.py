"""The mixture-of-experts router against its formulas in 64 bits: choices and
counts exactly, gates, losses and gradients within their roundings; masks,
ties, strides, uneven and empty devices, graphs and streams."""
import math

import numpy as np
import pytest

from _gpu_common import log, same_bits, torch_dev
from oracle import training as ot

pytestmark = pytest.mark.gpu
U = 2.0**-24


@pytest.fixture(scope="module")
def sc():
    import paper_2301_08897_amd as sc
    return sc


#: (tokens, experts, k, devices)
SHAPES = [(1, 1, 1, 1), (1, 8, 2, 1), (5, 3, 3, 2), (64, 8, 2, 1), (300, 16, 16, 4), (257, 17, 4, 3), (129, 31, 5, 1),
          (1000, 60, 4, 8), (513, 64, 8, 2), (200, 100, 1, 64), (333, 128, 8, 5), (400, 255, 16, 3), (2048, 256, 8, 32),
          (100, 500, 8, 2), (70, 1000, 16, 2), (71, 1024, 3, 1), (140_001, 8, 2, 5), (30_000, 130, 3, 7)]


def bounds(T, K, rng):
    """Uneven devices, some of them empty."""
    cut = np.sort(rng.integers(0, T + 1, K - 1)) if K > 1 else np.zeros(0, dtype=np.int64)
    return [0] + [int(c) for c in cut] + [T]


def logits(T, E, kind, rng):
    x = rng.normal(0, 1.5, (T, E))
    if kind == "zeros":                         # a few other values, then zeros, half or few of them positive
        sign = rng.random((T, E)) < rng.choice([0.02, 0.05, 0.5], (T, 1))
        x = np.where(rng.random((T, E)) < rng.choice([0.0, 0.01], (T, 1)), x, np.where(sign, 0.0, -0.0))
    if kind == "ties":
        x = np.round(x * 2) / 2 + 0.0 * x
        x[rng.random((T, E)) < 0.1] = -0.0
    if kind == "masked":
        x[rng.random((T, E)) < 0.4] = -np.inf
        x[rng.random(T) < 0.1] = -np.inf
    if kind == "lowest":
        x[rng.random((T, E)) < 0.5] = np.finfo(np.float32).min
        x[rng.random(T) < 0.1] = np.finfo(np.float32).min
    if kind == "large":
        x = x * 5 + 3000.0
    return x.astype(np.float32)


def compare(sc, T, E, k, K, kind, *, bf16=False, renormalise=False, padding=False, pad=0, seed=0, check_back=True):
    torch, dev = torch_dev()
    rng = np.random.default_rng(seed + T * 7 + E)
    x = torch.from_numpy(logits(T, E, kind, rng)).to(dev)
    if bf16:
        x = x.to(torch.bfloat16)
        if kind == "lowest":                    # rounding to bfloat16 would give -inf
            x = torch.where(torch.isinf(x), torch.finfo(torch.bfloat16).min, x)
    buf = torch.full((T, E + pad), 7.0, dtype=x.dtype, device=dev).flatten()[pad:] if pad else None
    if pad:                                     # rows that start at odd addresses, with other data between them
        buf = torch.full((T * (E + pad) + pad,), 7.0, dtype=x.dtype, device=dev)[pad:].view(T, E + pad)
        buf[:, :E] = x
        x = buf[:, :E]
    off = bounds(T, K, rng)
    w = np.diff(off).astype(np.float64) + 1.0
    w = (w / w.sum()).astype(np.float32)        # not the devices' shares: empty ones have a weight too
    valid = rng.random(T) < 0.8 if padding else None
    r = sc.Router(T + 3, E, k, devices=K, renormalise=renormalise)
    f = r.forward(x, tok_off=off, weights=w, valid=None if valid is None else torch.from_numpy(valid).to(dev))
    host = x.float().cpu().numpy()
    want = ot.route64(host, k, off, w.astype(np.float64), valid=valid, renormalise=renormalise)
    got = {n: getattr(f, n).cpu().numpy() for n in ("idx", "gate", "lse", "counts", "load", "share", "loss")}
    assert np.array_equal(got["idx"], want["idx"])
    assert np.array_equal(got["counts"], want["counts"])
    # an exponential's argument of size s is rounded to s U, its result again; sums add a rounding per
    # element of a lane and per exchange; the quotient one
    span = float(np.ptp(host[np.isfinite(host) & (np.abs(host) < 1e30)])) if np.isfinite(host).any() else 0.0
    near = U * (48 + 4 * span)
    assert np.all(np.abs(got["gate"] - want["gate"]) <= near * want["gate"] + 1e-37)
    assert np.all(np.abs(got["lse"] - want["lse"]) <= near + 2 * U * np.abs(want["lse"]))
    assert np.all(np.abs(got["load"] - want["load"]) <= 2 * U * want["load"])
    assert np.all(np.abs(got["share"] - want["share"]) <= 2 * U * want["share"])
    # sums of probabilities: at most 256 rounds in float, then double
    assert abs(got["loss"][0] - want["loss"][0]) <= (near + 300 * U) * abs(want["loss"][0])
    if want["loss"][1] > np.finfo(np.float32).max:
        assert got["loss"][1] == math.inf
    else:
        assert abs(got["loss"][1] - want["loss"][1]) <= (4 * near + 8 * U * np.abs(want["lse"]).max()) * (1 + want["loss"][1])
    again = r.forward(x, tok_off=off, weights=w, valid=None if valid is None else torch.from_numpy(valid).to(dev))
    for n in got:
        a, b = got[n], getattr(again, n).cpu().numpy()
        assert np.array_equal(a.view(np.uint32), b.view(np.uint32)), f"{n} depends on the order of the workgroups"
    if not check_back:
        return
    dg = rng.normal(0, 1.0, (T, k)).astype(np.float32)
    dl = np.array([0.7, -0.3], dtype=np.float32)
    for d_gate, d_loss, weights in ((dg, dl, None), (dg, None, None), (None, dl, np.ones(K, dtype=np.float32))):
        out = torch.full((T * (E + pad) + pad,), 5.0, dtype=x.dtype, device=dev)[pad:].view(T, E + pad)[:, :E] if pad else None
        dx = r.backward(x, f, None if d_gate is None else torch.from_numpy(d_gate).to(dev),
                        None if d_loss is None else torch.from_numpy(d_loss).to(dev), weights=weights, d_logits=out)
        ref, size = ot.route_back64(want, off, w if weights is None else weights, d_gate, d_loss, renormalise=renormalise)
        dx = dx.float().cpu().numpy()
        tol = (4 * near + 64 * U) * size + (2.0**-8 * np.abs(ref) if bf16 else 0.0) + 1e-37
        assert np.all(np.abs(dx - ref) <= tol), float((np.abs(dx - ref) / tol).max())
        if pad and T > 1:
            assert bool((out._base.view(-1)[pad:].view(T, E + pad)[:-1, E:] == 5.0).all()), "wrote between the rows"


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_shapes(sc, shape, bf16):
    log(f"router {shape} bf16={bf16}")
    compare(sc, *shape, "normal", bf16=bf16, renormalise=bf16, padding=shape[0] % 2 == 0)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("kind", ["ties", "masked", "lowest", "large", "zeros"])
@pytest.mark.parametrize("shape", [(5, 3, 3, 2), (300, 16, 16, 4), (1000, 60, 4, 8), (400, 255, 16, 3), (100, 500, 8, 2), (71, 1024, 3, 1),
                                   (600, 100, 8, 2), (600, 200, 3, 2)], ids=str)
def test_values(sc, shape, kind, bf16):
    log(f"router {kind} {shape} bf16={bf16}")
    for renormalise in (False, True):
        compare(sc, *shape, kind, bf16=bf16, renormalise=renormalise, padding=renormalise, seed=1)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("pad", [1, 3, 8])
def test_strides(sc, pad, bf16):
    log(f"router pad={pad} bf16={bf16}")
    for shape in ((77, 7, 2, 3), (200, 64, 8, 2), (50, 257, 4, 1)):
        compare(sc, *shape, "normal", bf16=bf16, pad=pad, seed=2)


def test_masks_that_leave_nothing(sc):
    torch, dev = torch_dev()
    T, E, k, K = 100, 12, 3, 4
    rng = np.random.default_rng(3)
    x = torch.from_numpy(logits(T, E, "normal", rng)).to(dev)
    off = [0, 30, 30, 60, 100]
    valid = torch.ones(T, dtype=torch.bool, device=dev)
    valid[30:60] = False                              # device 2 has only padding, device 1 no rows
    r = sc.Router(T, E, k, devices=K)
    f = r.forward(x, tok_off=off, weights=[0.25] * 4, valid=valid)
    assert f.share.tolist() == [np.float32(1 / 30), 0.0, 0.0, np.float32(1 / 40)]
    assert not bool(f.counts[1:3].any()) and bool((f.idx[30:60] == -1).all()) and not bool(f.gate[30:60].any())
    dx = r.backward(x, f, torch.ones(T, k, device=dev), torch.ones(2, device=dev))
    assert not bool(dx[30:60].any()) and bool(torch.isfinite(dx).all())
    f = r.forward(x, tok_off=off, weights=[0.25] * 4, valid=torch.zeros_like(valid))
    assert f.loss.tolist() == [0.0, 0.0] and not bool(f.load.any()) and not bool(f.counts.any())
    assert not bool(r.backward(x, f, torch.ones(T, k, device=dev), torch.ones(2, device=dev)).any())
    f = r.forward(x[:0], tok_off=[0] * 5, weights=[0.25] * 4)
    assert f.idx.shape == (0, k) and f.loss.tolist() == [0.0, 0.0] and not bool(f.counts.any())
    assert r.backward(x[:0], f, torch.ones(0, k, device=dev)).shape == (0, E)


@pytest.mark.parametrize("renormalise", [False, True])
def test_garbage_in_masked_places(sc, renormalise):
    """NaN and infinities in the logits of padding, and in the gradients of
    choices that are missing, change nothing."""
    torch, dev = torch_dev()
    T, E, k = 300, 60, 4
    rng = np.random.default_rng(10)
    x = torch.from_numpy(logits(T, E, "normal", rng)).to(dev)
    x[::7, 2:] = -math.inf                            # two experts left for four choices
    valid = torch.from_numpy(rng.random(T) < 0.7).to(dev)
    dg, dl = torch.from_numpy(rng.normal(0, 1, (T, k)).astype(np.float32)).to(dev), torch.ones(2, device=dev)
    r, q = (sc.Router(T, E, k, renormalise=renormalise) for _ in range(2))
    f = r.forward(x, valid=valid)
    dx = r.backward(x, f, torch.where(f.idx >= 0, dg, 0.0), dl)
    y = x.clone()
    y[~valid] = torch.tensor([math.nan, math.inf, -math.inf], device=dev).repeat(E // 3)
    g = q.forward(y, valid=valid)
    for bad in (math.nan, math.inf):
        dy = q.backward(y, g, torch.where(g.idx >= 0, dg, bad), dl)
        assert torch.equal(dx, dy) and bool(torch.isfinite(dx).all()) and not bool(dx[~valid].any())
    for n in ("idx", "gate", "lse", "counts", "load", "share", "loss"):
        assert torch.equal(getattr(f, n), getattr(g, n)), n


def test_rows_do_not_depend_on_their_neighbours(sc):
    """A row's choices, gates and gradient are the same bits wherever it lies."""
    torch, dev = torch_dev()
    for E, k in ((8, 2), (60, 4), (256, 8), (700, 12)):
        rng = np.random.default_rng(E)
        row = torch.from_numpy(logits(1, E, "normal", rng)).to(dev)
        dg = torch.ones(1, k, device=dev)
        r = sc.Router(100, E, k)
        f = r.forward(row)
        want = [x.clone() for x in (f.idx, f.gate, f.lse, r.backward(row, f, dg))]
        x = torch.from_numpy(logits(100, E, "masked", rng)).to(dev)
        x[10:20] = float(np.finfo(np.float32).min)
        x[20:30, 1] = math.inf
        x[30:40] *= 1e3
        x[5::9] = row
        f = r.forward(x)
        dx = r.backward(x, f, torch.ones(100, k, device=dev))
        for a, b in zip(want, (f.idx, f.gate, f.lse, dx)):
            assert torch.equal(a.expand_as(b[5::9]) if b.dim() > 1 else a.expand(b[5::9].shape), b[5::9]), (E, k)


@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_not_finite(sc, bad, renormalise):
    """A row with a NaN or +infinity is NaN where it is computed, and nowhere else."""
    torch, dev = torch_dev()
    T, E, k = 200, 60, 4
    x = torch.from_numpy(logits(T, E, "normal", np.random.default_rng(4))).to(dev)
    r = sc.Router(T, E, k, renormalise=renormalise)
    fine = {n: getattr(r.forward(x), n).clone() for n in ("idx", "gate", "lse")}
    x[17, 5] = bad
    x[90] = math.nan
    f = r.forward(x)
    rows = torch.ones(T, dtype=torch.bool, device=dev)
    rows[[17, 90]] = False
    assert all(torch.equal(getattr(f, n)[rows], fine[n][rows]) for n in fine)
    assert bool(torch.isnan(f.gate[~rows]).all()) and bool(torch.isnan(f.lse[~rows]).all())
    assert bool(torch.isnan(f.loss).all())
    assert bool((f.idx >= -1).all()) and bool((f.idx < E).all()) and bool(torch.isfinite(f.load).all())
    dx = r.backward(x, f, torch.ones(T, k, device=dev), torch.ones(2, device=dev))
    assert bool(torch.isnan(dx[~rows]).all()) and bool(torch.isfinite(dx[rows]).all())


def test_gradient_by_differences(sc):
    """The gradient against central differences of the same passes in 64 bits (the
    load held constant, as the definition has it)."""
    torch, dev = torch_dev()
    T, E, k, K = 12, 9, 3, 2
    rng = np.random.default_rng(6)
    x = logits(T, E, "normal", rng)
    off, w = [0, 5, 12], np.array([0.4, 0.6], dtype=np.float32)
    for renormalise in (False, True):
        dg = rng.normal(0, 1, (T, k)).astype(np.float32)
        r = sc.Router(T, E, k, devices=K, renormalise=renormalise)
        f = r.forward(torch.from_numpy(x).to(dev), tok_off=off, weights=w)
        dx = r.backward(torch.from_numpy(x).to(dev), f, torch.from_numpy(dg).to(dev), torch.tensor([0.5, 0.25], device=dev)).cpu().numpy()
        base = ot.route64(x, k, off, w, renormalise=renormalise)

        def value(y):
            g = ot.route64(y, k, off, w, renormalise=renormalise)
            gate = np.take_along_axis(g["p"], base["idx"], axis=1)      # the choice held as well
            if renormalise:
                gate = gate / gate.sum(axis=1, keepdims=True)
            prob = sum(w[d] * g["share"][d] * g["p"][off[d]:off[d + 1]].sum(axis=0) for d in range(K))
            return (gate * dg).sum() + 0.5 * E * (base["load"] * prob).sum() + 0.25 * g["loss"][1]

        h = 1e-5
        for t in range(T):
            for e in range(E):
                up, down = x.astype(np.float64), x.astype(np.float64)
                up[t, e] += h
                down[t, e] -= h
                slope = (value(up) - value(down)) / (2 * h)
                assert abs(dx[t, e] - slope) <= 1e-5 * (1 + abs(slope))


def test_other_streams_and_smaller_calls(sc):
    torch, dev = torch_dev()
    T, E, k = 5000, 64, 4
    x = torch.from_numpy(logits(T, E, "normal", np.random.default_rng(8))).to(dev)
    dg = torch.ones(T, k, device=dev)
    r, q = sc.Router(T, E, k, devices=2), sc.Router(70_000, E, k, devices=2)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for n in (T, 1, 63, 64, 65, 1000):
        f = r.forward(x[:n], tok_off=[0, n // 3, n])
        dx = r.backward(x[:n], f, dg[:n], torch.ones(2, device=dev))
        side.wait_stream(torch.cuda.current_stream())
        g = q.forward(x[:n], tok_off=[0, n // 3, n], stream=side)
        dy = q.backward(x[:n], g, dg[:n], torch.ones(2, device=dev), stream=side)
        torch.cuda.synchronize()
        for a in ("idx", "gate", "lse", "counts", "load", "loss"):
            assert torch.equal(getattr(f, a), getattr(g, a)), (n, a)
        assert torch.equal(dx, dy)


def test_every_smaller_call_fits_the_workspace(sc):
    """However many of max_tokens rows a call has, the workspace is large enough (host only)."""
    torch, dev = torch_dev()
    for E in (8, 64, 256, 1024):
        r = sc.Router(40_000, E, 1, devices=3)
        x = torch.zeros(40_000, E, device=dev)
        for n in (40_000, 16_385, 16_384, 16_383, 4097, 4096, 4095, 1025, 1024, 3):
            f = r.forward(x[:n], tok_off=[0, n // 2, n // 2 + 1, n])
            assert int(f.counts.sum()) == n and int(f.counts[:, 0].sum()) == n      # all tied: the lowest index


def test_graph(sc):
    torch, dev = torch_dev()
    for T, K in ((50, 1), (3000, 4)):
        E, k = 64, 4
        x = torch.zeros(T, E, device=dev)
        dg, dl = torch.ones(T, k, device=dev), torch.ones(2, device=dev)
        off = [T * d // K for d in range(K + 1)]
        r, q = sc.Router(T, E, k, devices=K), sc.Router(T, E, k, devices=K)
        dx = torch.empty_like(x)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f = r.forward(x, tok_off=off)
            r.backward(x, f, dg, dl, d_logits=dx)
        rng = np.random.default_rng(9)
        for i in range(4):
            x.copy_(torch.from_numpy(logits(T, E, "normal", rng)))
            graph.replay()
            g = q.forward(x, tok_off=off)
            dy = q.backward(x, g, dg, dl)
            torch.cuda.synchronize()
            for a in ("idx", "gate", "lse", "counts", "load", "loss"):
                assert torch.equal(getattr(f, a), getattr(g, a)), (i, a)
            assert torch.equal(dx, dy)


def test_more_than_2_to_32_logits(sc):
    """Rows whose offsets pass 32 bits, in more workgroups than one launch usually has."""
    torch, dev = torch_dev()
    B, E, k, times = 4096, 64, 2, 16_400
    log(f"router {B * times} x {E}")
    block = torch.from_numpy(logits(B, E, "normal", np.random.default_rng(11))).to(dev).to(torch.bfloat16)
    x = block.repeat(times, 1)
    T = x.shape[0]
    assert T * E > 2**32
    small = sc.Router(B, E, k)
    f = small.forward(block)
    dg = torch.ones(B, k, device=dev)
    dl = torch.ones(2, device=dev)
    dx = small.backward(block, f, dg, dl)
    r = sc.Router(T, E, k, devices=2)
    off = [0, B * 5000, T]
    g = r.forward(x, tok_off=off)
    for lo in (0, B * 5000, T - B):
        assert torch.equal(g.idx[lo:lo + B], f.idx) and torch.equal(g.gate[lo:lo + B], f.gate) and torch.equal(g.lse[lo:lo + B], f.lse)
    assert torch.equal(g.counts[0], f.counts[0] * 5000) and torch.equal(g.counts[1], f.counts[0] * (times - 5000))
    assert torch.allclose(g.load, f.load, rtol=1e-6) and torch.allclose(g.loss, f.loss, rtol=1e-5)
    # the losses' part is times as small per row: without it the gradient is the block's own
    own = small.backward(block, f, dg, None)
    dy = r.backward(x, g, dg.repeat(times, 1), None)
    for lo in (0, B * 5000, T - B):
        assert torch.equal(dy[lo:lo + B], own)
    assert not torch.equal(dx, own)
