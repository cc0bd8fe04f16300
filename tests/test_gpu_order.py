"""Tokens sorted by expert and back, against their definition: the order exactly, rows bit
for bit, sums and gradients within their roundings; missing choices, NaN where nothing is
read, strides, other streams, graphs."""
import numpy as np
import pytest

from _gpu_common import torch_dev
from _language import FILL, U, around, bounds, host, near, space, tensor
from oracle import language as ol

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sc():
    import paper_2301_08897_amd as sc
    return sc


#: (tokens, experts, k, devices): one chunk, two to eight rounds of it, several chunks, experts at the digits' limit
SHAPES = [(1, 1, 1, 1), (1, 8, 2, 1), (3, 5, 5, 2), (64, 8, 2, 1), (257, 17, 4, 3), (1024, 2, 1, 1), (1025, 60, 1, 4), (512, 1024, 4, 64),
          (2049, 1023, 4, 2), (8192, 31, 1, 5), (8193, 31, 1, 5), (5000, 1024, 3, 7), (20_000, 64, 16, 8), (90_000, 256, 3, 64)]


def choices(T, E, k, missing, rng):
    idx = rng.integers(0, E, (T, k))
    hot = rng.random((T, k)) < 0.3
    idx[hot] = E // 2
    if missing == "some":
        idx[rng.random((T, k)) < 0.2] = -1
        idx[rng.random(T) < 0.2] = -1
        idx[rng.random((T, k)) < 0.02] = E
        idx[rng.random((T, k)) < 0.02] = np.iinfo(np.int32).min
    if missing == "all":
        idx[:] = -1
    return idx.astype(np.int32)


def make(sc, torch, dev, T, E, k, K, missing, seed=0):
    rng = np.random.default_rng(seed + 13 * T + E)
    idx, off = choices(T, E, k, missing, rng), bounds(T, K, rng)
    h = sc.ExpertOrder(E, k, devices=K)
    return rng, idx, off, h, h.sort(torch.from_numpy(idx).to(dev), tok_off=off)


@pytest.mark.parametrize("missing", ["none", "some", "all"])
@pytest.mark.parametrize("T,E,k,K", SHAPES)
def test_sort(sc, T, E, k, K, missing):
    torch, dev = torch_dev()
    rng, idx, off, h, r = make(sc, torch, dev, T, E, k, K, missing)
    pos, src, b = ol.order(idx, E, off)
    assert np.array_equal(r.bounds.cpu().numpy(), b)
    assert np.array_equal(r.pos.cpu().numpy(), pos)
    assert np.array_equal(r.src.cpu().numpy(), src)


def test_sort_of_nothing(sc):
    torch, dev = torch_dev()
    r = sc.ExpertOrder(8, 2, devices=3).sort(torch.empty((0, 2), dtype=torch.int32, device=dev), tok_off=[0, 0, 0, 0])
    assert r.pos.shape == (0, 2) and r.src.numel() == 0 and not r.bounds.any() and r.bounds.numel() == 25


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("T,E,k,dim,pad,missing", [
    (1, 4, 1, 1, 0, "none"), (1, 8, 8, 2048, 0, "none"), (7, 3, 2, 3, 1, "some"), (64, 8, 2, 64, 0, "some"), (33, 16, 16, 129, 3, "some"),
    (130, 60, 5, 1001, 5, "some"), (500, 8, 3, 256, 0, "all"), (2000, 64, 8, 40, 0, "some"), (17, 4, 4, 9001, 7, "some"), (3001, 5, 1, 8, 0, "none")])
def test_rows(sc, T, E, k, dim, pad, missing, kind):
    torch, dev = torch_dev()
    rng, idx, off, h, r = make(sc, torch, dev, T, E, k, 1, missing)
    pos = ol.order(idx, E, off)[0]
    n = int((pos >= 0).sum())
    gate = rng.normal(0, 1, (T, k)).astype(np.float32)
    gate[pos < 0] = np.nan                                     # not read
    y = rng.normal(0, 1, (T * k, dim))
    y[n:] = np.nan                                             # nor these
    x, y, g = (tensor(torch, dev, a, kind, pad) for a in (rng.normal(0, 1, (T, dim)), y, rng.normal(0, 1, (T, dim))))
    gate_t = torch.from_numpy(gate).to(dev)
    # dispatch
    out = space(torch, dev, T * k, dim, kind, pad)
    rows = h.dispatch(x, r, out=out)
    assert rows is out
    want = np.full((T * k, dim), FILL)
    want[pos[pos >= 0]] = np.repeat(host(x), k, axis=0).reshape(T, k, dim)[pos >= 0]
    assert np.array_equal(host(rows), want)
    if pad:
        assert np.all(around(rows) == FILL)
    # combine: the gate's product is exact in 64 bits and rounded once or twice, and every addition once
    sums, size = ol.combine(host(y), gate.astype(np.float64), pos)
    out = space(torch, dev, T, dim, kind, pad)
    near(h.combine(y, gate_t, r, out=out), sums, size * U * (k + 1), kind)
    if pad:
        assert np.all(around(out) == FILL)
    # and back
    d_y = space(torch, dev, T * k, dim, kind, pad)
    d_rows, d_gate = h.combine_backward(g, y, gate_t, r, d_rows=d_y)
    at, on = np.maximum(pos, 0), pos >= 0
    product = np.where(on[:, :, None], host(y)[at] * host(g)[:, None, :], 0.0)
    # a lane adds its elements, then up to six exchanges
    near(d_gate, product.sum(axis=2), np.abs(product).sum(axis=2) * U * (dim // 8 + 16))
    want = np.full((T * k, dim), FILL)
    want[pos[on]] = (gate.astype(np.float64)[:, :, None] * host(g)[:, None, :])[on]
    near(d_rows, want, np.abs(want) * U, kind)
    assert np.array_equal(host(d_rows)[n:], want[n:])
    if pad:
        assert np.all(around(d_rows) == FILL)
    sums, size = ol.combine(host(y), np.ones_like(gate), pos)
    near(h.dispatch_backward(y, r), sums, size * U * k, kind)
    # the gradient in the place of the rows
    got, again = h.combine_backward(g, y, gate_t, r, d_rows=y)
    assert got is y and torch.equal(again, d_gate) and np.array_equal(host(y)[:n], host(d_rows)[:n])


def test_gradients_are_the_differences(sc):
    torch, dev = torch_dev()
    rng, idx, off, h, r = make(sc, torch, dev, 20, 4, 2, 1, "some")
    f = lambda *s: torch.from_numpy(rng.normal(0, 1, s).astype(np.float32)).to(dev)  # noqa: E731
    x, gate, g, step = f(20, 12), f(20, 2), f(20, 12), f(20, 12)
    value = lambda x, gate: float((h.combine(h.dispatch(x, r, out=torch.zeros(40, 12, device=dev)), gate, r).double() * g.double()).sum())  # noqa: E731
    rows = h.dispatch(x, r, out=torch.zeros(40, 12, device=dev))
    d_rows, d_gate = h.combine_backward(g, rows, gate, r, d_rows=torch.zeros_like(rows))
    d_x = h.dispatch_backward(d_rows, r)
    e = 0.25                                                   # both are linear: the differences have no error of their own
    # values are sums of 480 products of size 1: each off by U relative, and divided by e
    room = 480 * 8 * U / e
    assert abs((value(x + e * step, gate) - value(x - e * step, gate)) / (2 * e) - float((d_x.double() * step.double()).sum())) < room
    turn = f(20, 2)
    assert abs((value(x, gate + e * turn) - value(x, gate - e * turn)) / (2 * e) - float((d_gate.double() * turn.double()).sum())) < room


def test_positions_outside_are_missing(sc):
    """Positions that no sort gives are not followed."""
    torch, dev = torch_dev()
    h = sc.ExpertOrder(4, 2)
    pos = torch.tensor([[0, 6], [2**31 - 1, -2], [1, -(2**31)]], dtype=torch.int32, device=dev)
    r = sc.ExpertRows(pos, None, None)
    x = torch.arange(9.0, device=dev).view(3, 3)
    rows = h.dispatch(x, r, out=torch.full((6, 3), FILL, device=dev))
    assert torch.equal(rows[:2], x[[0, 2]]) and bool((rows[2:] == FILL).all())
    assert torch.equal(h.dispatch_backward(rows, r), torch.stack([x[0], torch.zeros(3, device=dev), x[2]]))


def test_offsets_past_32_bits(sc):
    torch, dev = torch_dev()
    T, dim = 70_000, 32_768                                    # 2.3e9 elements, 4.6e9 bytes
    h = sc.ExpertOrder(2, 1)
    idx = (torch.arange(T, dtype=torch.int32, device=dev) % 2)[:, None].contiguous()
    r = h.sort(idx)
    x = torch.zeros((T, dim), dtype=torch.bfloat16, device=dev)
    x[:, 0] = torch.arange(T, device=dev) % 251
    x[:, -1] = torch.arange(T, device=dev) % 241
    rows = h.dispatch(x, r)
    back = h.dispatch_backward(rows, r)
    assert torch.equal(back, x)
    want = torch.cat([x[0::2, -1], x[1::2, -1]])
    assert torch.equal(rows[:, -1], want)


def test_other_stream_and_replays(sc):
    torch, dev = torch_dev()
    rng, idx, off, h, r = make(sc, torch, dev, 700, 16, 2, 4, "some")
    idx = torch.from_numpy(idx).to(dev)
    x = torch.from_numpy(rng.normal(0, 1, (700, 24)).astype(np.float32)).to(dev)
    gate = torch.rand(700, 2, device=dev)
    want = h.combine(h.dispatch(x, r), gate, r)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = h.sort(idx, tok_off=off, stream=s)
    out = h.combine(h.dispatch(x, got, stream=s), gate, got, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r2 = h.sort(idx, tok_off=off)
        out = h.combine(h.dispatch(x, r2), gate, r2)
    for seed in range(4):
        idx.copy_(torch.from_numpy(choices(700, 16, 2, "some", np.random.default_rng(seed))))
        x.mul_(-1.5)
        g.replay()
        e = h.sort(idx, tok_off=off)
        want = h.combine(h.dispatch(x, e), gate, e)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(r2.pos, e.pos) and torch.equal(r2.bounds, e.bounds)


def test_after_the_router(sc):
    torch, dev = torch_dev()
    T, E, k, K = 500, 12, 3, 4
    off = [0, 10, 200, 200, 500]
    router = sc.Router(T, E, k, devices=K)
    f = router.forward(torch.randn(T, E, device=dev), tok_off=off, valid=torch.rand(T, device=dev) < 0.9)
    r = sc.ExpertOrder(E, k, devices=K).sort(f.idx, tok_off=off)
    assert torch.equal(r.bounds.diff().view(E, K), f.counts.T)
