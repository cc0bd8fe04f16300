"""Layer norm and its gradients against the formulas in 64 bits: rows of one element to rows
that do not fit registers, large means, equal rows, strides, devices without rows, replays."""
import numpy as np
import pytest

from _gpu_common import torch_dev
from _language import FILL, U, around, bounds, dtype, host, near, space, tensor
from oracle import language as ol

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def sc():
    import paper_2301_08897_amd as sc
    return sc


#: (rows, dim, devices)
SHAPES = [(1, 1, 1), (1, 8, 1), (5, 3, 2), (64, 64, 1), (33, 129, 3), (200, 256, 64), (40, 511, 2), (100, 1000, 4), (17, 2047, 1), (30, 2048, 2),
          (9, 4097, 2), (12, 8192, 3), (7, 8193, 2), (5, 20_001, 1), (20_000, 40, 5), (3000, 500, 1)]


def run(sc, T, dim, K, kind, weights, pad, bias, seed=0, x=None):
    torch, dev = torch_dev()
    rng = np.random.default_rng(seed + T + dim)
    off = bounds(T, K, rng)
    if x is None:
        x = rng.normal(0, 1, (T, dim)) * rng.uniform(0.1, 4, (T, 1)) + rng.normal(0, 1, (T, 1))
    x, g = tensor(torch, dev, x, kind, pad), tensor(torch, dev, rng.normal(0, 1, (T, dim)), kind, pad)
    w = torch.from_numpy(rng.normal(1, 0.3, dim).astype(np.float32)).to(dev).to(dtype(torch, weights))
    b = torch.from_numpy(rng.normal(0, 0.3, dim).astype(np.float32)).to(dev).to(dtype(torch, weights)) if bias else None
    h = sc.LayerNorm(dim, eps=EPS, devices=K)
    y, dx = space(torch, dev, T, dim, kind, pad), space(torch, dev, T, dim, kind, pad)
    f = h.forward(x, w, b, out=y)
    flat = torch.full((K, 1 + 2 * dim + 2), FILL, device=dev)       # parts of flat gradients, at odd addresses
    dw, db = flat[:, 1:1 + dim], flat[:, 1 + dim:1 + 2 * dim]
    d = h.backward(x, w, f, g, list(dw), list(db) if bias else None, tok_off=off, d_x=dx)
    assert d is dx and f.y is y
    if pad and T > 1:
        assert np.all(around(y) == FILL) and np.all(around(dx) == FILL)
    assert bool((flat[:, 0] == FILL).all()) and bool((flat[:, -2:] == FILL).all())
    if not bias:
        assert bool((db == FILL).all())
    # the definition
    hx, hw, hg = host(x), host(w), host(g)
    want_y, mean, rstd, hh = ol.layer_norm(hx, hw, None if b is None else host(b), float(np.float32(EPS)))
    want_dx, want_dw, want_db = ol.layer_norm_gradients(hh, rstd, hw, hg, off)
    # a lane adds up to 32 elements (more in long rows) and the lanes at most 8 exchanges; 1 / dim and the products round
    chain = 12 + max(32, dim // 256 + 1)
    e_mean = U * chain * np.abs(hx).mean(axis=1)
    near(f.mean, mean, e_mean)
    # (x - mean) is off by e_mean and a rounding, its square twice that; half of it in the root
    dev_x = np.abs(hx - mean[:, None])
    e_c = e_mean[:, None] + U * dev_x
    var = 1 / rstd**2
    e_var = (2 * dev_x * e_c + e_c**2).mean(axis=1) + U * chain * var
    e_r = rstd * (e_var / var / 2 * 1.01 + 4 * U) + 0.0
    near(f.rstd, rstd, e_r)
    e_h = e_c * rstd[:, None] + dev_x * e_r[:, None] + 2 * U * np.abs(hh)
    near(f.y, want_y, e_h * np.abs(hw) + 2 * U * (np.abs(hh * hw) + np.abs(want_y)), kind)
    e_w = U * np.abs(hg * hw)
    mean_w = np.abs(hg * hw).mean(axis=1, keepdims=True)
    a = U * (chain + 2) * mean_w
    bh = (hg * hw * hh).mean(axis=1, keepdims=True)
    e_b = U * (chain + 4) * np.abs(hg * hw * hh).mean(axis=1, keepdims=True) + (np.abs(hg * hw) * e_h).mean(axis=1, keepdims=True)
    e_in = e_w + a + e_h * np.abs(bh) + np.abs(hh) * e_b + 4 * U * (np.abs(hg * hw) + mean_w + np.abs(hh * bh))
    inner = np.abs(want_dx / rstd[:, None])
    near(dx, want_dx, e_in * rstd[:, None] + inner * e_r[:, None] + 2 * U * np.abs(want_dx), kind)
    # a group's rows one after the other, the groups, the workgroups' slices and those
    rows = max(16, T // 1024 + 1)
    deep = rows + 16 + 64 + 16
    for k in range(K):
        s = slice(off[k], off[k + 1])
        near(dw[k], want_dw[k], (np.abs(hg[s]) * (e_h[s] + U * (deep + 1) * np.abs(hh[s]))).sum(axis=0))
        if bias:
            near(db[k], want_db[k], np.abs(hg[s]).sum(axis=0) * U * deep)
    return f, dx, dw


@pytest.mark.parametrize("kind,weights,pad,bias", [("f32", "f32", 0, True), ("bf16", "f32", 3, True), ("bf16", "bf16", 0, False), ("f32", "bf16", 1, False)])
@pytest.mark.parametrize("T,dim,K", SHAPES)
def test_norm(sc, T, dim, K, kind, weights, pad, bias):
    run(sc, T, dim, K, kind, weights, pad, bias)


def test_large_means_keep_the_variance(sc):
    rng = np.random.default_rng(3)
    run(sc, 50, 700, 2, "f32", "f32", 0, True, x=rng.normal(0, 1, (50, 700)) + 1000.0)


def test_equal_elements(sc):
    """A row without variance gives the bias, and rstd = 1 / sqrt(eps)."""
    torch, dev = torch_dev()
    h = sc.LayerNorm(64, eps=EPS)
    b = torch.arange(64.0, device=dev)
    f = h.forward(torch.full((3, 64), 2.0, device=dev), torch.ones(64, device=dev), b)
    assert torch.equal(f.y, b.expand(3, 64)) and torch.allclose(f.rstd, torch.full((3,), EPS**-0.5, device=dev), rtol=1e-6)


def test_a_row_that_is_not_finite_stays_alone(sc):
    torch, dev = torch_dev()
    h = sc.LayerNorm(300)
    x, w = torch.randn(40, 300, device=dev), torch.randn(300, device=dev)
    want = h.forward(x, w)
    x2 = x.clone()
    x2[7, 5], x2[20, 0] = float("inf"), float("nan")
    got = h.forward(x2, w)
    rest = [i for i in range(40) if i not in (7, 20)]
    assert torch.equal(got.y[rest], want.y[rest]) and bool(got.y[[7, 20]].isnan().all())


def test_nothing(sc):
    torch, dev = torch_dev()
    h = sc.LayerNorm(10, devices=2)
    x, w = torch.empty(0, 10, device=dev), torch.ones(10, device=dev)
    f = h.forward(x, w)
    dw, db = torch.full((2, 10), FILL, device=dev), torch.full((2, 10), FILL, device=dev)
    assert h.backward(x, w, f, x, dw, db, tok_off=[0, 0, 0]).shape == (0, 10) and not dw.any() and not db.any()


def test_gradients_are_the_differences(sc):
    torch, dev = torch_dev()
    rng = np.random.default_rng(11)
    T, dim = 6, 24
    t = lambda *s: torch.from_numpy(rng.normal(0, 1, s).astype(np.float32)).to(dev)  # noqa: E731
    x, w, b, g, sx, sw, sb = t(T, dim), t(dim), t(dim), t(T, dim), t(T, dim), t(dim), t(dim)
    h = sc.LayerNorm(dim)
    f = h.forward(x, w, b)
    dw, db = torch.empty(1, dim, device=dev), torch.empty(1, dim, device=dev)
    dx = h.backward(x, w, f, g, dw, db)
    value = lambda x, w, b: float((h.forward(x, w, b).y.double() * g.double()).sum())  # noqa: E731
    e = 2.0**-6
    # values are sums of 144 terms of size 3: errors of 144 * 3 * 16 U / 2e; the curvature of a row adds e^2 times its
    # third derivative along the step, which is below 100 here
    room = 144 * 3 * 16 * U / (2 * e) + 100 * e * e
    dot = lambda a, b: float((a.double() * b.double()).sum())  # noqa: E731
    assert abs((value(x + e * sx, w, b) - value(x - e * sx, w, b)) / (2 * e) - dot(dx, sx)) < room
    assert abs((value(x, w + e * sw, b) - value(x, w - e * sw, b)) / (2 * e) - dot(dw[0], sw)) < room
    assert abs((value(x, w, b + e * sb) - value(x, w, b - e * sb)) / (2 * e) - dot(db[0], sb)) < room


def test_replays_and_streams(sc):
    torch, dev = torch_dev()
    T, dim, K = 900, 200, 3
    off = [0, 10, 10, 900]
    h = sc.LayerNorm(dim, devices=K)
    x, g, w = torch.randn(T, dim, device=dev), torch.randn(T, dim, device=dev), torch.randn(dim, device=dev)
    dw, dw2 = torch.empty(K, dim, device=dev), torch.empty(K, dim, device=dev)
    graph = torch.cuda.CUDAGraph()
    h.backward(x, w, h.forward(x, w), g, dw, tok_off=off)
    with torch.cuda.graph(graph):
        dx2 = h.backward(x, w, h.forward(x, w), g, dw2, tok_off=off)
    for _ in range(4):
        x.mul_(-1.5).add_(0.1)
        graph.replay()
        dx = h.backward(x, w, h.forward(x, w), g, dw, tok_off=off)
        torch.cuda.synchronize()
        assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    dx3 = h.backward(x, w, h.forward(x, w, stream=s), g, dw2, tok_off=off, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(dx, dx3) and torch.equal(dw, dw2)
