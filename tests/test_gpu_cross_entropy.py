"""The cross entropy of a linear layer and its gradients against the formulas in 64 bits:
one entry to several pieces of the vocabulary, one element to odd rows, devices without
rows, rows that are not counted, strides, far logits, replays."""
import numpy as np
import pytest

from _gpu_common import torch_dev
from _language import FILL, U, around, bounds, dtype, host, near, space, tensor
from oracle import language as ol

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sc():
    import paper_2301_08897_amd as sc
    return sc


def run(sc, T, V, dim, K, kind, grad, *, pad=0, padding=True, wide=True, forward_weights=False, scale=1.5, seed=0, check=True):
    torch, dev = torch_dev()
    rng = np.random.default_rng(seed + 31 * T + V + 7 * dim)
    off = bounds(T, K, rng)
    target = rng.integers(0, V, T)
    if padding and T > 1:
        target = np.where(rng.random(T) < 0.2, rng.choice([-1, V, -2**31, 2**31 - 1], T), target)
    on = (target >= 0) & (target < V)
    x = tensor(torch, dev, rng.normal(0, 1, (T, dim)), kind, pad)
    hx = host(x)
    if padding:
        x[torch.from_numpy(~on).to(dev)] = float("nan")           # rows that nothing may come of
    w = tensor(torch, dev, rng.normal(0, scale / dim**0.5, (V, dim)), kind, pad)
    ids = torch.from_numpy(target).to(torch.int64 if wide else torch.int32).to(dev)
    weights = rng.uniform(0, 1, K).astype(np.float32)
    h = sc.LinearCrossEntropy(V, dim, devices=K)
    f = h.forward(x, w, ids, tok_off=off, weights=weights)
    flat = torch.full((K, 1 + V * dim + 3), FILL, dtype=dtype(torch, grad), device=dev)
    dx = space(torch, dev, T, dim, kind, pad)
    d_loss = torch.tensor([-0.75], device=dev)
    got = h.backward(x, w, ids, f, [r[1:-3] for r in flat], tok_off=off, weights=weights if forward_weights else None, d_loss=d_loss, d_x=dx)
    assert got is dx
    if not check:
        return f, dx, flat
    hw = host(w)
    z, nll, lse, each, share, loss = ol.cross_entropy(hx, hw, target, off, weights.astype(np.float64))
    # a product's terms go through one addition per instruction of 32 and those within it; the matrix cores'
    # additions may be off by a step, not half of one. Floats are two half floats, each rounding 2^-11: 2^-22 of
    # them is left out, and the product of the second parts; below 2^-14 a half float's steps are 2^-24, where the
    # largest of the row is 2^13 at least: half a step is 2^-38 of that
    parts, floor = (3, 2.0**-38) if kind == "f32" else (1, 0.0)
    size = np.abs(hx) @ np.abs(hw).T
    e_z = size * (U * (2 * (parts * (dim // 32 + 1) + 40) + 2) + (3 * 2.0**-22 if parts == 3 else 0.0))
    e_z += floor * (np.abs(hx).max(axis=1)[:, None] * np.abs(hw).sum(axis=1) + np.abs(hx).sum(axis=1)[:, None] * np.abs(hw).max(axis=1))
    span = float(np.ptp(z[on])) if on.any() else 0.0
    # exponentials: their argument and 1.44 times it are rounded, and the result; 32 of a lane, the lanes, the tiles
    e_sum = U * (4 * span + 8 + 40 + V // 256 / 16 + 32 * 4)
    e_lse = (e_z.max(axis=1) + e_sum + 3 * U * np.abs(lse)) * on
    near(f.lse, lse, e_lse)
    at = np.where(on, target, 0)
    e_nll = (e_lse + e_z[np.arange(T), at]) * on + 2 * U * np.abs(nll)
    near(f.nll, nll, e_nll)
    assert not host(f.nll)[~on].any() and not host(f.lse)[~on].any()
    near(f.share, share, 0)
    e_each = np.array([e_nll[a:b].sum() for a, b in zip(off, off[1:])]) * share
    near(f.device_loss, each, e_each)
    near(f.loss, np.array([loss]), (e_each * weights).sum())
    # gradients
    c = share * -0.75 * (weights.astype(np.float64) if forward_weights else 1.0)
    g, want_dx, want_dw = ol.cross_entropy_gradients(hx, hw, target, off, z, lse, c)
    p = np.exp(z - lse[:, None])
    e_g = np.where(on[:, None], np.abs(np.repeat(c, np.diff(off)))[:, None] * p * (e_z + e_lse[:, None] + U * (4 * span + 8)), 0.0)
    e_g += 8 * U * np.abs(g)
    # what is below 2^-126, the least normal float and bfloat16, may become zero: the exponential (times a factor
    # below 1), its product with the factor, and each of the three parts; so a term is off by up to 5 * 2^-126 |x|
    e_g += 5 * 2.0**-126 * on[:, None]
    # G, and the other operand: one bfloat16 if everything is; else two half floats of 2^13 G (one suffices for bfloat16
    # gradients), and bfloat16 x and weight are half floats but for what is below a column's largest by 2^-38
    half = (kind, grad) != ("bf16", "bf16")
    low = 2.0**-38 if half else 0.0
    e_g += low * np.where(on[:, None], np.abs(np.repeat(c, np.diff(off)))[:, None], 0.0)
    for_x = 2.0**-8 if not half else 2.0**-11 if kind == "bf16" else 3 * 2.0**-22
    for_w = 2.0**-8 if not half else 2.0**-10 if (kind, grad) == ("f32", "bf16") else 3 * 2.0**-22
    pieces = 32
    steps = lambda n: 2 * U * (3 * (n // 32 + 2) + 40 + pieces)  # noqa: E731
    room = (e_g + np.abs(g) * for_x) @ np.abs(hw) + (np.abs(g) @ np.abs(hw)) * steps(V)
    near(dx, want_dx, room + low * np.abs(g).sum(axis=1)[:, None] * np.abs(hw).max(axis=0), kind, "d_x")
    dw = flat[:, 1:-3].reshape(K, V, dim)
    top = np.abs(hx[on]).max(axis=0) if on.any() else np.zeros(dim)
    for k in range(K):
        s = slice(off[k], off[k + 1])
        xk = np.where(on[s, None], np.abs(hx[s]), 0.0)
        room = (e_g[s] + np.abs(g[s]) * for_w).T @ xk + (np.abs(g[s]).T @ xk) * steps(T)
        near(dw[k], want_dw[k], room + low * np.abs(g[s]).sum(axis=0)[:, None] * top, grad, "d_weight")
    assert bool((flat[:, 0] == FILL).all()) and bool((flat[:, -3:] == FILL).all())
    assert not host(dx)[~on].any()
    if pad and T > 1:
        assert np.all(around(dx) == FILL)
    return f, dx, flat


TYPES = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")]
SHAPES = [(1, 1, 1, 1), (1, 300, 64, 1), (3, 2, 5, 2), (64, 256, 64, 1), (65, 255, 63, 2), (130, 257, 128, 5), (300, 1000, 65, 3), (257, 513, 200, 1),
          (700, 70, 512, 64), (40, 5000, 33, 4), (1000, 600, 264, 2)]


@pytest.mark.parametrize("kind,grad", TYPES)
@pytest.mark.parametrize("T,V,dim,K", SHAPES)
def test_cross_entropy(sc, T, V, dim, K, kind, grad):
    run(sc, T, V, dim, K, kind, grad)


@pytest.mark.parametrize("kind,grad", TYPES)
def test_strides_and_weights(sc, kind, grad):
    run(sc, 200, 300, 64, 3, kind, grad, pad=3, wide=False, forward_weights=True)
    run(sc, 200, 300, 64, 3, kind, grad, pad=8, padding=False)


@pytest.mark.parametrize("kind,grad", TYPES)
def test_several_pieces_of_the_vocabulary(sc, kind, grad):
    run(sc, 16_500, 8300, 16, 3, kind, grad)


def test_far_logits(sc):
    run(sc, 90, 400, 64, 2, "f32", "f32", scale=40.0)
    run(sc, 90, 400, 64, 2, "bf16", "f32", scale=40.0)


def test_nothing_is_counted(sc):
    torch, dev = torch_dev()
    h = sc.LinearCrossEntropy(50, 16, devices=2)
    x, w = torch.randn(9, 16, device=dev), torch.randn(50, 16, device=dev)
    for T, off in ((9, [0, 4, 9]), (0, [0, 0, 0])):
        ids = torch.full((T,), -1, device=dev)
        f = h.forward(x[:T], w, ids, tok_off=off, weights=[0.5, 0.5])
        assert not f.loss.any() and not f.device_loss.any() and not f.share.any() and not f.nll.any()
        dw = torch.full((2, 50, 16), FILL, device=dev)
        dx = h.backward(x[:T], w, ids, f, dw, tok_off=off)
        assert not dx.any() and not dw.any() and dx.shape == (T, 16)


def test_without_the_table_s_gradient(sc):
    torch, dev = torch_dev()
    h = sc.LinearCrossEntropy(300, 40)
    x, w, ids = torch.randn(70, 40, device=dev), torch.randn(300, 40, device=dev), torch.randint(300, (70,), device=dev)
    f = h.forward(x, w, ids)
    assert torch.equal(h.backward(x, w, ids, f), h.backward(x, w, ids, f, torch.empty(300, 40, device=dev)))


def test_a_row_that_is_not_finite_stays_alone(sc):
    torch, dev = torch_dev()
    h = sc.LinearCrossEntropy(300, 64)
    x, w, ids = torch.randn(70, 64, device=dev), torch.randn(300, 64, device=dev), torch.randint(300, (70,), device=dev)
    f = h.forward(x, w, ids)
    d = h.backward(x, w, ids, f)
    x2 = x.clone()
    x2[5, 3] = float("nan")
    f2 = h.forward(x2, w, ids)
    d2 = h.backward(x2, w, ids, f2)
    rest = [i for i in range(70) if i != 5]
    assert torch.equal(f.nll[rest], f2.nll[rest]) and torch.equal(d[rest], d2[rest])
    assert bool(f2.nll[5].isnan()) and bool(d2[5].isnan().all())


def test_logits_at_minus_infinity(sc):
    """Infinities in a bfloat16 table mask its entries."""
    torch, dev = torch_dev()
    h = sc.LinearCrossEntropy(300, 64)
    x = torch.rand(70, 64, device=dev).add_(0.5).to(torch.bfloat16)
    w = torch.randn(300, 64, device=dev).to(torch.bfloat16)
    ids = torch.randint(0, 256, (70,), device=dev)
    small = sc.LinearCrossEntropy(256, 64).forward(x, w[:256], ids)
    w[256:] = float("-inf")
    f = h.forward(x, w, ids)
    assert torch.equal(f.nll, small.nll) and torch.equal(f.lse, small.lse)


def test_gradients_are_the_differences(sc):
    torch, dev = torch_dev()
    rng = np.random.default_rng(5)
    T, V, dim = 12, 20, 6
    t = lambda *s: torch.from_numpy(rng.normal(0, 1, s).astype(np.float32)).to(dev)  # noqa: E731
    x, w, sx, sw = t(T, dim), t(V, dim), t(T, dim), t(V, dim)
    ids = torch.from_numpy(rng.integers(0, V, T)).to(dev)
    h = sc.LinearCrossEntropy(V, dim)
    f = h.forward(x, w, ids)
    dw = torch.empty(V, dim, device=dev)
    dx = h.backward(x, w, ids, f, dw)
    value = lambda x, w: float(h.forward(x, w, ids).nll.double().mean())  # noqa: E731
    e = 2.0**-7
    dot = lambda a, b: float((a.double() * b.double()).sum())  # noqa: E731
    # nll below 20, off by 50 U of it; a logit's change along the step is below 30 (its second along both is 0 in x
    # alone or w alone), the third derivative of log sum exp below 30^3 / 5
    room = 20 * 50 * U / e + 30**3 / 5 * e * e / 6
    assert abs((value(x + e * sx, w) - value(x - e * sx, w)) / (2 * e) - dot(dx, sx)) < room
    assert abs((value(x, w + e * sw) - value(x, w - e * sw)) / (2 * e) - dot(dw, sw)) < room


def test_replays_and_streams(sc):
    torch, dev = torch_dev()
    T, V, dim, K = 500, 900, 72, 3
    off = [0, 100, 100, 500]
    h = sc.LinearCrossEntropy(V, dim, devices=K)
    x, w = torch.randn(T, dim, device=dev), torch.randn(V, dim, device=dev)
    ids = torch.randint(-50, V, (T,), device=dev)
    dw, dw2 = torch.empty(K, V, dim, device=dev), torch.empty(K, V, dim, device=dev)
    h.backward(x, w, ids, h.forward(x, w, ids, tok_off=off), dw, tok_off=off)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f2 = h.forward(x, w, ids, tok_off=off)
        dx2 = h.backward(x, w, ids, f2, dw2, tok_off=off)
    for _ in range(4):
        x.mul_(-1.1).add_(0.01)
        graph.replay()
        f = h.forward(x, w, ids, tok_off=off)
        dx = h.backward(x, w, ids, f, dw, tok_off=off)
        torch.cuda.synchronize()
        assert torch.equal(dx, dx2) and torch.equal(dw, dw2) and torch.equal(f.loss, f2.loss)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    dx3 = h.backward(x, w, ids, h.forward(x, w, ids, tok_off=off, stream=s), dw2, tok_off=off, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(dx, dx3) and torch.equal(dw, dw2)
