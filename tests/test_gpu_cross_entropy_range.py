"""The gradients of the cross entropy of a linear layer where magnitudes lie far apart: rows of
a table masked with finite values, a device beside one with huge rows, huge rows beside
others of their device, improbable entries, terms that cancel."""
import numpy as np
import pytest

from _gpu_common import torch_dev
from _language import U, dtype, host, near
from oracle import language as ol

pytestmark = pytest.mark.gpu

TYPES = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")]


@pytest.fixture(scope="module")
def sc():
    import paper_2301_08897_amd as sc
    return sc


def both(sc, x, w, ids, off, grad):
    """(forward's, d_x, d_weight) of one call each."""
    torch, dev = torch_dev()
    K = len(off) - 1
    h = sc.LinearCrossEntropy(w.shape[0], w.shape[1], devices=K)
    f = h.forward(x, w, ids, tok_off=off, weights=[1.0] * K)
    dw = torch.empty(K, *w.shape, dtype=dtype(torch, grad), device=dev)
    return f, h.backward(x, w, ids, f, dw, tok_off=off), dw


@pytest.mark.parametrize("low", [-1e6, -1e30, "lowest"])
@pytest.mark.parametrize("kind,grad", TYPES)
def test_rows_masked_with_finite_values(sc, kind, grad, low):
    """They have probability 0, so that all else is what it is without them, bit for bit."""
    torch, dev = torch_dev()
    V, M, dim, T = 290, 9, 64, 70                     # as many steps of the products with the rows as without
    t = dtype(torch, kind)
    x, w = (torch.rand(T, dim, device=dev) + 0.5).to(t), torch.randn(V + M, dim, device=dev).to(t)
    ids = torch.randint(0, V, (T,), device=dev)
    f, dx, dw = both(sc, x, w[:V], ids, [0, T], grad)
    w[V:] = torch.finfo(t).min if low == "lowest" else low
    f2, dx2, dw2 = both(sc, x, w, ids, [0, T], grad)
    assert torch.equal(f.nll, f2.nll)
    assert torch.equal(dx, dx2) and bool((dx != 0).any())
    assert torch.equal(dw, dw2[:, :V]) and not dw2[:, V:].any()


@pytest.mark.parametrize("size", [1e9, 1e30])
@pytest.mark.parametrize("kind,grad", TYPES)
def test_a_device_beside_one_with_huge_rows(sc, kind, grad, size):
    torch, dev = torch_dev()
    V, dim, off = 300, 40, [0, 33, 100]
    t = dtype(torch, kind)
    x, w = torch.randn(100, dim, device=dev).to(t), torch.randn(V, dim, device=dev).to(t)
    ids = torch.randint(0, V, (100,), device=dev)
    f, dx, dw = both(sc, x, w, ids, off, grad)
    x2 = x.clone()
    x2[:33] *= size
    f2, dx2, dw2 = both(sc, x2, w, ids, off, grad)
    assert torch.equal(f.nll[33:], f2.nll[33:])
    assert torch.equal(dw[1], dw2[1]) and torch.equal(dx[33:], dx2[33:])
    assert bool(dw2.isfinite().all()) and bool(dx2.isfinite().all())


def sums(T):
    """What a sum over T tokens or entries is off by, relative to the sum of its terms' magnitudes: up to six products,
    each with one addition per instruction of 32 and those within it, a step each; the units and pieces."""
    return 2 * U * (6 * (T // 32 + 2) + 40 + 32)


# What the parts that are multiplied leave out of a product. bfloat16 roundings are off by 2^-8, so that the second
# and third part are below 2^-8 and 2^-16 and three parts leave 2^-24; six products leave out 2 * 2^-24 and less, and
# the three parts' rests. Two parts leave 2^-16 each, and the product of the second ones.
LEFT_X = {("f32", "f32"): 5 * U, ("f32", "bf16"): 5 * U, ("bf16", "f32"): 2.0**-16, ("bf16", "bf16"): 2.0**-8}
LEFT_W = {("f32", "f32"): 5 * U, ("f32", "bf16"): 4 * 2.0**-16, ("bf16", "f32"): 2 * U, ("bf16", "bf16"): 2.0**-8}


@pytest.mark.parametrize("size", [1e9, 1e25])
@pytest.mark.parametrize("kind,grad", TYPES)
def test_a_huge_row_beside_others_of_its_device(sc, kind, grad, size):
    """Its probabilities are 1 and 0, so that it adds nothing to the table's gradient but in two rows; there it is most of it."""
    torch, dev = torch_dev()
    rng = np.random.default_rng(3)
    T, V, dim = 90, 200, 24
    t = dtype(torch, kind)
    x, w = torch.from_numpy(rng.normal(0, 1, (T, dim))).to(dev).to(t), torch.from_numpy(rng.normal(0, 0.3, (V, dim))).to(dev).to(t)
    x[5] *= size
    target = rng.integers(0, V, T)
    f, dx, dw = both(sc, x, w, torch.from_numpy(target).to(dev), [0, T], grad)
    hx, hw = host(x), host(w)
    z, nll, lse, each, share, loss = ol.cross_entropy(hx, hw, target, [0, T], np.ones(1))
    g, want_dx, want_dw = ol.cross_entropy_gradients(hx, hw, target, [0, T], z, lse, share)
    top = np.sort(z[5])
    assert top[-1] - top[-2] > 1e-4 * np.abs(z[5]).max()       # so that no rounding decides
    e_g = error_of_g(hx, hw, z, lse, target, kind) / T
    e_g[5] = 0.0
    left, floor = LEFT_W[kind, grad], 2.0**-126
    room = (e_g + np.abs(g) * (left + sums(T)) + floor).T @ np.abs(hx)
    two = [int(z[5].argmax()), int(target[5])]
    rest = np.setdiff1d(np.arange(V), two)
    room_rest = (e_g + np.abs(g) * (left + sums(T)) + floor)[np.arange(T) != 5].T @ np.abs(hx[np.arange(T) != 5])
    near(dw[0][torch.from_numpy(rest).to(dev)], want_dw[0][rest], room_rest[rest], grad, "other rows")
    near(dw[0][torch.tensor(two, device=dev)], want_dw[0][two], room[two], grad, "the two rows")
    left = LEFT_X[kind, grad]
    near(dx, want_dx, (e_g + np.abs(g) * (left + sums(V)) + floor) @ np.abs(hw), kind, "d_x")


def error_of_g(hx, hw, z, lse, target, kind):
    """How far softmax minus one may be off. Logits of floats come from two half floats each: 2^-22 of a factor and
    the product of the second parts are left out; below 2^-14 a half float's steps are 2^-24, where the largest of the
    row is 2^13 at least."""
    dim, V = hx.shape[1], len(hw)
    size = np.abs(hx) @ np.abs(hw).T
    parts = 3 if kind == "f32" else 1
    e_z = size * (U * (2 * (parts * (dim // 32 + 1) + 40) + 2) + (3 * 2.0**-22 if parts == 3 else 0.0))
    if parts == 3:
        e_z += 2.0**-38 * (np.abs(hx).max(axis=1)[:, None] * np.abs(hw).sum(axis=1) + np.abs(hx).sum(axis=1)[:, None] * np.abs(hw).max(axis=1))
    p = np.exp(z - lse[:, None])
    # exponentials: their argument and 1.44 times it are rounded, and the result; 32 of a lane, the lanes, the tiles
    span = np.ptp(z, axis=1)[:, None]
    e_lse = (p * e_z).sum(axis=1)[:, None] * 2 + U * (4 * span + 8 + 40 + V // 256 / 16 + 32 * 4) + 3 * U * np.abs(lse)[:, None]
    g = p.copy()
    g[np.arange(len(z)), target] -= 1.0
    return p * (e_z + e_lse + U * (4 * span + 8)) + 8 * U * np.abs(g)


@pytest.mark.parametrize("far", [20.0, 30.0, 60.0])
@pytest.mark.parametrize("kind,grad", TYPES)
def test_improbable_entries(sc, kind, grad, far):
    """Entries that are no token's target have gradients of their probabilities alone, down to e^-60, each with the
    precision of its own size."""
    torch, dev = torch_dev()
    rng = np.random.default_rng(11)
    T, V, dim, some = 150, 320, 32, 64
    t = dtype(torch, kind)
    a, b = rng.normal(0, 1, (T, dim)), rng.normal(0, 0.2, (V, dim))
    a[:, 0] = 1.0
    b[some:, 0] = -far
    x, w = torch.from_numpy(a).to(dev).to(t), torch.from_numpy(b).to(dev).to(t)
    target = rng.integers(0, some, T)
    f, dx, dw = both(sc, x, w, torch.from_numpy(target).to(dev), [0, T], grad)
    hx, hw = host(x), host(w)
    z, nll, lse, each, share, loss = ol.cross_entropy(hx, hw, target, [0, T], np.ones(1))
    g, want_dx, want_dw = ol.cross_entropy_gradients(hx, hw, target, [0, T], z, lse, share)
    room = (error_of_g(hx, hw, z, lse, target, kind) / T + np.abs(g) * (LEFT_W[kind, grad] + sums(T)) + 2.0**-126).T @ np.abs(hx)
    assert np.median(room[some:] / np.abs(g).T[some:].sum(axis=1)[:, None]) < 2.0**-6        # a bound that says something
    near(dw[0], want_dw[0], room, grad)


@pytest.mark.parametrize("kind,grad", TYPES)
def test_terms_that_cancel(sc, kind, grad):
    """With a table of zeros all probabilities are 1 / V, and a column of ones makes d_x the sum of G, which is 0: what
    is left is what G is off by."""
    torch, dev = torch_dev()
    t, V = dtype(torch, kind), 6
    x, w = torch.zeros(V, 8, device=dev, dtype=t), torch.ones(V, 8, device=dev, dtype=t)
    ids = torch.arange(V, device=dev)
    f, dx, _ = both(sc, x, w, ids, [0, V], grad)
    left = LEFT_X[kind, grad]
    size = 2 * (V - 1) / V / V                          # of the magnitudes of a token's terms; its logarithm and exponentials: 24 U
    assert host(dx).__abs__().max() <= size * (left + 24 * U + sums(V)) * (1 + 2.0**-8)
    _, _, dw = both(sc, torch.ones_like(x), torch.zeros_like(w), ids, [0, V], grad)
    assert host(dw).__abs__().max() <= size * (LEFT_W[kind, grad] + 24 * U + sums(V)) * (1 + 2.0**-8)


def test_the_second_part_of_x_for_bfloat16_gradients(sc):
    """Two tokens with G of 1/2 and -1/2, apart by 2^-13."""
    torch, dev = torch_dev()
    x = torch.tensor([[1.0], [1.0 + 2.0**-13]], device=dev)
    f, dx, dw = both(sc, x, torch.zeros(2, 1, device=dev), torch.tensor([0, 1], device=dev), [0, 2], "bf16")
    want = 0.25 * 2.0**-13 * np.array([[1.0], [-1.0]])
    # G is off by its exponential and logarithm, 8 U each, and both products are rounded
    near(dw[0], want, np.full((2, 1), 0.5 * 20 * U), "bf16")


@pytest.mark.parametrize("V,hit", [(300, 299), (300, 7), (9000, 8000), (9000, 0)])
def test_logits_at_infinity(sc, V, hit):
    """The log-sum of a row with one is infinite, and so is the loss of any other target; rows that have it at -infinity,
    and other devices, are as without it."""
    torch, dev = torch_dev()
    T, dim, off = 70, 64, [0, 40, 70]
    x = torch.rand(T, dim, device=dev).add_(0.5).to(torch.bfloat16)
    x[40:] *= -1
    x[3] *= -1
    w = torch.randn(V, dim, device=dev).to(torch.bfloat16)
    ids = torch.randint(0, V - 2, (T,), device=dev)
    ids = torch.where(ids >= hit, ids + 1, ids)
    ids[5] = hit
    h = sc.LinearCrossEntropy(V, dim, devices=2)
    w[hit] = float("inf")
    f = h.forward(x, w, ids, tok_off=off, weights=[1.0, 1.0])
    rows = [t for t in range(40) if t != 3]
    assert bool((f.lse[rows] == float("inf")).all())
    assert bool((f.nll[[t for t in rows if t != 5]] == float("inf")).all()) and bool(f.nll[5].isnan())     # inf - inf
    keep = [3] + list(range(40, T))
    want = h.forward(-x.abs(), w, ids, tok_off=off, weights=[1.0, 1.0])       # the entry is at -infinity for every row
    assert torch.equal(f.lse[keep], want.lse[keep]) and torch.equal(f.nll[keep], want.nll[keep])
    assert bool(f.lse[keep].isfinite().all()) and bool(f.device_loss[1].isfinite())
    ids[5] = ids[6]
    f = h.forward(x, w, ids, tok_off=off, weights=[1.0, 1.0])
    assert f.device_loss[0] == float("inf") and f.loss[0] == float("inf") and torch.equal(f.device_loss[1], want.device_loss[1])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_logits_beyond_the_largest_float(sc, kind):
    torch, dev = torch_dev()
    V, dim, T = 600, 32, 9
    t = dtype(torch, kind)
    x, w = (torch.rand(T, dim, device=dev) + 0.5).to(t), torch.randn(V, dim, device=dev).to(t)
    x[4] = 0
    w[500] = torch.finfo(t).max
    f = sc.LinearCrossEntropy(V, dim).forward(x, w, torch.arange(T, device=dev))
    rest = [i for i in range(T) if i != 4]
    assert bool((f.lse[rest] == float("inf")).all()) and bool((f.nll[rest] == float("inf")).all())
    assert abs(float(f.lse[4]) - float(np.log(V))) <= 8 * U * np.log(V) + 24 * U


@pytest.mark.parametrize("kind,grad", TYPES)
def test_devices_without_counted_rows_under_an_infinite_gradient(sc, kind, grad):
    """The sum over no rows is 0, whatever it is multiplied with."""
    torch, dev = torch_dev()
    T, V, dim, off = 400, 70, 24, [0, 100, 100, 400]
    t = dtype(torch, kind)
    x, w = torch.randn(T, dim, device=dev).to(t), torch.randn(V, dim, device=dev).to(t)
    ids = torch.randint(0, V, (T,), device=dev)
    ids[100:] = -1
    h = sc.LinearCrossEntropy(V, dim, devices=3)
    f = h.forward(x, w, ids, tok_off=off)
    dw = torch.ones(3, V, dim, dtype=dtype(torch, grad), device=dev)
    dx = h.backward(x, w, ids, f, dw, tok_off=off, d_loss=torch.tensor([float("inf")], device=dev))
    assert not dw[1:].any() and not dx[100:].any() and not dw[0].isfinite().any()
