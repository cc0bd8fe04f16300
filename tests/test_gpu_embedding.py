"""The embedding's rows and its gradients against their definition: padding, ids often and
never used, devices without tokens, sums of long runs, strides, accumulation, replays."""
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


def words(T, V, kind, rng):
    ids = rng.integers(0, V, T)
    if kind == "often":                     # one id for most tokens, another for many
        ids = np.where(rng.random(T) < 0.6, V // 2, np.where(rng.random(T) < 0.5, V - 1, ids))
    if kind == "one":
        ids[:] = V - 1
    if kind == "padded":
        ids = np.where(rng.random(T) < 0.3, -1, ids)
        ids = np.where(rng.random(T) < 0.05, V, ids)
        ids = np.where(rng.random(T) < 0.05, 2**31 - 1, ids)
    if kind == "nothing":
        ids[:] = -1
    return ids


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,dim,pad,wide", [(1, 1, 1, 0, True), (0, 5, 3, 0, False), (5, 7, 3, 1, False), (300, 1000, 129, 3, True),
                                              (64, 50, 2048, 0, True), (2000, 31, 8, 0, False), (3, 4, 9001, 5, True)])
def test_forward(sc, T, V, dim, pad, wide, kind):
    torch, dev = torch_dev()
    rng = np.random.default_rng(T + V)
    ids = words(T, V, "padded", rng)
    w = tensor(torch, dev, rng.normal(0, 1, (V, dim)), kind, pad)
    tokens = torch.from_numpy(ids).to(torch.int64 if wide else torch.int32).to(dev)
    if wide and T:
        tokens[0] = 2**40 + 1               # not an id of 32 bits
        ids[0] = -1
    out = space(torch, dev, T, dim, kind, pad) if T else None
    got = sc.Embedding(V, dim, scale=0.3).forward(tokens, w, out=out)
    want = ol.embed(ids, host(w), float(np.float32(0.3)))
    near(got, want, np.abs(want) * U, kind)
    assert pad == 0 or T == 0 or np.all(around(out) == FILL)


#: (tokens, vocabulary, dim, devices): one launch of the sort, several; one to three passes of it
BACK = [(1, 1, 1, 1), (1, 40_000, 8, 1), (33, 3, 5, 2), (500, 1, 16, 3), (1024, 1100, 129, 4), (1500, 70, 64, 64), (4096, 2000, 7, 5),
        (4097, 3000, 9, 5), (9000, 1023, 40, 2), (6000, 1024, 24, 1), (2000, 300, 1030, 2), (5000, 1_100_000, 2, 1)]


@pytest.mark.parametrize("words_kind", ["any", "often", "one", "padded", "nothing"])
@pytest.mark.parametrize("T,V,dim,K", BACK)
def test_backward(sc, T, V, dim, K, words_kind):
    torch, dev = torch_dev()
    rng = np.random.default_rng(T + V + dim)
    ids, off, scale = words(T, V, words_kind, rng), bounds(T, K, rng), -1.5
    for kind, grad, pad, add, wide in (("f32", "f32", 0, False, True), ("bf16", "f32", 3, False, False), ("bf16", "bf16", 0, True, True),
                                       ("f32", "bf16", 1, False, False), ("f32", "f32", 0, True, False)):
        g = tensor(torch, dev, rng.normal(0, 1, (T, dim)), kind, pad)
        # the gradients are parts of longer vectors, at offsets that are aligned to nothing else
        flat = torch.full((K, 3 + V * dim + 5), FILL, dtype=dtype(torch, grad), device=dev)
        flat[:, 3:-5] = 0.5 if add else float("nan")
        h = sc.Embedding(V, dim, scale=scale, devices=K)
        tokens = torch.from_numpy(ids).to(torch.int64 if wide else torch.int32).to(dev)
        h.backward(tokens, g, [f[3:-5] for f in flat], tok_off=off, accumulate=add)
        want, size = ol.embed_gradients(ids, host(g), V, scale, off)
        # the longest chain of additions: 32 tokens, the parts of a slice, the slices; the factor and the sum with what was there
        chain = 32 + T // 32 + 256
        start = 0.5 if add else 0.0
        near(flat[:, 3:-5].reshape(K, V, dim), want + start, size * U * chain + (size + start) * U * 2, grad, (kind, grad, add))
        assert bool((flat[:, :3] == FILL).all()) and bool((flat[:, -5:] == FILL).all())
        if add:
            untouched = size == 0
            assert np.all(host(flat[:, 3:-5]).reshape(K, V, dim)[untouched] == 0.5)


def test_gradients_are_the_differences(sc):
    torch, dev = torch_dev()
    rng = np.random.default_rng(4)
    T, V, dim = 60, 9, 5
    ids = torch.from_numpy(words(T, V, "padded", rng)).to(dev)
    h = sc.Embedding(V, dim, scale=2.0)
    w, step = (torch.from_numpy(rng.normal(0, 1, (V, dim)).astype(np.float32)).to(dev) for _ in range(2))
    g = torch.from_numpy(rng.normal(0, 1, (T, dim)).astype(np.float32)).to(dev)
    d = h.backward(ids, g, torch.empty(1, V, dim, device=dev))[0]
    value = lambda w: float((h.forward(ids, w).double() * g.double()).sum())  # noqa: E731
    # linear in the table: the difference's only errors are the 300 products' roundings
    got = (value(w + 0.5 * step) - value(w - 0.5 * step))
    assert abs(got - float((d.double() * step.double()).sum())) < 300 * 16 * U


def test_replays_and_repeats(sc):
    torch, dev = torch_dev()
    rng = np.random.default_rng(8)
    T, V, dim, K = 5000, 4000, 33, 3
    off = bounds(T, K, rng)
    h = sc.Embedding(V, dim, devices=K)
    ids = torch.from_numpy(words(T, V, "often", rng)).to(dev)
    g = torch.from_numpy(rng.normal(0, 1, (T, dim)).astype(np.float32)).to(dev)
    d, e = (torch.empty(K, V, dim, device=dev) for _ in range(2))
    h.backward(ids, g, d, tok_off=off)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h.backward(ids, g, e, tok_off=off)
    for seed in range(4):
        ids.copy_(torch.from_numpy(words(T, V, ["any", "often", "one", "padded"][seed], rng)))
        g.mul_(1.25)
        graph.replay()
        h.backward(ids, g, d, tok_off=off)
        torch.cuda.synchronize()
        assert torch.equal(d, e)            # the same bits, whatever the order of workgroups
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    f = torch.empty_like(e)
    h.backward(ids, g, f, tok_off=off, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(f, d)


def test_offsets_past_32_bits(sc):
    torch, dev = torch_dev()
    V, dim = 70_000, 40_000                 # 2.8e9 elements
    h = sc.Embedding(V, dim)
    ids = torch.tensor([V - 1, 0, V - 1], device=dev)
    g = torch.ones(3, dim, dtype=torch.bfloat16, device=dev)
    d = torch.full((V, dim), 3.0, dtype=torch.bfloat16, device=dev)
    h.backward(ids, g, d)
    assert bool((d[V - 1] == 2).all()) and bool((d[0] == 1).all()) and not bool(d[1:V - 1].any())
    assert bool((h.forward(ids, d)[0] == 2).all())
