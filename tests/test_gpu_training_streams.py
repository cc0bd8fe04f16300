"""The training objects' calls on changing streams, with nothing but the objects
between them to keep their order, against the same calls on one stream."""
import numpy as np
import pytest

from _gpu_common import log, torch_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sc():
    import paper_2301_08897_amd as sc
    return sc


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(sc, bits):
    torch, dev = torch_dev()
    log(f"adamw on changing streams, bits={bits}")
    sizes = [3_000_001, 77, 2_000_000]
    gen = torch.Generator(device=dev).manual_seed(3)
    n = sum(sizes)
    flat = [torch.empty(n, device=dev).normal_(generator=gen) for _ in range(3)]
    mine, other = flat[0].clone(), flat[0].clone()
    sets = [list(torch.split(g, sizes)) for g in flat[1:]]
    a, b = (sc.AdamW(list(torch.split(p, sizes)), sets[0], state_bits=bits) for p in (mine, other))
    streams = [torch.cuda.Stream(), None, torch.cuda.Stream()]
    torch.cuda.synchronize()
    for i in range(12):
        s = [streams[(i + j * (1 + i % 2)) % 3] for j in range(4)]
        for opt, (p, q, u, v) in ((a, s), (b, [None] * 4)):
            clip = opt.grad_norm(1e3 + i, stream=p)
            opt.step(1e-3, clip=clip, stream=q)
            opt.set_grads(sets[(i + 1) % 2], stream=u)
            if i % 5 == 4:
                opt.load(opt.t, opt.m, opt.v, tops=opt.tops, stream=v)
    torch.cuda.synchronize()
    assert torch.equal(mine, other) and torch.equal(a.clip, b.clip)
    for x, y in zip(a.moments(), b.moments()):
        assert torch.equal(x, y)


def test_router(sc):
    torch, dev = torch_dev()
    T, E, k = 40_000, 64, 4
    log("router on changing streams")
    rng = np.random.default_rng(4)
    xs = [torch.from_numpy(rng.normal(0, 1.5, (T, E)).astype(np.float32)).to(dev) for _ in range(4)]
    dg, dl = torch.ones(T, k, device=dev), torch.ones(2, device=dev)
    r, q = sc.Router(T, E, k, devices=3), sc.Router(T, E, k, devices=3)
    streams = [torch.cuda.Stream(), None, torch.cuda.Stream()]
    torch.cuda.synchronize()
    out = {id(r): [], id(q): []}
    for i in range(9):
        x, off = xs[i % 4], [0, 1000 * i, 30_000, T]
        for router, s, t in ((r, streams[i % 3], streams[(i * i + 1) % 3]), (q, None, None)):
            f = router.forward(x, tok_off=off, stream=s)
            d = torch.empty_like(x)
            router.backward(x, f, dg, dl, d_logits=d, stream=t)
            out[id(router)].append(d)
        torch.cuda.synchronize() if i % 4 == 3 else None
    torch.cuda.synchronize()
    for i, (d, e) in enumerate(zip(out[id(r)], out[id(q)])):
        assert torch.equal(d, e), i
    for a in ("idx", "gate", "lse", "counts", "load", "share", "loss"):
        assert torch.equal(getattr(r, a), getattr(q, a)), a
