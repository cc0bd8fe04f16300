"""AdamW over many tensors at once: 32- and 8-bit moments, the gradient norm
with its clip factor, plans, streams and graphs, against the update in 64 bits
(within its roundings) and, for the moments, against the same float32
operations bit for bit."""
import math

import numpy as np
import pytest

from _gpu_common import log, same_bits, torch_dev
from oracle import training as ot

pytestmark = pytest.mark.gpu

HYPER = dict(b1=0.9, b2=0.999, eps=1e-8)
U = 2.0**-24            # unit roundoff of float32


@pytest.fixture(scope="module")
def sc():
    import paper_2301_08897_amd as sc
    return sc


SIZES = {
    "one": [1],
    "tails": [1, 2, 3, 4, 5, 255, 256, 257],
    "chunks": [2047, 2048, 2049, 4096, 4097],
    "empty": [0, 7, 0, 0, 300, 0],
    "many": [int(x) for x in np.random.default_rng(5).integers(1, 600, 133)],
    "long": [1_000_003, 64, 300_000],
}


def make(sizes, seed, *, bf16=False, offset=0, spread=True):
    """Parameters, gradients and moments of every tensor, as parts of flat
    buffers that start `offset` elements off their alignment."""
    torch, dev = torch_dev()
    rng = np.random.default_rng(seed)
    n = sum(sizes)
    scale = np.exp(rng.normal(0, 2.0, n)) * 1e-3 if spread else np.full(n, 1e-3)
    host = {"p": rng.normal(0, 0.05, n), "g": rng.normal(0, 1, n) * scale, "m": rng.normal(0, 0.3, n) * scale,
            "v": scale**2 * rng.uniform(0.5, 1.5, n)}
    for k in ("g", "m", "v"):
        host[k][rng.random(n) < 0.02] = 0.0
    host = {k: x.astype(np.float32) for k, x in host.items()}

    def flat(x, dtype=torch.float32):
        big = torch.zeros(n + offset, dtype=dtype, device=dev)
        big[offset:] = torch.from_numpy(x).to(dev)
        return big[offset:]

    t = {"p": flat(host["p"]), "g": flat(host["g"], torch.bfloat16 if bf16 else torch.float32)}
    host["g"] = t["g"].float().cpu().numpy()
    return host, t, [list(torch.split(t[k], sizes)) for k in ("p", "g")]


def cuts(x, sizes):
    return np.split(x, np.cumsum(sizes)[:-1])


def check_params(p, host, m, v, decay, sizes, t, lr, factor=1.0):
    """Parameters against 64 bits from the moments m, v before the step. Every
    product and sum of the update rounds once: the update term has at most 12
    roundings (with its factors'), the parameter's own two, and the sum one."""
    ref, off, at = [], [], 0
    for i, n in enumerate(sizes):
        s = slice(at, at + n)
        r, m1, v1 = ot.adamw64(host["p"][s], m[s], v[s], host["g"][s], lr=lr, wd=decay[i], t=t, factor=factor, **HYPER)
        ref.append(r)
        # m = b1 m + c1 g may cancel: its error is relative to its terms
        terms = 0.9 * np.abs(m[s].astype(np.float64)) + 0.1 * np.abs(host["g"][s].astype(np.float64)) * factor
        d = np.sqrt(v1 / (1 - HYPER["b2"]**t)) + HYPER["eps"]
        off.append(U * (4 * np.abs(host["p"][s]) + 16 * lr * terms / (1 - HYPER["b1"]**t) / d) + 1e-45)
        at += n
    assert np.all(np.abs(p.astype(np.float64) - np.concatenate(ref)) <= np.concatenate(off))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bf16,offset", [(False, 0), (False, 1), (True, 0), (True, 3)])
@pytest.mark.parametrize("name", list(SIZES))
def test_step(sc, name, bf16, offset, bits):
    torch, dev = torch_dev()
    sizes = SIZES[name]
    log(f"adamw {name} bits={bits} bf16={bf16} offset={offset}")
    host, t, (params, grads) = make(sizes, 11, bf16=bf16, offset=offset)
    decay = [0.01 if i % 2 else 0.0 for i in range(len(sizes))]
    copy = torch.zeros(sum(sizes) + offset, dtype=torch.bfloat16, device=dev)[offset:]
    opt = sc.AdamW(params, grads, weight_decay=decay, state_bits=bits, copies=list(torch.split(copy, sizes)))
    opt.load(41, torch.from_numpy(host["m"]).to(dev), torch.from_numpy(host["v"]).to(dev))
    m, v = (x.cpu().numpy() for x in opt.moments())
    if bits == 32:
        assert same_bits(m, host["m"]) and same_bits(v, host["v"])
    else:
        want = [[], []]
        for a, b in zip(cuts(host["m"], sizes), cuts(host["v"], sizes)):
            want[0].append(ot.decode(*ot.encode(a, 41, signed=True), signed=True))
            want[1].append(ot.decode(*ot.encode(b, 41, signed=False), signed=False))
        assert same_bits(m, np.concatenate(want[0])) and same_bits(v, np.concatenate(want[1]))
    lr = 1e-3
    for step in range(2):
        m0, v0 = m, v
        host["p"] = t["p"].cpu().numpy()
        opt.step(lr)
        torch.cuda.synchronize()
        assert opt.t == 42 + step
        m, v = (x.cpu().numpy() for x in opt.moments())
        m1, v1 = ot.adamw32(m0, v0, host["g"], b1=0.9, b2=0.999)
        if bits == 8:
            m1 = np.concatenate([ot.decode(*ot.encode(x, opt.t, signed=True), signed=True) for x in cuts(m1, sizes)])
            v1 = np.concatenate([ot.decode(*ot.encode(x, opt.t, signed=False), signed=False) for x in cuts(v1, sizes)])
        assert same_bits(m, m1) and same_bits(v, v1), f"moments differ at step {step}"
        p = t["p"].cpu().numpy()
        check_params(p, host, m0, v0, decay, sizes, opt.t, lr)
        assert torch.equal(copy.cpu(), torch.from_numpy(p).to(torch.bfloat16))
    if offset:          # what lies before the flat buffers is not touched
        assert float(t["p"]._base[:offset].abs().sum() if t["p"]._base is not None else 0.0) == 0.0


def test_moments_in_64_bits(sc):
    """32-bit moments against the formula in 64 bits: three roundings each and the constants'."""
    torch, dev = torch_dev()
    sizes = [100_003, 17]
    host, t, (params, grads) = make(sizes, 12)
    opt = sc.AdamW(params, grads)
    opt.load(7, torch.from_numpy(host["m"]).to(dev), torch.from_numpy(host["v"]).to(dev))
    opt.step(1e-3)
    m, v = (x.cpu().numpy().astype(np.float64) for x in opt.moments())
    _, m64, v64 = ot.adamw64(host["p"], host["m"], host["v"], host["g"], lr=1e-3, wd=0.0, t=8, **HYPER)
    g = host["g"].astype(np.float64)
    assert np.all(np.abs(m - m64) <= 4 * U * (0.9 * np.abs(host["m"]) + 0.1 * np.abs(g)))
    assert np.all(np.abs(v - v64) <= 5 * U * v64 + 2e-45)


def test_8bit_rounding_is_to_a_neighbour(sc):
    """A code stands for one of the two steps around the value, within the block's range."""
    torch, dev = torch_dev()
    n = 100_000
    host, t, (params, grads) = make([n], 13)
    opt = sc.AdamW(params, grads, state_bits=8)
    opt.load(3, torch.from_numpy(host["m"]).to(dev), torch.from_numpy(host["v"]).to(dev))
    m, v = (x.cpu().numpy() for x in opt.moments())
    for got, x, octaves in ((m, host["m"], 15.75), (v, host["v"], 31.75)):
        top = np.abs(np.pad(x, (0, -n % 256)).reshape(-1, 256)).max(axis=1).repeat(256)[:n]
        inside = np.abs(x) > top * 2.0**-octaves * 1.2
        assert inside.mean() > 0.9
        assert np.all(np.abs(got - x)[inside] <= np.abs(x)[inside] * 0.125)
        assert np.array_equal(got[x == 0], x[x == 0])
        assert abs((got[inside].astype(np.float64) / x[inside]).mean() - 1) < 2e-3     # no bias: sigma is 0.04 / sqrt(n)
    assert np.all(v[host["v"] > 0] > 0), "a v that is not zero never becomes zero"


def test_8bit_run_follows_the_32bit_run(sc):
    """1000 steps with noisy gradients: the 8-bit second moment stays at the
    32-bit one's on average (rounded to nearest it would stand at half of it)."""
    torch, dev = torch_dev()
    n = 65_536
    gen = torch.Generator(device=dev).manual_seed(5)
    scale = torch.exp(torch.empty(n, device=dev).normal_(generator=gen)) * 1e-3
    grad = torch.zeros(n, device=dev)
    a, b = (sc.AdamW([torch.zeros(n, device=dev)], [grad], weight_decay=0.0, state_bits=k) for k in (32, 8))
    for _ in range(1000):
        grad.normal_(0.2, 1.0, generator=gen).mul_(scale)
        a.step(1e-3)
        b.step(1e-3)
    ratio = (b.moments()[1] / a.moments()[1]).sqrt()
    assert abs(float(ratio.mean()) - 1) < 0.03 and float(ratio.std()) < 0.15
    move = float((a.params[0] - b.params[0]).norm() / a.params[0].norm())
    log(f"  sqrt(v) ratio {float(ratio.mean()):.4f} +- {float(ratio.std()):.4f}, parameters apart {move:.4f}")
    assert move < 0.1


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bf16", [False, True])
def test_clip(sc, bits, bf16):
    torch, dev = torch_dev()
    sizes = SIZES["many"]
    host, t, (params, grads) = make(sizes, 14, bf16=bf16, offset=1)
    opt = sc.AdamW(params, grads, weight_decay=0.01, state_bits=bits)
    total, _ = ot.norm([host["g"]], 1.0)
    for max_norm in (total / 3, total * 3, math.inf):
        norm, factor = (float(x) for x in opt.grad_norm(max_norm).cpu())
        assert norm == float(np.float32(total)) or abs(norm / total - 1) <= U
        want = min(1.0, max_norm / total)
        assert abs(factor / want - 1) <= 2 * U
    factor = float(opt.grad_norm(total / 3).cpu()[1])
    opt.step(1e-3, clip=opt.clip)
    m, v = (x.cpu().numpy() for x in opt.moments())
    zero = np.zeros(sum(sizes), dtype=np.float32)
    m1, v1 = ot.adamw32(zero, zero, host["g"], b1=0.9, b2=0.999, factor=factor)
    if bits == 8:
        m1 = np.concatenate([ot.decode(*ot.encode(x, 1, signed=True), signed=True) for x in cuts(m1, sizes)])
        v1 = np.concatenate([ot.decode(*ot.encode(x, 1, signed=False), signed=False) for x in cuts(v1, sizes)])
    assert same_bits(m, m1) and same_bits(v, v1)
    check_params(t["p"].cpu().numpy(), host, zero, zero, [0.01] * len(sizes), sizes, 1, 1e-3, factor)


@pytest.mark.parametrize("n", [1, 4, 1000, 2048 * 3 + 1, 5_000_011])
def test_norm(sc, n):
    torch, dev = torch_dev()
    rng = np.random.default_rng(n)
    for scale in (1.0, 1e-30, 1e30):
        g = (rng.normal(0, 1, n) * scale).astype(np.float32)
        opt = sc.AdamW([torch.zeros(n, device=dev)], [torch.from_numpy(g).to(dev)])
        a = opt.grad_norm(scale).cpu().numpy().copy()
        b = opt.grad_norm(scale).cpu().numpy()
        assert same_bits(a, b), "the norm depends on the order of the workgroups"
        want = math.sqrt(math.fsum((g.astype(np.float64) ** 2).tolist()))
        assert abs(float(a[0]) / want - 1) <= U * (1 + 1e-6)
        assert abs(float(a[1]) / min(1.0, scale / want) - 1) <= U * (1 + 1e-6)


def test_norm_beyond_float(sc):
    torch, dev = torch_dev()
    g = torch.full((100,), 3e38, device=dev)
    opt = sc.AdamW([torch.zeros(100, device=dev)], [g])
    norm, factor = (float(x) for x in opt.grad_norm(3e38).cpu())
    assert norm == math.inf and abs(factor / 0.1 - 1) < 1e-6
    g.zero_()
    assert opt.grad_norm(1.0).tolist() == [0.0, 1.0]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_not_finite(sc, bits, bad):
    torch, dev = torch_dev()
    sizes = [300, 5000]
    host, t, (params, grads) = make(sizes, 15)
    opt = sc.AdamW(params, grads, state_bits=bits)
    opt.step(1e-3)
    before = [x.clone() for x in (t["p"], *opt.moments())]
    grads[1][700] = bad
    clip = opt.grad_norm(1.0)
    assert math.isnan(float(clip[1]))
    opt.step(1e-3, clip=clip)                       # turned off as a whole
    for a, b in zip(before, (t["p"], *opt.moments())):
        assert torch.equal(a, b)
    opt.step(1e-3)                                  # without a clip it goes where it belongs
    m, v = opt.moments()
    at = 300 + 700
    own = torch.zeros(5300, dtype=torch.bool, device=dev)
    if bits == 8:
        own[300 + 512:300 + 768] = True             # the block's moments read as NaN
        assert bool(torch.isnan(m[own]).all()) and bool(torch.isnan(v[own]).all())
    else:
        own[at] = True
        assert not math.isfinite(float(m[at])) and not math.isfinite(float(v[at]))
    assert bool(torch.isfinite(m[~own]).all()) and bool(torch.isfinite(v[~own]).all())
    rest = torch.ones(5300, dtype=torch.bool, device=dev)
    rest[at] = False
    assert bool(torch.isfinite(t["p"][rest]).all())


def test_zero_gradients_and_extremes(sc):
    """Zeros stay zero; the largest and the smallest values keep their codes."""
    torch, dev = torch_dev()
    n = 1024
    zero = torch.zeros(n, device=dev)
    for bits in (32, 8):
        p = torch.ones(n, device=dev)
        opt = sc.AdamW([p], [zero], weight_decay=0.0, state_bits=bits)
        opt.step(0.1)
        assert torch.equal(p, torch.ones_like(p)) and not any(bool(x.any()) for x in opt.moments())
    opt = sc.AdamW([p], [zero], state_bits=8)
    for value in (float(np.finfo(np.float32).max), 1e-38, 1e-42, 1.4e-45, 1.0):
        m = torch.full((n,), value, device=dev) * torch.where(torch.arange(n, device=dev) % 2 == 0, 1.0, -1.0)
        m = torch.where(torch.arange(n, device=dev) % 3 == 0, 0.0, m)
        host = m.cpu().numpy()
        opt.load(9, m, m.abs())
        a, b = (x.cpu().numpy() for x in opt.moments())
        assert same_bits(a, ot.decode(*ot.encode(host, 9, signed=True), signed=True))
        assert same_bits(b, ot.decode(*ot.encode(np.abs(host), 9, signed=False), signed=False))
        assert np.isfinite(a).all() and np.array_equal(b > 0, host != 0)
        opt.load(10, *opt.moments())                # values of codes are kept at any step
        again = [x.cpu().numpy() for x in opt.moments()]
        assert same_bits(a, again[0]) and same_bits(b, again[1])


def test_codes_load(sc):
    torch, dev = torch_dev()
    sizes = [300, 5000, 1]
    host, t, (params, grads) = make(sizes, 16)
    a = sc.AdamW(params, grads, state_bits=8)
    a.step(1e-3)
    b = sc.AdamW([p.clone() for p in params], grads, state_bits=8)
    b.load(a.t, a.m, a.v, tops=a.tops)
    a.step(1e-3)
    b.step(1e-3)
    assert torch.equal(a.m, b.m) and torch.equal(a.v, b.v) and torch.equal(a.tops, b.tops)
    assert all(torch.equal(x, y) for x, y in zip(a.params, b.params))


def test_set_grads_and_other_streams(sc):
    torch, dev = torch_dev()
    sizes = [40_000, 33]
    host, t, (params, grads) = make(sizes, 17)
    mine = [p.clone() for p in params]
    a = sc.AdamW(params, grads)
    side = torch.cuda.Stream()
    b = sc.AdamW(mine, [torch.zeros_like(g) for g in grads])
    other = [g.clone() for g in grads]
    b.set_grads(other)
    side.wait_stream(torch.cuda.current_stream())
    a.step(1e-3, clip=a.grad_norm(1e-2))
    b.step(1e-3, clip=b.grad_norm(1e-2, stream=side), stream=side)
    with torch.cuda.stream(side):
        m, v = b.moments()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(params, mine))
    assert torch.equal(a.m, m) and torch.equal(a.v, v)


@pytest.mark.parametrize("bits", [32, 8])
def test_graph(sc, bits):
    """A captured norm and step, replayed between eager work, against eager calls."""
    torch, dev = torch_dev()
    sizes = [50_000, 777]
    host, t, (params, grads) = make(sizes, 18)
    mine = [p.clone() for p in params]
    a = sc.AdamW(params, grads, state_bits=bits)
    b = sc.AdamW(mine, grads, state_bits=bits)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.step(1e-3, clip=b.grad_norm(0.05))
    for i in range(4):
        for g in grads:
            g.mul_(1.5)
        a.t = 0                                       # the captured step's number is the captured one
        a.step(1e-3, clip=a.grad_norm(0.05))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(params, mine)), f"replay {i}"
        for x, y in zip(a.moments(), b.moments()):
            assert torch.equal(x, y), f"replay {i}"


def test_after_the_aggregation(sc):
    """The aggregate of a fused step as the gradients, layer by layer."""
    torch, dev = torch_dev()
    rng = np.random.default_rng(3)
    K, sizes = 4, [3000, 17, 9000, 250]
    n = sum(sizes)
    G = torch.from_numpy(rng.normal(0, 1e-2, (K, n)).astype(np.float32)).to(dev)
    step = sc.FusedStep(G, [0.1] * K)
    w, _ = sc.stream_weights([4, 8, 2, 16], base_batch=30)
    p = torch.zeros(n, device=dev)
    opt = sc.AdamW(list(torch.split(p, sizes)), list(torch.split(step.dense, sizes)), weight_decay=0.0)
    out = step.run(w)
    opt.step(0.5, clip=opt.grad_norm(math.inf))
    torch.cuda.synchronize()
    dense, got = out.dense.cpu().numpy(), p.cpu().numpy()
    assert (dense == 0).sum() > n // 2
    assert np.array_equal(got == 0, dense == 0)
    big = np.abs(dense) > 1e-4                      # the first step moves by lr towards -sign(g)
    assert np.allclose(got[big], -0.5 * np.sign(dense[big]), rtol=1e-3)


@pytest.mark.parametrize("bits", [32, 8])
def test_more_than_2_to_32_bytes(sc, bits):
    """A tensor whose offsets pass 32 bits: its end is updated as a short tensor is."""
    torch, dev = torch_dev()
    n, tail = 2**30 + 2**20 + 3, 2**20 + 3                    # the tail starts a block of 8-bit moments
    log(f"adamw n={n} bits={bits}")
    p, g = torch.zeros(n, device=dev), torch.zeros(n, device=dev)
    rng = np.random.default_rng(19)
    g[-tail:] = torch.from_numpy(rng.normal(0, 1e-3, tail).astype(np.float32)).to(dev)
    q, h = p[-tail:].clone(), g[-tail:].clone()
    a = sc.AdamW([p], [g], state_bits=bits)
    b = sc.AdamW([q], [h], state_bits=bits)
    x, y = a.grad_norm(1e-2).tolist(), b.grad_norm(1e-2).tolist()
    assert abs(x[0] / y[0] - 1) <= 4 * U
    a.step(1e-3)
    b.step(1e-3)
    assert torch.equal(p[-tail:], q) and not bool(p[:-tail].any())
    m, v = a.moments()
    if bits == 32:                                            # the dither of 8 bits goes by the element's number
        assert torch.equal(m[-tail:], b.m) and torch.equal(v[-tail:], b.v)
    else:
        m1, v1 = b.moments()
        assert float((m[-tail:] / m1 - 1).abs().nan_to_num().max()) <= 0.3 and bool((v[-tail:] > 0).eq(v1 > 0).all())
    assert not bool(m[:-tail].any()) and not bool(v[:-tail].any())
