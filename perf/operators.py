"""The training operators around the aggregated gradient, as cases that can be
timed and compared: AdamW over many tensors at once (moments in 32 or 8 bits),
the gradients' global norm with the clip factor, and the mixture-of-experts
router (Top-k choice, gates, per-device expert counts, balance and z loss) with
its backward pass.

With ``own`` false every pass is computed with plain torch operations in 32
bits. Parameters, gradients and moments are flat buffers that the tensors are
consecutive pieces of, so most tensors start at odd addresses.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

# Parameter counts of the workloads' models; the small ones are a LeNet-sized
# model and one 128 x 128 x 3 x 3 layer.
LENET, CONV, RESNET18, RESNET50, RESNET152, VGG19 = 61_706, 147_456, 11_173_962, 25_557_032, 60_192_808, 143_667_240

B1, B2, EPS, DECAY, LR, MAX_NORM = 0.9, 0.999, 1e-8, 0.01, 1e-3, 1.0
BLOCK = 256                      # elements that share one offset of the 8-bit moments

ADAMW = {"call": "adamw", "n": LENET, "tensors": 10, "bits": 32, "grads": "f32", "copies": False, "clip": False}
ROUTE = {"call": "forward", "tokens": 64, "experts": 8, "k": 2, "devices": 1, "logits": "f32", "renormalise": False,
         "padding": False}


def listed():
    return [
        # A small model's update: one launch's latency, and the norm's before it.
        dict(ADAMW, name="adamw_lenet", clip=True),
        # ResNet-18 with moments in 8 bits, the ordinary memory-saving step.
        dict(ADAMW, name="adamw8_resnet18", n=RESNET18, tensors=62, bits=8),
        # Mixed precision: bf16 gradients, f32 parameters with a bf16 copy for
        # the next forward pass, clipped.
        dict(ADAMW, name="adamw_resnet50_bf16", n=RESNET50, tensors=161, grads="bf16", copies=True, clip=True),
        # The most tensors; 8-bit moments, f32 gradients as the aggregation
        # gives them.
        dict(ADAMW, name="adamw8_resnet152", n=RESNET152, tensors=467, bits=8),
        # The largest model: bandwidth.
        dict(ADAMW, name="adamw_vgg19", n=VGG19, tensors=38),
        # The norm on its own, for logging or a skipped-step check: one layer,
        # and a whole model.
        dict(ADAMW, name="norm_conv", call="norm", n=CONV, tensors=1),
        dict(ADAMW, name="norm_resnet152", call="norm", n=RESNET152, tensors=467),
        # One short batch on one device.
        dict(ROUTE, name="route_64x8"),
        # Eight devices of uneven batches, evaluation (no gradient).
        dict(ROUTE, name="route_16k_64", tokens=16384, experts=64, devices=8, logits="bf16"),
        # Many experts with many choices, every device of the largest workload.
        dict(ROUTE, name="route_128k_256", tokens=131072, experts=256, k=8, devices=32),
        # Training, an odd number of experts and tokens, padded batches.
        dict(ROUTE, name="route_train_16k_60", call="train", tokens=16381, experts=60, k=4, devices=8, logits="bf16",
             renormalise=True, padding=True),
        # Training at the largest size.
        dict(ROUTE, name="route_train_128k_256", call="train", tokens=131072, experts=256, k=8, devices=32),
    ]


def draw(rng):
    call = rng.choice(["adamw", "adamw", "adamw", "norm", "forward", "train", "train"])
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    if call in ("adamw", "norm"):
        n = log(LENET, VGG19)
        c = dict(ADAMW, call=call, n=n, tensors=max(1, min(log(1, 467), n // 256)), grads=rng.choice(["f32", "f32", "bf16"]))
        if call == "adamw":
            c.update(bits=rng.choice([32, 8]), copies=rng.random() < 0.3)
            c["clip"] = c["bits"] == 32 and rng.random() < 0.5
        return c
    experts = log(4, 256)
    if rng.random() < 0.5:
        experts = min(256, 1 << round(math.log2(experts)))
    return dict(ROUTE, call=call, tokens=log(32, 131072), experts=experts, k=rng.randint(1, min(8, experts)),
                devices=rng.choice([1, 2, 5, 8, 16, 32]), logits=rng.choice(["f32", "bf16"]),
                renormalise=rng.random() < 0.5, padding=rng.random() < 0.5)


# ---- inputs -----------------------------------------------------------------------------------

def tensor_sizes(case):
    """Sizes of the model's tensors: as many short ones (biases, norms) as long ones."""
    n, L = case["n"], case["tensors"]
    r = np.random.RandomState(2000 + L)
    w = np.exp(np.where(np.arange(L) % 2 == 0, r.uniform(math.log(6e3), math.log(2.4e6), L), r.uniform(math.log(64.0), math.log(2048.0), L)))
    b = np.round(np.cumsum(w) / w.sum() * (n - L)).astype(np.int64) + np.arange(1, L + 1)
    b[-1] = n
    return np.diff(np.concatenate([[0], b]))


def generator(seed, salt):
    return torch.Generator(device="cuda").manual_seed(seed * 7919 + salt)


def normal(seed, salt, *shape):
    return torch.empty(*shape, dtype=torch.float32, device="cuda").normal_(generator=generator(seed, salt))


def uniform(seed, salt, *shape):
    return torch.empty(*shape, dtype=torch.float32, device="cuda").uniform_(generator=generator(seed, salt))


def blocks_of(sizes):
    """Where the elements of the 8-bit blocks lie: (element's place in the blocks, per
    block place the element's number in its tensor, whether there is one, its flat place)."""
    size = torch.tensor(sizes, dtype=torch.int64, device="cuda")
    n, blocks = int(sizes.sum()), (size + BLOCK - 1) // BLOCK
    start, first = torch.cumsum(size, 0) - size, (torch.cumsum(blocks, 0) - blocks) * BLOCK
    shift = torch.repeat_interleave(first - start, size)
    place = torch.arange(n, device="cuda") + shift
    pos = torch.arange(int(blocks.sum()) * BLOCK, device="cuda") - torch.repeat_interleave(first, blocks * BLOCK)
    flat = torch.zeros_like(pos)
    flat[place] = torch.arange(n, device="cuda")
    there = torch.zeros(pos.numel(), dtype=torch.bool, device="cuda")
    there[place] = True
    return place, pos, there, flat


def tensor_inputs(case, seed):
    sizes = tensor_sizes(case)
    n, cut = case["n"], [int(x) for x in sizes]
    s = {"case": case}
    r = np.random.RandomState(seed % (1 << 31))
    sigma = torch.tensor(10.0 ** r.uniform(-5.0, -2.0, len(cut)), dtype=torch.float32, device="cuda")
    scale = torch.repeat_interleave(sigma, torch.tensor(sizes, device="cuda"))
    grad = normal(seed, 11, n).mul_(scale)
    s["grad"] = grad.to(torch.bfloat16) if case["grads"] == "bf16" else grad
    s["param"] = normal(seed, 12, n).mul_(0.05)
    s["copy"] = torch.zeros(n, dtype=torch.bfloat16, device="cuda") if case["copies"] else None
    decay = [DECAY if x > 4096 else 0.0 for x in cut]            # none on biases and norms
    s["decay"] = torch.repeat_interleave(torch.tensor(decay, dtype=torch.float32, device="cuda"), torch.tensor(sizes, device="cuda"))
    s["t"] = 100                                                 # a run under way
    if case["call"] == "adamw":
        m = normal(seed, 13, n).mul_(0.3).mul_(scale)
        v = uniform(seed, 14, n).add_(0.5).mul_(scale).mul_(scale)
        if case["bits"] == 8:
            s["place"], s["pos"], s["there"], s["flat"] = blocks_of(sizes)
            s["m"], s["mtop"] = encode(spread(s, m), dither(s, 0x9E3779B9, 0xBB67AE85), 127, True)
            s["v"], s["vtop"] = encode(spread(s, v), dither(s, 0x6A09E667, 0x9E3779B9), 255, False)
        else:
            s["m"], s["v"] = m, v
    s["cut"], s["decays"] = cut, decay
    return s


def router_inputs(case, seed):
    T, E, K = case["tokens"], case["experts"], case["devices"]
    r = np.random.RandomState(seed % (1 << 31))
    share = 128.0 ** (np.arange(K) / max(K - 1, 1))              # streams from slow to fast
    bounds = np.round(np.cumsum(share) / share.sum() * T).astype(np.int64)
    bounds[-1] = T
    s = {"case": case, "bounds": [0] + [int(x) for x in bounds]}
    count = np.diff(s["bounds"])
    s["weights"] = (count / max(1, count.sum())).astype(np.float32)
    x = normal(seed, 21, T, E).mul_(1.5) + torch.tensor(r.normal(0, 0.7, E), dtype=torch.float32, device="cuda")
    s["x"] = x.to(torch.bfloat16) if case["logits"] == "bf16" else x
    s["device"] = torch.repeat_interleave(torch.arange(K, device="cuda"), torch.tensor(count, device="cuda"))
    s["valid"] = uniform(seed, 22, T) < 0.9 if case["padding"] else None
    s["w"] = torch.tensor(s["weights"], device="cuda")
    if case["call"] == "train":
        s["dgate"] = normal(seed, 23, T, case["k"]).mul_(1e-3)
        s["dloss"] = torch.tensor([0.01, 0.001], device="cuda")  # the losses' coefficients
    return s


def inputs(case, seed):
    return (tensor_inputs if case["call"] in ("adamw", "norm") else router_inputs)(case, seed)


def handle(s):
    """What a program keeps from step to step: the optimizer over its tensors, or the router."""
    import paper_2301_08897_amd as sc
    case = s["case"]
    if case["call"] in ("forward", "train"):
        return sc.Router(case["tokens"], case["experts"], case["k"], devices=case["devices"], renormalise=case["renormalise"])
    pieces = lambda x: list(torch.split(x, s["cut"]))  # noqa: E731
    opt = sc.AdamW(pieces(s["param"]), pieces(s["grad"]), betas=(B1, B2), eps=EPS, weight_decay=s["decays"],
                   state_bits=case["bits"], copies=None if s["copy"] is None else pieces(s["copy"]))
    if case["call"] == "adamw":
        opt.load(s["t"], s["m"], s["v"], tops=s["mtop"] | s["vtop"] << 16 if case["bits"] == 8 else None)
    return opt


def prepare(case, seed):
    s = inputs(case, seed)
    if own:
        s["handle"] = handle(s)
    return s


# ---- plain forms --------------------------------------------------------------------------------

def spread(s, x):
    """A flat vector in the places of the 8-bit blocks, zero where there is no element."""
    return torch.where(s["there"], x[s["flat"]], torch.zeros((), device="cuda"))


def dither(s, a, b):
    return ((s["pos"] * a + s["t"] * b & 0xFFFFFFFF) >> 12).to(torch.int32)


def encode(x, u, span, signed):
    """Codes of the blocks of ``x`` and every block's largest step: a step is the exponent
    and the first three mantissa bits, rounded up where the dither carries."""
    step = ((x.view(torch.int32) & 0x7FFFFFFF) + u >> 20).view(-1, BLOCK)
    top = step.amax(dim=1)
    base = (top.clamp(min=span) - span)[:, None]
    code = (step - base).clamp(min=0, max=span)
    if signed:
        code = code + torch.where((x.view(-1, BLOCK) < 0) & (code > 0), 128, 0)
    else:
        code = torch.where(x.view(-1, BLOCK) > 0, code.clamp(min=1), code)
    return code.to(torch.uint8), top


def decode(code, top, span):
    c = code.to(torch.int32)
    size = c & span
    step = size + (top.clamp(min=span) - span)[:, None]
    x = torch.where(size > 0, step << 20, torch.zeros_like(step)).view(torch.float32)
    return (torch.where(c > span, -x, x)).flatten()


def plain_norm(s):
    g = s["grad"].float()
    norm = (g * g).sum().sqrt()
    return torch.stack([norm, (MAX_NORM / norm).clamp(max=1.0)])


def plain_adamw(s):
    case = s["case"]
    s["t"] += 1
    t, out = s["t"], {}
    g = s["grad"].float()
    if case["clip"]:
        out["clip"] = plain_norm(s)
        g = g * out["clip"][1]
    if case["bits"] == 8:
        g8 = spread(s, g)
        m = decode(s["m"], s["mtop"], 127) * B1 + g8 * (1 - B1)
        v = decode(s["v"], s["vtop"], 255) * B2 + g8 * g8 * (1 - B2)
        s["m"], s["mtop"] = encode(m, dither(s, 0x9E3779B9, 0xBB67AE85), 127, True)
        s["v"], s["vtop"] = encode(v, dither(s, 0x6A09E667, 0x9E3779B9), 255, False)
        out["m"], out["v"] = decode(s["m"], s["mtop"], 127)[s["place"]], decode(s["v"], s["vtop"], 255)[s["place"]]
        m, v = m[s["place"]], v[s["place"]]
    else:
        out["m"] = m = s["m"].mul_(B1).add_(g * (1 - B1))
        out["v"] = v = s["v"].mul_(B2).add_(g * g * (1 - B2))
    d = v.sqrt() * (1 / math.sqrt(1 - B2**t)) + EPS
    out["param"] = s["param"].mul_(1 - s["decay"] * LR).sub_(m / d * (LR / (1 - B1**t)))
    if s["copy"] is not None:
        out["copy"] = s["copy"].copy_(s["param"])
    return out


def plain_route(s):
    case, x = s["case"], s["x"].float()
    T, E, K, k = case["tokens"], case["experts"], case["devices"], case["k"]
    valid = s["valid"] if s["valid"] is not None else torch.ones(T, dtype=torch.bool, device="cuda")
    e = torch.exp(x - x.amax(dim=1, keepdim=True))
    total = e.sum(dim=1, keepdim=True)
    p = e / total * valid[:, None]
    lse = (x.amax(dim=1) + total[:, 0].log()) * valid
    idx = torch.sort(s["x"], dim=1, descending=True, stable=True).indices[:, :k]       # ties: the lower index first
    gate = p.gather(1, idx)
    if case["renormalise"]:
        gate = torch.where(valid[:, None], gate / gate.sum(dim=1, keepdim=True), 0.0)
    one = valid.to(torch.int64)
    cell = s["device"][:, None] * E + idx
    counts = torch.zeros(K * E, dtype=torch.int64, device="cuda").scatter_add_(0, cell.flatten(), one.repeat_interleave(k)).view(K, E)
    rows = torch.zeros(K, dtype=torch.int64, device="cuda").scatter_add_(0, s["device"], one)
    share = s["w"] / rows.clamp(min=1)
    load = (counts * share[:, None]).sum(dim=0) / k
    each = share[s["device"]]
    prob = (p * each[:, None]).sum(dim=0)
    loss = torch.stack([E * (load * prob).sum(), (lse * lse * each).sum()])
    out = {"idx": torch.where(valid[:, None], idx, -1).to(torch.int32), "gate": gate, "lse": lse,
           "counts": counts.to(torch.int32), "load": load, "loss": loss}
    if case["call"] == "train":
        a, b = s["dloss"][0], s["dloss"][1]
        mean = (p * load).sum(dim=1, keepdim=True)
        dx = each[:, None] * p * (a * E * (load - mean) + 2 * b * lse[:, None])
        h = gate * s["dgate"]
        part = h.sum(dim=1, keepdim=True)
        dx = dx.scatter_add(1, idx, h - gate * part) if case["renormalise"] else (dx - p * part).scatter_add(1, idx, h)
        out["dlogits"] = (dx * valid[:, None]).to(s["x"].dtype)
    return out


# ---- one pass -----------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if not own:
        return {"adamw": plain_adamw, "norm": plain_norm}.get(case["call"], plain_route)(s)
    h = s["handle"]
    if case["call"] == "norm":
        return h.grad_norm(MAX_NORM)
    if case["call"] == "adamw":
        out = {"param": s["param"]}
        if case["clip"]:
            out["clip"] = h.grad_norm(MAX_NORM)
        h.step(LR, clip=out.get("clip"))
        out["m"], out["v"] = h.moments()
        if s["copy"] is not None:
            out["copy"] = s["copy"]
        return out
    f = h.forward(s["x"], tok_off=s["bounds"], weights=s["weights"], valid=s["valid"])
    out = {"idx": f.idx, "gate": f.gate, "lse": f.lse, "counts": f.counts, "load": f.load, "loss": f.loss}
    if case["call"] == "train":
        out["dlogits"] = h.backward(s["x"], f, s["dgate"], s["dloss"])
    return out


def work(case):
    if case["call"] in ("adamw", "norm"):
        n, g = case["n"], 2 if case["grads"] == "bf16" else 4
        if case["call"] == "norm":
            return {"bytes": n * g + 8, "flops": 2 * n}
        if case["bits"] == 8:            # moments read and written in 8 bits, and given as values
            return {"bytes": n * (8 + g + 4 + 8 + 2 * case["copies"]) + n // BLOCK * 8, "flops": 14 * n}
        return {"bytes": n * (24 + g + 2 * case["copies"]), "flops": (16 if case["clip"] else 14) * n}
    T, E, K, k = case["tokens"], case["experts"], case["devices"], case["k"]
    x = 2 if case["logits"] == "bf16" else 4
    byte, flop = T * (E * x + 8 * k + 4) + K * E * 4 + E * 4, T * E * 4
    if case["padding"]:
        byte += T
    if case["call"] == "train":
        byte, flop = byte + T * (E * x + 4 * k), flop + T * E * 8
    return {"bytes": byte, "flops": flop}


# ---- the definition in 64 bits ------------------------------------------------------------------

def exact(case, seed):
    s = inputs(case, seed)

    def steps(code, top, span):
        """The values that 8-bit codes stand for: step 8 (e + 127) + j is 2^e (1 + j/8)."""
        size = (code.to(torch.int64) % (span + 1)).flatten()
        step = size + (top.to(torch.int64) - span).clamp(min=0).repeat_interleave(BLOCK)
        x = torch.ldexp(1 + (step % 8).double() / 8, step // 8 - 127)
        return torch.where(size == 0, 0.0, torch.where(code.flatten() > span, -x, x))[s["place"]]

    def rounded(x, a, b, span, lowest):
        """What the 8-bit moments of ``x`` stand for, tensor by tensor: 2^e (1 + f) goes to
        step 8 (e + 127) + floor(8 f + u), u in [0, 1) from the element's number and the step."""
        out, at = torch.empty_like(x), 0
        for size in s["cut"]:
            y, i = x[at:at + size], torch.arange(size, device="cuda")
            u = ((i * a + (s["t"] + 1) * b) % 2**32 // 2**12).double() / 2**20
            e = torch.frexp(y.abs()).exponent.to(torch.int64) - 1
            step = torch.where(y == 0, 0, 8 * (e + 127) + torch.floor(8 * (torch.ldexp(y.abs(), -e) - 1) + u).to(torch.int64))
            top = torch.nn.functional.pad(step, (0, -size % BLOCK)).view(-1, BLOCK).amax(dim=1).repeat_interleave(BLOCK)[:size]
            low = top.clamp(min=span) - span
            step = torch.where(step > low, step, torch.where(y == 0, 0, (low + 1) * lowest))
            out[at:at + size] = torch.where(step > 0, torch.copysign(torch.ldexp(1 + (step % 8).double() / 8, step // 8 - 127), y), 0.0)
            at += size
        return out

    def tensors():
        g, p, out, t = s["grad"].double(), s["param"].double(), {}, s["t"] + 1
        norm = torch.linalg.vector_norm(g)
        clip = torch.stack([norm, torch.minimum(MAX_NORM / norm, torch.ones_like(norm))])
        if case["call"] == "norm":
            return clip
        if case["clip"]:
            out["clip"] = clip
            g *= clip[1]
        small = case["bits"] == 8
        m, v = (steps(s["m"], s["mtop"], 127), steps(s["v"], s["vtop"], 255)) if small else (s["m"].double(), s["v"].double())
        m, v = torch.lerp(g, m, B1), torch.lerp(g.square(), v, B2)
        out["m"] = rounded(m, 0x9E3779B9, 0xBB67AE85, 127, 0) if small else m
        out["v"] = rounded(v, 0x6A09E667, 0x9E3779B9, 255, 1) if small else v
        out["param"] = p - LR * (s["decay"].double() * p + (m / (1 - B1**t)) / ((v / (1 - B2**t)).sqrt() + EPS))
        if case["copies"]:
            out["copy"] = out["param"]
        return out

    def router():
        E, k, x = case["experts"], case["k"], s["x"].double()
        valid = torch.ones(len(x), dtype=torch.bool, device="cuda") if s["valid"] is None else s["valid"]
        lse, p = torch.logsumexp(x, dim=1), torch.softmax(x, dim=1)
        idx = torch.argsort(x, dim=1, descending=True, stable=True)[:, :k]
        chosen = torch.zeros_like(x).scatter_(1, idx, 1.0)
        gates = p * chosen
        if case["renormalise"]:
            gates = gates / gates.sum(dim=1, keepdim=True)
        load, prob, z = (torch.zeros(n, dtype=torch.float64, device="cuda") for n in (E, E, 1))
        counts, each = [], torch.zeros(len(x), 1, dtype=torch.float64, device="cuda")
        for d in range(case["devices"]):
            lo, hi = s["bounds"][d], s["bounds"][d + 1]
            on = valid[lo:hi]
            counts.append(chosen[lo:hi][on].sum(dim=0))
            rows = int(on.sum())
            if rows:
                w = float(s["weights"][d]) / rows
                each[lo:hi] = w
                load += w / k * counts[-1]
                prob += w * p[lo:hi][on].sum(dim=0)
                z += w * lse[lo:hi][on].square().sum()
        on = valid.double()[:, None]
        out = {"idx": torch.where(valid[:, None], idx, -1).to(torch.int32), "gate": gates.gather(1, idx) * on, "lse": lse * on[:, 0],
               "counts": torch.stack(counts).to(torch.int32), "load": load, "loss": torch.cat([E * torch.dot(load, prob)[None], z])}
        if case["call"] == "train":
            a, b = (float(y) for y in s["dloss"])
            up = torch.zeros_like(x).scatter_(1, idx, s["dgate"].double())
            soft = lambda q, h: q * (h - (q * h).sum(dim=1, keepdim=True))  # noqa: E731
            part = soft(gates if case["renormalise"] else p, up)
            out["dlogits"] = on * (each * (soft(p, a * E * load[None]) + 2 * b * lse[:, None] * p) + part)
        return out

    return tensors() if case["call"] in ("adamw", "norm") else router()
