#!/usr/bin/env python3
"""Trains a small mixture-of-experts layer on K simulated devices whose streams
run at different rates, with the framework's calls in the order in which a
training program makes them:

  stream buffers -> batch sizes and Eqn 4a weights
  Router.forward / backward: choices, gates, balance and z loss over all devices
  FusedStep: every device's Top-k, weighted aggregation (Eqn 4b)
  AdamW: global norm, clip, step (moments in 32 or 8 bits)

The experts' products and their gradients are plain torch operations. Data and
weights are random: token x of cluster c has the target T_c x.

    python examples/moe_router.py [--steps 60] [--state-bits 8]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2301_08897_amd as sc  # noqa: E402

DIM, EXPERTS, CHOICES, DEVICES = 32, 8, 2, 4


def train(steps: int = 60, state_bits: int = 32, ratio: float = 0.25, lr: float = 3e-3, seed: int = 0, log=None):
    """Runs ``steps`` steps; returns per step (task loss, balance loss, z loss, norm)."""
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev).manual_seed(seed)
    draw = lambda *shape: torch.empty(*shape, device=dev).normal_(generator=gen)  # noqa: E731
    centres, targets = draw(EXPERTS, DIM) * 2.0, draw(EXPERTS, DIM, DIM) / DIM**0.5

    # one flat parameter vector, as the aggregation has it; the layer's tensors are parts of it
    shapes = [(EXPERTS, DIM)] + [(DIM, DIM)] * EXPERTS
    sizes = [a * b for a, b in shapes]
    n = sum(sizes)
    flat = draw(n) * 0.1
    parts = [p.view(s) for p, s in zip(torch.split(flat, sizes), shapes)]
    grads = torch.zeros(DEVICES, n, device=dev)
    device_parts = [[g.view(s) for g, s in zip(torch.split(grads[d], sizes), shapes)] for d in range(DEVICES)]

    streams = sc.StreamBuffers([16, 48, 160, 512], b_min=16, b_max=256, policy="truncation", base_batch=128 * DEVICES)
    router = sc.Router(256 * DEVICES, EXPERTS, CHOICES, devices=DEVICES, renormalise=True)
    fused = sc.FusedStep(grads, [ratio] * DEVICES)
    opt = sc.AdamW([p.reshape(-1) for p in parts], list(torch.split(fused.dense, sizes)), state_bits=state_bits,
                   weight_decay=[0.0] + [0.01] * EXPERTS)
    d_loss = torch.tensor([0.02, 1e-3], device=dev)      # coefficients of the balance and the z loss
    ones = np.ones(DEVICES, dtype=np.float32)
    history = []
    for step in range(steps):
        batch, weights, gamma = streams.iteration(1_000_000)
        off = np.concatenate([[0], np.cumsum(batch)]).astype(np.int64)
        T = int(off[-1])
        cluster = torch.randint(EXPERTS, (T,), generator=gen, device=dev)
        x = centres[cluster] + draw(T, DIM) * 0.5
        want = torch.empty(T, DIM, device=dev)
        for c in range(EXPERTS):
            want[cluster == c] = x[cluster == c] @ targets[c].T

        logits = x @ parts[0].T
        f = router.forward(logits, tok_off=off, weights=weights)
        y, outs, rows = torch.zeros_like(want), [], []
        for e in range(EXPERTS):
            t, c = (f.idx == e).nonzero(as_tuple=True)   # the tokens that chose e, and where
            rows.append((t, c))
            outs.append(x[t] @ parts[1 + e].T)
            y.index_add_(0, t, outs[e] * f.gate[t, c, None])
        error = y - want

        # every device's gradient of its own mean loss; r_d weights them in the aggregation
        per_row = torch.repeat_interleave(1.0 / torch.tensor(batch.astype(np.float64)), torch.tensor(batch.astype(np.int64)))
        dy = 2.0 * error / DIM * per_row.to(dev, torch.float32)[:, None]
        d_gate = torch.zeros(T, CHOICES, device=dev)
        grads.zero_()
        for e in range(EXPERTS):
            t, c = rows[e]
            d_gate[t, c] = (outs[e] * dy[t]).sum(dim=1)
            for d in range(DEVICES):
                mine = (t >= int(off[d])) & (t < int(off[d + 1]))
                device_parts[d][1 + e] += (dy[t[mine]] * f.gate[t[mine], c[mine], None]).T @ x[t[mine]]
        d_logits = router.backward(logits, f, d_gate, d_loss, weights=ones)
        for d in range(DEVICES):
            s = slice(int(off[d]), int(off[d + 1]))
            device_parts[d][0] += d_logits[s].T @ x[s]

        fused.run(weights)
        clip = opt.grad_norm(1.0)
        opt.step(lr * gamma, clip=clip)
        task = sum(float(weights[d]) * float((error[int(off[d]):int(off[d + 1])] ** 2).mean()) for d in range(DEVICES))
        history.append((task, float(f.loss[0]), float(f.loss[1]), float(clip[0])))
        if log and (step % 10 == 0 or step == steps - 1):
            log(f"step {step:3d}: tokens {T}, loss {task:.4f}, balance {history[-1][1]:.4f}, z {history[-1][2]:.3f}, "
                f"norm {history[-1][3]:.4f}, per device and expert {f.counts.tolist()}")
    return history


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--state-bits", type=int, default=32, choices=(8, 32))
    ap.add_argument("--ratio", type=float, default=0.25, help="Top-k compression ratio")
    a = ap.parse_args()
    train(a.steps, a.state_bits, a.ratio, log=lambda m: print(m, flush=True))


if __name__ == "__main__":
    main()
