#!/usr/bin/env python3
"""Trains a small mixture-of-experts language model on K simulated devices whose
streams run at different rates, with the framework's operators from tokens to
the update:

  stream buffers -> batch sizes and Eqn 4a weights
  Embedding -> LayerNorm -> Router -> ExpertOrder -> the experts -> LayerNorm
  -> LinearCrossEntropy on the embedding's own table, and back: every device's
  gradient of its own loss, in its flat gradient
  FusedStep: every device's Top-k, weighted aggregation (Eqn 4b)
  AdamW: global norm, clip, step

The experts' products are plain torch operations, an expert's rows at a time.
Tokens are random; the next one is a fixed function of a token, but for noise.

    python examples/moe_language.py [--steps 60]
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


class Model:
    """Parameters in one flat vector, as the aggregation has them, and a flat gradient
    for each device."""

    def __init__(self, vocab=500, dim=48, experts=6, choices=2, devices=4, max_tokens=4096, seed=0):
        self.experts, self.choices, self.devices = experts, choices, devices
        self.names = ["table", "norm1.weight", "norm1.bias", "router"] + [f"expert{e}" for e in range(experts)] + ["norm2.weight", "norm2.bias"]
        shapes = [(vocab, dim), (dim,), (dim,), (experts, dim)] + [(dim, dim)] * experts + [(dim,), (dim,)]
        self.sizes = [int(np.prod(s)) for s in shapes]
        dev = torch.device("cuda:0")
        gen = torch.Generator(device=dev).manual_seed(seed)
        self.flat = torch.empty(sum(self.sizes), device=dev).normal_(generator=gen).mul_(dim**-0.5)
        self.grads = torch.zeros(devices, sum(self.sizes), device=dev)
        part = lambda flat: {n: p.view(s) for n, p, s in zip(self.names, torch.split(flat, self.sizes), shapes)}  # noqa: E731
        self.p, self.g = part(self.flat), [part(g) for g in self.grads]
        for n in ("norm1", "norm2"):
            self.p[n + ".weight"].fill_(1.0)
            self.p[n + ".bias"].zero_()
        self.embedding = sc.Embedding(vocab, dim, scale=dim**0.5, devices=devices)
        self.norm = sc.LayerNorm(dim, devices=devices)
        self.router = sc.Router(max_tokens, experts, choices, devices=devices, renormalise=True)
        self.order = sc.ExpertOrder(experts, choices, devices=devices)
        self.loss = sc.LinearCrossEntropy(vocab, dim, devices=devices)

    def parts(self, name):
        """Every device's gradient of a parameter."""
        return [g[name] for g in self.g]

    def step(self, tokens, target, off, weights, d_router=None):
        """One forward and backward pass; fills the devices' gradients and returns the
        outputs of the loss and of the router. ``d_router``: the coefficients of the
        balance and the z loss, or None."""
        p, K = self.p, self.devices
        h0 = self.embedding.forward(tokens, p["table"])
        n1 = self.norm.forward(h0, p["norm1.weight"], p["norm1.bias"])
        logits = n1.y @ p["router"].T
        f = self.router.forward(logits, tok_off=off, weights=weights)
        order = self.order.sort(f.idx, tok_off=off)
        first = order.bounds.tolist()                     # an expert's rows, device by device
        rows = self.order.dispatch(n1.y, order)
        y = torch.zeros_like(rows)
        span = lambda e: slice(first[e * K], first[(e + 1) * K])  # noqa: E731
        for e in range(self.experts):
            y[span(e)] = rows[span(e)] @ p[f"expert{e}"].T
        h1 = h0 + self.order.combine(y, f.gate, order)
        n2 = self.norm.forward(h1, p["norm2.weight"], p["norm2.bias"])
        out = self.loss.forward(n2.y, p["table"], target, tok_off=off, weights=weights)

        d_n2 = self.loss.backward(n2.y, p["table"], target, out, self.parts("table"), tok_off=off)
        d_h1 = self.norm.backward(h1, p["norm2.weight"], n2, d_n2, self.parts("norm2.weight"), self.parts("norm2.bias"), tok_off=off)
        d_y, d_gate = self.order.combine_backward(d_h1, y, f.gate, order, d_rows=torch.zeros_like(y))
        d_rows = torch.zeros_like(rows)
        for e in range(self.experts):
            d_rows[span(e)] = d_y[span(e)] @ p[f"expert{e}"]
            for d in range(K):
                s = slice(first[e * K + d], first[e * K + d + 1])
                self.g[d][f"expert{e}"].copy_(d_y[s].T @ rows[s])
        d_logits = self.router.backward(logits, f, d_gate, d_router, weights=np.ones(K, dtype=np.float32))
        for d in range(K):
            s = slice(int(off[d]), int(off[d + 1]))
            self.g[d]["router"].copy_(d_logits[s].T @ n1.y[s])
        d_n1 = self.order.dispatch_backward(d_rows, order) + d_logits @ p["router"]
        d_h0 = d_h1 + self.norm.backward(h0, p["norm1.weight"], n1, d_n1, self.parts("norm1.weight"), self.parts("norm1.bias"), tok_off=off)
        self.embedding.backward(tokens, d_h0, self.parts("table"), tok_off=off, accumulate=True)    # the table is the logits' too
        return out, f


def train(steps: int = 60, ratio: float = 0.25, lr: float = 3e-3, seed: int = 0, log=None):
    """Runs ``steps`` steps; returns per step (loss, balance loss, norm)."""
    model = Model(seed=seed)
    dev, K, vocab = model.flat.device, model.devices, model.embedding.vocab
    gen = torch.Generator(device=dev).manual_seed(seed + 1)
    follows = torch.randperm(vocab, generator=gen, device=dev)
    streams = sc.StreamBuffers([16, 48, 160, 512], b_min=16, b_max=256, policy="truncation", base_batch=128 * K)
    fused = sc.FusedStep(model.grads, [ratio] * K)
    opt = sc.AdamW(list(torch.split(model.flat, model.sizes)), list(torch.split(fused.dense, model.sizes)),
                   weight_decay=[0.0 if "norm" in n else 0.01 for n in model.names])
    d_router = torch.tensor([0.02, 1e-3], device=dev)
    history = []
    for step in range(steps):
        batch, weights, gamma = streams.iteration(1_000_000)
        off = np.concatenate([[0], np.cumsum(batch)]).astype(np.int64)
        tokens = torch.randint(vocab, (int(off[-1]),), generator=gen, device=dev)
        noise = torch.rand(len(tokens), generator=gen, device=dev) < 0.05
        target = torch.where(noise, torch.randint(vocab, (len(tokens),), generator=gen, device=dev), follows[tokens])
        out, f = model.step(tokens, target, off, weights, d_router)
        fused.run(weights)
        clip = opt.grad_norm(1.0)
        opt.step(lr * gamma, clip=clip)
        history.append((float(out.loss), float(f.loss[0]), float(clip[0])))
        if log and (step % 10 == 0 or step == steps - 1):
            log(f"step {step:3d}: tokens {len(tokens)}, loss {history[-1][0]:.4f}, balance {history[-1][1]:.4f}, norm {history[-1][2]:.4f}, "
                f"per device {[round(x, 3) for x in out.device_loss.tolist()]}")
    return history


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--ratio", type=float, default=0.25, help="Top-k compression ratio")
    a = ap.parse_args()
    train(a.steps, a.ratio, log=lambda m: print(m, flush=True))


if __name__ == "__main__":
    main()
