"""The operators between tokens and logits in a run of them, as examples/moe_language.py
has it: it runs, and every device's gradient of every parameter is that of the same
model in 64 bits with torch's own operators and autograd."""
import os
import sys

import numpy as np
import pytest

from _gpu_common import torch_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    sys.path.insert(0, os.path.join(root, "examples"))
    import moe_language
    yield moe_language
    sys.path.remove(os.path.join(root, "examples"))


def test_the_example_runs(example):
    history = example.train(steps=3)
    assert len(history) == 3 and np.isfinite(np.array(history)).all()


def test_gradients_of_the_whole_model(example):
    torch, dev = torch_dev()
    F = torch.nn.functional
    K, off = 3, [0, 30, 30, 200]
    m = example.Model(vocab=97, dim=24, experts=5, choices=2, devices=K, max_tokens=256, seed=3)
    gen = torch.Generator(device=dev).manual_seed(9)
    tokens = torch.randint(97, (200,), generator=gen, device=dev)
    target = torch.randint(-5, 97, (200,), generator=gen, device=dev)      # some are not counted
    weights = np.array([0.2, 0.0, 0.8], dtype=np.float32)
    out, f = m.step(tokens, target, off, weights)
    p = {n: x.double().cpu().requires_grad_() for n, x in m.p.items()}
    tok, tgt, idx = tokens.cpu(), target.cpu(), f.idx.cpu().long()
    h0 = p["table"][tok] * m.embedding.scale
    n1 = F.layer_norm(h0, (24,), p["norm1.weight"], p["norm1.bias"], 1e-5)
    gate = torch.softmax((n1 @ p["router"].T).gather(1, idx), dim=1)       # renormalised over the chosen
    y = torch.stack([n1 @ p[f"expert{e}"].T for e in range(5)], dim=1)
    h1 = h0 + (y.gather(1, idx[:, :, None].expand(-1, -1, 24)) * gate[:, :, None]).sum(dim=1)
    n2 = F.layer_norm(h1, (24,), p["norm2.weight"], p["norm2.bias"], 1e-5)
    nll = F.cross_entropy(n2 @ p["table"].T, torch.where(tgt >= 0, tgt, -100), ignore_index=-100, reduction="none")
    U = 2.0**-24
    for d in range(K):
        s = slice(off[d], off[d + 1])
        count = int((tgt[s] >= 0).sum())
        mean = nll[s].sum() / max(count, 1)
        # a chain of about ten operators in float, each off by some tens of roundings of its terms' sizes, which add up
        # to few times the result over rows of 24 and batches of 200: 10 * 50 * 4 U
        near = 2000 * U
        assert abs(float(out.device_loss[d]) - float(mean.detach())) <= near * max(float(mean.detach()), 1.0)
        got = torch.autograd.grad(mean, list(p.values()), retain_graph=True, allow_unused=True) if count else [None] * len(p)
        for n, g in zip(p, got):
            have = m.g[d][n].double().cpu()
            want = torch.zeros_like(have) if g is None else g
            assert float((have - want).abs().max()) <= near * max(float(want.abs().max()), 1e-30), (d, n)
    assert abs(float(out.loss) - sum(float(w) * float(x) for w, x in zip(weights, out.device_loss))) <= 8 * U * float(out.loss)
