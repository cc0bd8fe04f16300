"""The host side of the training objects (no GPU needed): what they keep from call
to call, and in what order they let the GPU work."""
import numpy as np
import pytest
import torch

import _fake_gpu as fake


@pytest.fixture(scope="module")
def sc():
    import paper_2301_08897_amd as sc
    return sc


@pytest.fixture
def lib(sc, monkeypatch):
    return fake.Library(sc, monkeypatch)


def logits(T=12, E=8, gpu=0, dtype=torch.float32):
    return fake.on(gpu, torch.zeros(T, E, dtype=dtype))


def bounds_of(call, K):
    """(tok_off, weights, tokens) that a router call was given."""
    shape = call[3][0]
    return [shape.tok_off[d] for d in range(K + 1)], [shape.weights[d] for d in range(K)], shape.tokens


@pytest.mark.parametrize("T", [12, 7])
def test_refused_forward_leaves_the_last_pass(sc, lib, T):
    """After a forward pass that is refused, by the library or before it, the backward
    pass is still that of the pass before."""
    r = sc.Router(12, 8, 2, devices=2)
    x = logits()
    f = r.forward(x, tok_off=[0, 4, 12], weights=[0.25, 0.75])
    lib.status = 1
    with pytest.raises(sc.ScadlesError):
        r.forward(logits(T, dtype=torch.bfloat16), tok_off=[0, 5, T], weights=[0.5, 0.5])
    lib.status = 0
    with pytest.raises(ValueError):
        r.forward(logits(T), tok_off=[0, 6, T], weights=[0.5, 0.25, 0.25])
    r.backward(x, f)
    assert bounds_of(lib.calls()[-1], 2) == ([0, 4, 12], [0.25, 0.75], 12)
    r.backward(x, f, weights=[1.0, 1.0])
    assert bounds_of(lib.calls()[-1], 2) == ([0, 4, 12], [1.0, 1.0], 12)
    r.backward(x, f)
    assert bounds_of(lib.calls()[-1], 2) == ([0, 4, 12], [0.25, 0.75], 12)
    g = r.forward(x, tok_off=[0, 3, 12], weights=[0.5, 0.5])
    r.backward(x, g, weights=[1.0, 2.0])
    assert bounds_of(lib.calls()[-1], 2) == ([0, 3, 12], [1.0, 2.0], 12)
