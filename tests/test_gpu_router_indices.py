"""The router's backward pass on choices that no forward pass gives: an index
outside the experts is a missing choice, and nothing else is written."""
import numpy as np
import pytest

from _gpu_common import log, torch_dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("shape", [(3, 2), (8, 2), (30, 4), (64, 8), (100, 8), (256, 8), (500, 3), (1000, 16)], ids=str)
def test_indices_outside_the_experts(shape, renormalise):
    import paper_2301_08897_amd as sc
    torch, dev = torch_dev()
    E, k = shape
    T = 333
    log(f"router indices {shape} renormalise={renormalise}")
    rng = np.random.default_rng(E)
    x = torch.from_numpy(rng.normal(0, 1.5, (T, E)).astype(np.float32)).to(dev)
    dg, dl = torch.from_numpy(rng.normal(0, 1, (T, k)).astype(np.float32)).to(dev), torch.tensor([0.7, -0.3], device=dev)
    r = sc.Router(T, E, k, renormalise=renormalise)
    f = r.forward(x)
    where = torch.from_numpy(rng.random((T, k)) < 0.3).to(dev)
    f.idx.masked_fill_(where, -1)
    want = r.backward(x, f, dg, dl)
    assert bool((want[f.idx[:, 0] < 0] == 0).all()) and bool(want.any())
    for bad in (E, E + 1, 1024, 2**20, 2**31 - 1, -2, -2**31):
        f.idx.masked_fill_(where, bad)
        assert torch.equal(r.backward(x, f, dg, dl), want), bad
