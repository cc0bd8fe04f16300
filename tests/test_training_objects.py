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


def test_backward_of_an_overwritten_pass_is_refused(sc, lib):
    r = sc.Router(12, 8, 2, devices=2)
    a, b = logits(), logits()
    off, w = [0, 4, 12], [0.25, 0.75]
    f = r.forward(a, tok_off=off, weights=w)
    r.backward(a, f)
    g = r.forward(b, tok_off=off, weights=w)
    with pytest.raises(ValueError):
        r.backward(a, f)                        # f's memory holds g's choices
    r.backward(b, g)
    r.backward(logits(), g)                     # logits computed again
    old = g
    for change in (dict(tok_off=[0, 5, 12]), dict(weights=[0.5, 0.5]), dict(valid=fake.on(0, torch.ones(12, dtype=torch.bool)))):
        g = r.forward(b, **{**dict(tok_off=off, weights=w), **change})
        with pytest.raises(ValueError):
            r.backward(b, old)
        r.backward(b, g)
        old = g
    mask = fake.on(0, torch.ones(12, dtype=torch.bool))
    g = r.forward(b, tok_off=off, weights=w, valid=mask)
    mask[3] = False
    for valid in (mask, mask.clone()):
        h = r.forward(b, tok_off=off, weights=w, valid=valid)
        with pytest.raises(ValueError):
            r.backward(b, g)
        g = h
    h = r.forward(b, tok_off=off, weights=w)
    b += 1.0
    r.forward(b, tok_off=off, weights=w)
    with pytest.raises(ValueError):
        r.backward(b, h)
    with pytest.raises(ValueError):
        sc.Router(12, 8, 2, devices=2).backward(b, h)


def test_a_repeated_pass_is_the_same_pass(sc, lib):
    """The same logits, bounds, weights and mask give the same results, so that the
    first call's outputs are still right."""
    r = sc.Router(12, 8, 2, devices=2)
    x, mask = logits(), fake.on(0, torch.ones(12, dtype=torch.bool))
    for valid in (None, mask):
        f = r.forward(x, tok_off=[0, 4, 12], valid=valid)
        r.forward(x, tok_off=np.array([0, 4, 12]), weights=[4 / 12, 8 / 12], valid=valid)
        r.backward(x, f)
    with torch.inference_mode():                # tensors without a version
        y = logits()
        f = r.forward(y, tok_off=[0, 4, 12])
        r.forward(y, tok_off=[0, 4, 12])
        r.backward(y, f)


def in_order(log, names):
    """Whether every library call runs after all before it: on their streams, or
    behind events recorded on those after them and waited for."""
    before, events, made = {}, {}, set()             # what is ordered before a stream's next work; an event's
    for i, x in enumerate(log):
        mine = before.setdefault(x[1], set())
        if x[0] == "record":
            events[x[1], i] = set(mine)
        elif x[0] == "wait":
            mine |= events[x[2]]
        elif x[0] in names:
            if mine != made:
                return False
            made.add(i)
            mine.add(i)
    return True


def tensors(*sizes, gpu=0, dtype=torch.float32):
    return [fake.on(gpu, torch.zeros(n, dtype=dtype)) for n in sizes]


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_calls_on_several_streams_run_in_order(sc, lib, bits):
    """The plan's table, the norm's counter, the moments and the parameters are
    touched by every call: no call may overtake one on another stream."""
    a, b = lib.stream(11), lib.stream(12)
    opt = sc.AdamW(tensors(300, 5), tensors(300, 5), state_bits=bits)
    opt.step(1e-3, stream=a)
    opt.set_grads(tensors(300, 5))                       # rewrites what the step reads
    opt.grad_norm(1.0, stream=b)
    opt.set_grads(tensors(300, 5), stream=a)             # and what the norm counts in
    opt.step(1e-3, clip=opt.grad_norm(1.0, stream=b))
    m, v = opt.moments(stream=a)
    opt.load(3, fake.on(0, torch.zeros(305)), fake.on(0, torch.zeros(305)), stream=b)
    opt.step(1e-3)
    opt.step(1e-3)
    opt.step(1e-3, stream=a)
    assert in_order(lib.log, lib.CALLS)
    assert [x[1] for x in lib.calls()][-4:] == [12, 0, 0, 11]
    uses = [x for x in lib.log if x[0] == "use"]
    assert {11, 12} <= {x[1] for x in uses}              # the allocator knows of both streams
    n = len(lib.log)
    opt.step(1e-3, stream=a)
    assert len(lib.log) == n + 1                         # nothing but the call where the stream stays


def test_moments_wait_for_the_steps(sc, lib):
    a = lib.stream(11)
    opt = sc.AdamW(tensors(300), tensors(300))
    opt.step(1e-3, stream=a)
    n = len(lib.log)
    opt.moments()                                        # the object's own memory: no call, but the stream waits
    assert [x[:2] for x in lib.log[n:]][:2] == [("record", 11), ("wait", 0)]


def test_router_calls_on_several_streams_run_in_order(sc, lib):
    a, b = lib.stream(11), lib.stream(12)
    r = sc.Router(12, 8, 2)
    x = logits()
    f = r.forward(x, stream=a)
    r.backward(x, f, stream=b)                           # reads what the forward pass writes
    f = r.forward(x)                                     # overwrites what the backward pass reads
    r.backward(x, f, stream=a)
    r.forward(x, stream=b)
    assert in_order(lib.log, lib.CALLS)


def test_captures_do_not_wait_for_work_outside(sc, lib):
    """A capture cannot wait for work that it does not hold, nor eager work for what
    was only captured; streams of one capture wait for one another."""
    a, b = lib.stream(11), lib.stream(12)
    r = sc.Router(12, 8, 2)
    x = logits()
    r.forward(x)
    a.capturing = b.capturing = True
    n = len(lib.log)
    f = r.forward(x, stream=a)
    assert not [x for x in lib.log[n:] if x[0] in ("record", "wait")]
    n = len(lib.log)
    r.backward(x, f, stream=b)
    assert [x[:2] for x in lib.log[n:] if x[0] in ("record", "wait")] == [("record", 11), ("wait", 12)]
    n = len(lib.log)
    r.forward(x)
    assert not [x for x in lib.log[n:] if x[0] in ("record", "wait")]
    a.capturing = b.capturing = False
    r.forward(x, stream=a)
    assert lib.log[-2][:2] == ("wait", 11)
