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


def test_tensors_of_another_gpu_are_refused(sc, lib):
    here, there = tensors(300, 5), tensors(300, 5, gpu=1)
    mixed = [here[0], there[1]]
    for params, grads in ((mixed, here), (here, mixed), (there, here)):
        with pytest.raises(ValueError):
            sc.AdamW(params, grads)
    with pytest.raises(ValueError):
        sc.AdamW(here, here, copies=tensors(300, 5, gpu=1, dtype=torch.bfloat16))
    opt = sc.AdamW(here, here)
    calls = len(lib.calls())
    with pytest.raises(ValueError):
        opt.set_grads(there)
    with pytest.raises(ValueError):
        opt.step(1e-3, clip=fake.on(1, torch.ones(2)))
    for m, v in ((0, 1), (1, 0)):
        with pytest.raises(ValueError):
            opt.load(3, fake.on(m, torch.zeros(305)), fake.on(v, torch.zeros(305)))
    r = sc.Router(12, 8, 2)
    f = r.forward(logits())
    for more in (dict(logits=logits(gpu=1)), dict(logits=logits(), valid=fake.on(1, torch.ones(12, dtype=torch.bool)))):
        with pytest.raises(ValueError):
            r.forward(**more)
    x = logits()
    f = r.forward(x)
    for more in (dict(logits=logits(gpu=1)), dict(d_gate=fake.on(1, torch.zeros(12, 2))), dict(d_loss=fake.on(1, torch.zeros(2))),
                 dict(d_logits=logits(gpu=1))):
        with pytest.raises(ValueError):
            r.backward(**{**dict(logits=x, out=f), **more})
    assert len(lib.calls()) == calls + 2 and opt.t == 0


def test_calls_run_on_the_objects_gpu(sc, lib):
    """Default streams all have the address 0: a call means its object's GPU's, whatever
    GPU is current."""
    cuda = lib.torch.cuda
    cuda.current[1] = lib.stream(0, gpu=1)
    opt = sc.AdamW(tensors(300, 5, gpu=1), tensors(300, 5, gpu=1), state_bits=8)
    r = sc.Router(12, 8, 2, device="cuda:1")
    x = logits(gpu=1)
    assert cuda.gpu == 0 and opt.m.device.index == 1 and r.idx.device.index == 1
    opt.step(1e-3, clip=opt.grad_norm(1.0))
    opt.load(4, *opt.moments())
    opt.set_grads(tensors(300, 5, gpu=1))
    r.backward(x, r.forward(x))
    with cuda.device(1):
        opt.step(1e-3)
    cuda.current[1] = lib.stream(21, gpu=1)              # another current stream there
    opt.step(1e-3)
    opt.step(1e-3, stream=lib.stream(22, gpu=1))
    assert [x[2] for x in lib.calls()] == [1] * len(lib.calls())
    assert [x[1] for x in lib.calls()][-3:] == [0, 21, 22] and not any(x[1] for x in lib.calls()[:-2])
    calls = len(lib.calls())
    for call in (lambda s: opt.step(1e-3, stream=s), lambda s: opt.grad_norm(1.0, stream=s), lambda s: opt.moments(stream=s),
                 lambda s: opt.load(4, opt.m, opt.v, tops=opt.tops, stream=s), lambda s: opt.set_grads(opt.grads, stream=s),
                 lambda s: r.forward(x, stream=s)):
        with pytest.raises(ValueError):
            call(lib.stream(11, gpu=0))
    assert len(lib.calls()) == calls
    with pytest.raises(ValueError):
        sc.AdamW(tensors(300, gpu=1), tensors(300, gpu=1), stream=lib.stream(11, gpu=0))


def raised(tensors, call):
    """Which of the tensors' version counters a call raises."""
    before = [x._version for x in tensors]
    call()
    return [x._version > n for x, n in zip(tensors, before)]


def test_what_is_written_has_a_new_version(sc, lib):
    """autograd refuses a backward pass that needs a tensor written since; it sees by
    the version that one was."""
    flat, flat_copy = tensors(500)[0], tensors(500, dtype=torch.bfloat16)[0]
    params, grads = list(torch.split(flat, [300, 200])) + tensors(7), tensors(300, 200, 7)
    copies = list(torch.split(flat_copy, [300, 200])) + tensors(7, dtype=torch.bfloat16)
    opt = sc.AdamW(params, grads, copies=copies)
    seen = [flat, flat_copy, *params, *copies, opt.m, opt.v]
    assert all(raised(seen, lambda: opt.step(1e-3)))
    assert not any(raised(grads + [opt.clip], lambda: opt.step(1e-3)))
    assert raised([opt.clip, *seen], lambda: opt.grad_norm(1.0)) == [True] + [False] * len(seen)
    assert all(raised([opt.m, opt.v], lambda: opt.load(3, fake.on(0, torch.zeros(507)), fake.on(0, torch.zeros(507)))))
    small = sc.AdamW(params, grads, state_bits=8)
    assert all(raised([flat, params[2], small.m, small.v, small.tops], lambda: small.step(1e-3)))
    lib.status = 1
    for call in (lambda: opt.step(1e-3), lambda: opt.grad_norm(1.0)):
        with pytest.raises(sc.ScadlesError):
            assert not any(raised(seen + [opt.clip], call))
    lib.status = 0

    r = sc.Router(12, 8, 2)
    outs = [r.idx, r.gate, r.lse, r.counts, r.load, r.share, r.loss]
    x, d = logits(), logits()
    f = r.forward(x)
    assert all(raised(outs + [f.gate], lambda: r.forward(x)))
    assert raised([d, x, *outs], lambda: r.backward(x, f, d_logits=d)) == [True] + [False] * 8
    w = torch.ones(12, 2, requires_grad=True)
    y = (w * r.forward(x).gate).sum()
    r.forward(logits())
    with pytest.raises(RuntimeError):
        y.backward()


def test_inference_tensors(sc, lib):
    """Tensors without a version are taken as well."""
    with torch.inference_mode():
        params, copies = tensors(300, 5), tensors(300, 5, dtype=torch.bfloat16)
        opt, r, x, d = sc.AdamW(params, tensors(300, 5), copies=copies), sc.Router(12, 8, 2), logits(), logits()
    for mode in (True, False):
        with torch.inference_mode(mode):
            opt.step(1e-3, clip=opt.grad_norm(1.0))
            opt.load(3, fake.on(0, torch.zeros(305)), fake.on(0, torch.zeros(305)))
            r.backward(x, r.forward(x), d_logits=d)


def test_order_across_a_capture(sc, lib):
    """Calls after a capture wait for the calls before it, on whatever streams the
    captured ones were."""
    a, b = lib.stream(11), lib.stream(12)
    for after in (a, b):
        r = sc.Router(12, 8, 2)
        x = logits()
        r.forward(x)
        a.capturing = True
        r.backward(x, r.forward(x, stream=a), stream=a)
        a.capturing = False
        n = len(lib.log)
        r.forward(x, stream=after)
        r.forward(x, stream=after)
        assert [x[:2] for x in lib.log[n:] if x[0] in ("record", "wait")] == [("record", 0), ("wait", after.cuda_stream)]
    r = sc.Router(12, 8, 2)
    r.forward(x, stream=a)
    a.capturing = b.capturing = True                     # the same stream, then one that joins its capture
    f = r.forward(x, stream=a)
    n = len(lib.log)
    r.backward(x, f, stream=b)
    a.capturing = b.capturing = False
    r.forward(x)
    assert [x[:2] for x in lib.log[n:] if x[0] in ("record", "wait")] == [("record", 11), ("wait", 12), ("record", 11), ("wait", 0)]
