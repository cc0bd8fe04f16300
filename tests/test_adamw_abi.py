"""AdamW's C ABI on the host: what it refuses, before anything is launched (no
GPU needed), and the plain form of the 8-bit moments that the GPU tests use."""
import ctypes
import math

import numpy as np
import pytest

from oracle import training as ot

EINVAL, EWORKSPACE = 1, 2


@pytest.fixture(scope="module")
def sc():
    import paper_2301_08897_amd as sc
    return sc


def tensor(sc, **more):
    x = dict(param=1 << 20, grad=2 << 20, m=3 << 20, v=4 << 20, tops=None, copy=None, n=1000, weight_decay=0.01)
    x.update(more)
    return (sc.AdamWTensor * 1)(sc.AdamWTensor(**x))


def build(sc, t, *, count=1, bits=32, grads=0, table=1 << 28, size=1 << 20, plan=True):
    return sc._adamw_plan_build(t, count, bits, grads, table, size, ctypes.byref(sc.AdamWPlan()) if plan else None, None)


def test_plan_refusals(sc):
    assert build(sc, None) == EINVAL
    assert build(sc, tensor(sc), count=0) == EINVAL
    assert build(sc, tensor(sc), count=(1 << 20) + 1) == EINVAL       # before any tensor is read
    assert build(sc, tensor(sc), bits=16) == EINVAL
    assert build(sc, tensor(sc), grads=2) == EINVAL
    assert build(sc, tensor(sc), plan=False) == EINVAL
    assert build(sc, tensor(sc), table=None) == EWORKSPACE
    assert build(sc, tensor(sc), table=(1 << 28) + 64) == EWORKSPACE
    assert build(sc, tensor(sc), size=1024) == EWORKSPACE
    for name in ("param", "grad", "m", "v"):
        assert build(sc, tensor(sc, **{name: None})) == EINVAL, name
    for name, value in (("param", 2), ("grad", 2), ("m", 2), ("v", 1), ("copy", 1)):
        assert build(sc, tensor(sc, **{name: (9 << 20) + value})) == EINVAL, name
    assert build(sc, tensor(sc, grad=(2 << 20) + 1), grads=1) == EINVAL
    assert build(sc, tensor(sc), bits=8) == EINVAL                    # tops is missing
    assert build(sc, tensor(sc, tops=5 << 20)) == EINVAL              # tops is for 8 bits
    assert build(sc, tensor(sc, tops=(5 << 20) + 2), bits=8) == EINVAL
    assert build(sc, tensor(sc, m=(1 << 20) + 3996)) == EINVAL        # the last float of param
    assert build(sc, tensor(sc, copy=(4 << 20) + 3998)) == EINVAL
    assert build(sc, tensor(sc, weight_decay=math.nan)) == EINVAL
    assert build(sc, tensor(sc, n=2**32)) == EINVAL
    assert b"2^32" in sc._last_error()


def test_plan_bytes(sc):
    t = tensor(sc)
    assert sc._adamw_plan_bytes(t, 0) == 0 and sc._adamw_plan_bytes(None, 1) == 0
    small = sc._adamw_plan_bytes(t, 1)
    big = sc._adamw_plan_bytes(tensor(sc, n=143_667_240), 1)
    assert 0 < small < big < 143_667_240 // 16
    assert sc._adamw_plan_bytes(tensor(sc, n=2**32), 1) == 0
    assert sc._adamw_plan_bytes(tensor(sc, n=0), 1) > 0
    many = (sc.AdamWTensor * 9)(*[sc.AdamWTensor(n=2**32 - 1) for _ in range(9)])
    assert sc._adamw_plan_bytes(many, 9) == 0                         # more threads than one launch has


def made(sc, **more):
    x = dict(table=1 << 28, chunks_at=1 << 16, chunks=1, n=1000, moment_bits=32, grad_type=0, magic=0x5C4D0001)
    x.update(more)
    return ctypes.byref(sc.AdamWPlan(**x))


def test_call_refusals(sc):
    good = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)

    def step(plan=made(sc), clip=None, **more):
        return sc._adamw_step(plan, ctypes.byref(sc.AdamWOptions(**{**good, **more})), clip, None)

    assert step(plan=None) == EINVAL and step(plan=made(sc, magic=0)) == EINVAL
    assert sc._adamw_step(made(sc), None, None, None) == EINVAL
    for more in (dict(lr=math.inf), dict(lr=math.nan), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan),
                 dict(eps=0.0), dict(eps=1e-60), dict(eps=math.inf), dict(eps=1e39), dict(step=0)):
        assert step(**more) == EINVAL, more
    assert step(clip=(1 << 20) + 2) == EINVAL
    for bad in (0.0, -1.0, math.nan):
        assert sc._grad_norm(made(sc), bad, 1 << 20, None) == EINVAL
    assert sc._grad_norm(made(sc), 1.0, None, None) == EINVAL
    assert sc._grad_norm(made(sc), 1.0, (1 << 20) + 1, None) == EINVAL
    assert sc._grad_norm(made(sc, magic=1), 1.0, 1 << 20, None) == EINVAL
    for f in (lambda m, v: sc._adamw_get_moments(made(sc), m, v, None), lambda m, v: sc._adamw_set_moments(made(sc), m, v, 1, None)):
        assert f(None, 1 << 20) == EINVAL and f(1 << 20, None) == EINVAL
        assert f(1 << 20, (1 << 20) + 3996) == EINVAL and f((1 << 20) + 2, 2 << 20) == EINVAL
    assert sc._adamw_get_moments(None, 1 << 20, 2 << 20, None) == EINVAL


def test_python_refusals(sc):
    import torch
    p = torch.zeros(10)
    with pytest.raises(TypeError):
        sc.AdamW([p], [p])                                            # not on a GPU
    with pytest.raises(ValueError):
        sc.AdamW([], [])
    with pytest.raises(ValueError):
        sc.AdamW([p], [p], state_bits=16)


def test_encode_is_a_neighbour_and_keeps_its_own_values():
    rng = np.random.default_rng(1)
    x = (rng.normal(0, 1, 5001) * np.exp(rng.normal(0, 1.5, 5001))).astype(np.float32)
    for signed, y in ((True, x), (False, np.abs(x))):
        for t in (1, 2, 1000):
            z = ot.decode(*ot.encode(y, t, signed=signed), signed=signed)
            inside = np.abs(y) > np.abs(y).max() * 2.0**-15
            assert np.all(np.abs(z - y)[inside] <= 0.125 * np.abs(y)[inside])
            assert np.array_equal(ot.decode(*ot.encode(z, t + 7, signed=signed), signed=signed), z)


def test_dither_rounds_without_bias():
    """Of many equal values the share rounded up is the value's place between two
    steps: a Weyl sequence of n terms whose multiplier has small partial
    quotients is uniform to within 2 log2(n) / n."""
    n = 256 * 400
    for signed in (True, False):
        for place in (0.001, 0.1, 0.5, 0.93):
            for t in (1, 77, 10**6):
                x = np.full(n, 0.75 + 0.0625 * place, dtype=np.float32)
                up = (ot.decode(*ot.encode(x, t, signed=signed), signed=signed) > 0.75).mean()
                assert abs(up - (float(x[0]) - 0.75) / 0.0625) <= 2 * math.log2(n) / n
