"""What the operators between tokens and logits refuse, before anything is launched (no GPU
needed): the C calls with addresses that nothing reads, and the objects with stand-ins."""
import ctypes
import math

import numpy as np
import pytest
import torch

from _fake_gpu import on

OK, EINVAL, EWORKSPACE = 0, 1, 2
MB = 1 << 20


@pytest.fixture(scope="module")
def sc():
    import paper_2301_08897_amd as sc
    return sc


@pytest.fixture(scope="module")
def lang(sc):
    from paper_2301_08897_amd import language
    return language


def batch(lang, off=(0, 60, 100), **more):
    K = len(off) - 1
    x = dict(tokens=100, tok_off=(ctypes.c_uint64 * (K + 1))(*off), devices=K)
    x.update(more)
    return lang.Batch(**x)


BAD_BATCHES = [dict(tokens=2**31), dict(tokens=99), dict(devices=0), dict(devices=65), dict(off=(1, 60, 100)), dict(off=(0, 101, 100)), dict(tok_off=None)]


# ---- tokens sorted by expert ------------------------------------------------------------------

def sort(lang, b, *, idx=MB, experts=8, k=2, pos=2 * MB, src=3 * MB, bounds=4 * MB, ws=5 * MB, size=MB):
    return lang._order_sort(b, idx, experts, k, pos, src, bounds, ws, size, None)


def test_sort_refusals(lang):
    for more in BAD_BATCHES:
        assert sort(lang, batch(lang, **more)) == EINVAL, more
    b = batch(lang)
    assert sort(lang, None) == EINVAL
    for more in (dict(experts=0), dict(experts=1025), dict(k=0), dict(k=17, experts=20), dict(k=9), dict(idx=None), dict(pos=None), dict(src=None),
                 dict(bounds=None), dict(idx=MB + 2), dict(pos=MB + 2), dict(src=MB + 2), dict(bounds=MB + 2),
                 dict(pos=MB + 400), dict(src=2 * MB), dict(bounds=3 * MB + 796), dict(bounds=MB)):
        assert sort(lang, b, **more) == EINVAL, more
    assert sort(lang, b, ws=None) == EWORKSPACE and sort(lang, b, ws=5 * MB + 128) == EWORKSPACE
    big = batch(lang, off=(0, 6000, 10_000), tokens=10_000)
    assert sort(lang, big, size=256) == EWORKSPACE                  # several chunks need their counts
    many = batch(lang, off=(0, 2**31 - 1), tokens=2**31 - 1, devices=1)
    assert sort(lang, many, k=2) == EINVAL                          # positions pass 31 bits


def test_order_workspace_holds_every_call(lang):
    ws = lang._order_ws_bytes
    for bad in ((2**31, 8, 1), (10, 0, 1), (10, 1025, 1), (10, 8, 0), (10, 8, 9), (10, 64, 17), (2**30, 8, 2)):
        assert ws(*bad) == 0, bad
    sizes = [ws(t, 1024, 16) for t in (1, 1000, 30_000, 2**14, 2**17, 2**17 + 1, 2**20, 2**22)]
    assert sizes == sorted(sizes) and sizes[0] > 0


def order(lang, **more):
    x = dict(tokens=100, pos=MB, k=2, dim=64, type=0)
    x.update(more)
    return lang.OrderShape(**x)


BAD_ORDERS = [dict(tokens=2**31), dict(tokens=2**30), dict(pos=None), dict(pos=MB + 2), dict(k=0), dict(k=17), dict(dim=0), dict(dim=2**24), dict(type=2)]


def moves(lang, o, *, a=2 * MB, lda=64, b=4 * MB, ldb=64, gate=6 * MB, d=8 * MB, ldd=64, d_gate=10 * MB):
    """The three calls: tokens' rows at a, experts' rows at b."""
    return (lang._dispatch(o, a, lda, b, ldb, None), lang._combine(o, b, ldb, gate, a, lda, None),
            lang._combine_backward(o, a, lda, b, ldb, gate, d, ldd, d_gate, None))


def test_move_refusals(lang):
    for more in BAD_ORDERS:
        assert moves(lang, order(lang, **more)) == (EINVAL,) * 3, more
    o = order(lang)
    assert moves(lang, None) == (EINVAL,) * 3
    for more in (dict(a=None), dict(b=None), dict(a=2 * MB + 2), dict(b=4 * MB + 1), dict(lda=63), dict(ldb=63), dict(lda=2**31)):
        assert moves(lang, o, **more) == (EINVAL,) * 3, more
    assert moves(lang, o, b=2 * MB)[:2] == (EINVAL, EINVAL)
    back = lambda **more: moves(lang, o, **more)[2]  # noqa: E731
    assert moves(lang, o, gate=6 * MB + 1)[1:] == (EINVAL, EINVAL)
    for more in (dict(gate=None), dict(d=4 * MB + 4), dict(d=4 * MB, ldd=65), dict(d=2 * MB), dict(d=6 * MB - 64), dict(d_gate=10 * MB + 2), dict(d_gate=6 * MB),
                 dict(d_gate=8 * MB), dict(d_gate=MB), dict(d_gate=4 * MB), dict(ldd=63)):
        assert back(**more) == EINVAL, more
    assert lang._dispatch(o, 2 * MB, 64, MB - 8, 64, None) == EINVAL                    # over the positions
    assert lang._combine(o, 4 * MB, 64, 2 * MB, 2 * MB, 64, None) == EINVAL             # over the gates
    empty = order(lang, tokens=0, pos=None)
    assert moves(lang, empty, a=None, b=None, gate=None, d=None, d_gate=None) == (OK,) * 3


# ---- embedding ------------------------------------------------------------------------------------

def table(lang, **more):
    x = dict(vocab=1000, dim=64, type=0, grad_type=0, token_bytes=8, scale=1.0)
    x.update(more)
    return lang.EmbeddingShape(**x)


BAD_TABLES = [dict(vocab=0), dict(vocab=2**32 - 1), dict(dim=0), dict(dim=2**24), dict(type=2), dict(grad_type=-1), dict(token_bytes=2), dict(scale=math.nan),
              dict(scale=math.inf)]


def embed(lang, e, *, tokens=100, ids=MB, weight=2 * MB, ldw=64, out=4 * MB, ldo=64):
    return lang._embedding_forward(e, tokens, ids, weight, ldw, out, ldo, None)


def embed_back(lang, e, b, *, ids=MB, d=2 * MB, ld=64, w=(4 * MB, 6 * MB), ws=8 * MB, size=64 * MB):
    at = None if w is None else (ctypes.c_void_p * len(w))(*w)
    return lang._embedding_backward(e, b, ids, d, ld, at, 0, ws, size, None)


def test_embedding_refusals(lang):
    for more in BAD_TABLES:
        assert embed(lang, table(lang, **more)) == EINVAL and embed_back(lang, table(lang, **more), batch(lang)) == EINVAL, more
    e = table(lang)
    for more in (dict(tokens=2**31), dict(ids=None), dict(ids=MB + 4), dict(weight=None), dict(weight=2 * MB + 2), dict(out=None), dict(ldw=63), dict(ldo=63),
                 dict(out=2 * MB + 256_000 - 4), dict(out=MB + 796)):
        assert embed(lang, e, **more) == EINVAL, more
    assert embed(lang, e, tokens=0, ids=None, out=None) == OK
    assert embed(lang, None) == EINVAL and embed_back(lang, None, batch(lang)) == EINVAL
    for more in BAD_BATCHES:
        assert embed_back(lang, e, batch(lang, **more)) == EINVAL, more
    b = batch(lang)
    for more in (dict(ids=None), dict(ids=MB + 4), dict(d=None), dict(d=2 * MB + 2), dict(ld=63), dict(w=None), dict(w=(None, 6 * MB)), dict(w=(4 * MB, 4 * MB + 2)),
                 dict(w=(4 * MB, 4 * MB + 4)), dict(w=(2 * MB, 6 * MB)), dict(w=(4 * MB, 8 * MB)), dict(w=(MB - 4, 6 * MB)), dict(ws=2 * MB)):
        assert embed_back(lang, e, b, **more) == EINVAL, more
    assert embed_back(lang, table(lang, vocab=2**31), b) == EINVAL                      # rows of all devices pass 32 bits
    assert embed_back(lang, e, b, ws=None) == EWORKSPACE and embed_back(lang, e, b, ws=8 * MB + 8) == EWORKSPACE
    assert embed_back(lang, e, b, size=256) == EWORKSPACE
    ws = lang._embedding_ws_bytes
    assert ws(2**31, 10, 8) == ws(10, 0, 8) == ws(10, 10, 0) == ws(10, 2**32, 8) == 0
    sizes = [ws(t, 50_000, 64) for t in (0, 1, 4096, 4097, 2**18, 2**18 + 1, 2**20)]
    assert sizes == sorted(sizes) and sizes[0] > 0


# ---- layer norm -------------------------------------------------------------------------------------

def norm(lang, **more):
    x = dict(dim=64, type=0, weight_type=0, eps=1e-5)
    x.update(more)
    return lang.NormShape(**x)


BAD_NORMS = [dict(dim=0), dict(dim=2**24), dict(type=2), dict(weight_type=3), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf)]


def norm_forward(lang, n, *, tokens=100, x=MB, ldx=64, w=2 * MB, b=3 * MB, y=4 * MB, ldy=64, mean=5 * MB, rstd=6 * MB):
    return lang._layer_norm_forward(n, tokens, x, ldx, w, b, y, ldy, mean, rstd, None)


def norm_back(lang, n, bt, *, x=MB, ldx=64, w=2 * MB, mean=3 * MB, rstd=4 * MB, g=5 * MB, ldg=64, dx=6 * MB, ldd=64, dw=(7 * MB, 8 * MB), db=(9 * MB, 10 * MB),
              ws=11 * MB, size=MB):
    at = [None if v is None else (ctypes.c_void_p * len(v))(*v) for v in (dw, db)]
    return lang._layer_norm_backward(n, bt, x, ldx, w, mean, rstd, g, ldg, dx, ldd, at[0], at[1], ws, size, None)


def test_layer_norm_refusals(lang):
    bt = batch(lang)
    for more in BAD_NORMS:
        assert norm_forward(lang, norm(lang, **more)) == EINVAL and norm_back(lang, norm(lang, **more), bt) == EINVAL, more
    n = norm(lang)
    assert norm_forward(lang, None) == EINVAL and norm_back(lang, None, bt) == EINVAL and norm_back(lang, n, None) == EINVAL
    for more in (dict(tokens=2**31), dict(x=None), dict(w=None), dict(y=None), dict(mean=None), dict(rstd=None), dict(x=MB + 2), dict(b=3 * MB + 1), dict(ldx=63),
                 dict(ldy=63), dict(y=MB), dict(y=2 * MB), dict(y=3 * MB), dict(mean=MB), dict(rstd=5 * MB), dict(mean=4 * MB)):
        assert norm_forward(lang, n, **more) == EINVAL, more
    assert norm_forward(lang, n, tokens=0, x=None, y=None, mean=None, rstd=None) == OK
    for more in BAD_BATCHES:
        assert norm_back(lang, n, batch(lang, **more)) == EINVAL, more
    for more in (dict(x=None), dict(w=None), dict(mean=None), dict(rstd=None), dict(g=None), dict(dx=None), dict(g=5 * MB + 2), dict(ldx=63), dict(ldg=63),
                 dict(ldd=63), dict(dx=MB), dict(dx=5 * MB), dict(dx=11 * MB), dict(dw=(None, 8 * MB)), dict(dw=(7 * MB + 1, 8 * MB)), dict(dw=(7 * MB, 7 * MB + 252)),
                 dict(db=(7 * MB, 10 * MB)), dict(dw=(MB, 8 * MB)), dict(db=(6 * MB, 10 * MB)), dict(ws=5 * MB)):
        assert norm_back(lang, n, bt, **more) == EINVAL, more
    assert norm_back(lang, n, bt, ws=None) == EWORKSPACE and norm_back(lang, n, bt, ws=11 * MB + 4) == EWORKSPACE
    assert norm_back(lang, n, bt, size=256) == EWORKSPACE
    ws = lang._layer_norm_ws_bytes
    assert ws(2**31, 8) == ws(8, 0) == ws(8, 2**24) == 0 and ws(0, 1) > 0


# ---- cross entropy -------------------------------------------------------------------------------------

def entropy(lang, **more):
    x = dict(vocab=1000, dim=64, type=0, grad_type=0, target_bytes=8)
    x.update(more)
    return lang.CrossEntropyShape(**x)


BAD_ENTROPIES = [dict(vocab=0), dict(vocab=2**22 + 1), dict(dim=0), dict(dim=65_537), dict(type=2), dict(grad_type=2), dict(target_bytes=1)]


def outs(lang, **more):
    x = dict(nll=5 * MB, lse=6 * MB, device_loss=7 * MB, share=8 * MB, loss=9 * MB)
    x.update(more)
    return lang.CrossEntropyOut(**x)


def weights(*w):
    return (ctypes.c_float * len(w))(*w)


def loss(lang, e, b, *, wt=weights(0.5, 0.5), x=MB, ldx=64, w=2 * MB, ldw=64, t=4 * MB, o=None, ws=16 * MB, size=64 * MB):
    return lang._cross_entropy_forward(e, b, wt, x, ldx, w, ldw, t, o or outs(lang), ws, size, None)


def loss_back(lang, e, b, *, wt=None, x=MB, ldx=64, w=2 * MB, ldw=64, t=4 * MB, o=None, d=None, dx=10 * MB, ldd=64, dw=(11 * MB, 13 * MB), ws=16 * MB, size=64 * MB):
    at = None if dw is None else (ctypes.c_void_p * len(dw))(*dw)
    return lang._cross_entropy_backward(e, b, wt, x, ldx, w, ldw, t, o or outs(lang), d, dx, ldd, at, ws, size, None)


def test_cross_entropy_refusals(lang):
    b = batch(lang)
    for more in BAD_ENTROPIES:
        assert loss(lang, entropy(lang, **more), b) == EINVAL and loss_back(lang, entropy(lang, **more), b) == EINVAL, more
        assert lang._cross_entropy_ws_bytes(entropy(lang, **more), b, 1) == 0
    e = entropy(lang)
    assert loss(lang, None, b) == EINVAL and loss(lang, e, None) == EINVAL and loss_back(lang, None, b) == EINVAL
    for more in BAD_BATCHES:
        assert loss(lang, e, batch(lang, **more)) == EINVAL and loss_back(lang, e, batch(lang, **more)) == EINVAL, more
        assert lang._cross_entropy_ws_bytes(e, batch(lang, **more), 0) == 0
    many = batch(lang, off=(0, 2**22 + 1), tokens=2**22 + 1, devices=1)
    assert loss(lang, e, many, wt=weights(1.0)) == EINVAL and loss_back(lang, e, many, dw=(11 * MB,)) == EINVAL
    for more in (dict(x=None), dict(w=None), dict(t=None), dict(x=MB + 2), dict(w=2 * MB + 1), dict(t=4 * MB + 4), dict(ldx=63), dict(ldw=63), dict(ldw=2**31),
                 dict(wt=weights(0.5, -0.5)), dict(wt=weights(0.5, math.nan)), dict(o=outs(lang, lse=None)), dict(o=outs(lang, share=None)),
                 dict(o=outs(lang, lse=6 * MB + 2)), dict(o=outs(lang, share=8 * MB + 1))):
        assert loss(lang, e, b, **more) == EINVAL and loss_back(lang, e, b, **more) == EINVAL, more
    assert loss(lang, e, b, wt=None) == EINVAL
    for more in (dict(nll=None), dict(device_loss=None), dict(loss=None), dict(nll=5 * MB + 2), dict(nll=6 * MB), dict(nll=MB), dict(loss=2 * MB), dict(lse=16 * MB),
                 dict(share=7 * MB + 4)):
        assert loss(lang, e, b, o=outs(lang, **more)) == EINVAL, more
    for more in (dict(dx=None), dict(dx=10 * MB + 2), dict(ldd=63), dict(d=2), dict(dx=MB), dict(dx=2 * MB), dict(dx=16 * MB), dict(dx=6 * MB), dict(dw=(None, 13 * MB)),
                 dict(dw=(11 * MB + 2, 13 * MB)), dict(dw=(11 * MB, 11 * MB + 4)), dict(dw=(2 * MB, 13 * MB)), dict(dw=(11 * MB, 16 * MB)), dict(ws=2 * MB)):
        assert loss_back(lang, e, b, **more) == EINVAL, more
    for call in (loss, loss_back):
        assert call(lang, e, b, ws=None) == EWORKSPACE and call(lang, e, b, ws=16 * MB + 4) == EWORKSPACE and call(lang, e, b, size=256) == EWORKSPACE


def test_refusals_have_a_message(sc, lang):
    with pytest.raises(sc.ScadlesError, match="dim = 0"):
        sc._check(norm_forward(lang, norm(lang, dim=0)))


# ---- objects --------------------------------------------------------------------------------------------

def test_objects_refuse_their_shapes(sc):
    for make in (lambda: sc.ExpertOrder(0, 1), lambda: sc.ExpertOrder(8, 9), lambda: sc.ExpertOrder(8, 0), lambda: sc.ExpertOrder(2000, 2), lambda: sc.ExpertOrder(8, 2, devices=65),
                 lambda: sc.ExpertOrder(-1, 1), lambda: sc.Embedding(0, 8), lambda: sc.Embedding(8, 0), lambda: sc.Embedding(8, 8, devices=0), lambda: sc.Embedding(8, 8, scale=math.inf),
                 lambda: sc.Embedding(2**31, 8, devices=2), lambda: sc.LayerNorm(0), lambda: sc.LayerNorm(8, eps=-1.0), lambda: sc.LayerNorm(8, eps=math.nan), lambda: sc.LayerNorm(8, devices=65),
                 lambda: sc.LinearCrossEntropy(0, 8), lambda: sc.LinearCrossEntropy(2**23, 8), lambda: sc.LinearCrossEntropy(8, 2**17), lambda: sc.LinearCrossEntropy(8, 8, devices=0)):
        with pytest.raises(sc.ScadlesError):
            make()


def test_objects_refuse_tensors_of_the_host(sc):
    x, w, i = torch.zeros(4, 8), torch.zeros(8), torch.zeros(4, dtype=torch.int64)
    r = sc.ExpertRows(torch.zeros(4, 2, dtype=torch.int32), None, None)
    o, e, n, c = sc.ExpertOrder(8, 2), sc.Embedding(10, 8), sc.LayerNorm(8), sc.LinearCrossEntropy(10, 8)
    f = sc.LayerNormOutputs(x, w[:4], w[:4])
    g = sc.CrossEntropyOutputs(w[:4], w[:4], w[:1], w[:1], w[:1])
    for call in (lambda: o.sort(r.pos), lambda: o.dispatch(x, r), lambda: o.combine(torch.zeros(8, 8), torch.zeros(4, 2), r), lambda: o.dispatch_backward(torch.zeros(8, 8), r),
                 lambda: o.combine_backward(x, torch.zeros(8, 8), torch.zeros(4, 2), r), lambda: e.forward(i, torch.zeros(10, 8)), lambda: e.backward(i, x, torch.zeros(10, 8)),
                 lambda: n.forward(x, w), lambda: n.backward(x, w, f, x), lambda: c.forward(x, torch.zeros(10, 8), i), lambda: c.backward(x, torch.zeros(10, 8), i, g)):
        with pytest.raises(TypeError, match="must be a GPU tensor"):
            call()


def gpu(*shape, dtype=torch.float32, g=0):
    return on(g, torch.zeros(*shape, dtype=dtype))


def test_objects_refuse_other_shapes_types_and_gpus(sc):
    bf = torch.bfloat16
    x, w = gpu(4, 8), gpu(8)
    r = sc.ExpertRows(gpu(4, 2, dtype=torch.int32), None, None)
    o, e, n, c = sc.ExpertOrder(8, 2, devices=2), sc.Embedding(10, 8, devices=2), sc.LayerNorm(8, devices=2), sc.LinearCrossEntropy(10, 8, devices=2)
    i, table, grads = gpu(4, dtype=torch.int64), gpu(10, 8), gpu(2, 10, 8)
    f = sc.LayerNormOutputs(x, w[:4], w[:4])
    g = sc.CrossEntropyOutputs(w[:4], w[:4], w[:2], w[:2], w[:1])
    off = [0, 2, 4]
    bad = [
        lambda: o.sort(gpu(4, 3, dtype=torch.int32), tok_off=off), lambda: o.sort(gpu(4, 2, dtype=torch.int64), tok_off=off), lambda: o.sort(r.pos), lambda: o.sort(r.pos, tok_off=[0, 4]),
        lambda: o.sort(r.pos, tok_off=[0, -1, 4]), lambda: o.sort(gpu(2, 4, dtype=torch.int32).T, tok_off=off),
        lambda: o.dispatch(gpu(5, 8), r), lambda: o.dispatch(gpu(4, 8, dtype=torch.float16), r), lambda: o.dispatch(gpu(4, 8, g=1), r), lambda: o.dispatch(gpu(8, 4).T, r),
        lambda: o.dispatch(gpu(1, 8).expand(4, 8), r), lambda: o.dispatch(x, r, out=gpu(7, 8)), lambda: o.dispatch(x, r, out=gpu(8, 8, dtype=bf)),
        lambda: o.combine(gpu(8, 8), gpu(4, 3), r), lambda: o.combine(gpu(7, 8), gpu(4, 2), r), lambda: o.combine(gpu(8, 8), gpu(4, 2, dtype=bf), r),
        lambda: o.combine_backward(gpu(4, 7), gpu(8, 8), gpu(4, 2), r), lambda: o.combine_backward(gpu(4, 8, dtype=bf), gpu(8, 8), gpu(4, 2), r),
        lambda: e.forward(i, gpu(9, 8)), lambda: e.forward(gpu(4), table), lambda: e.forward(gpu(4, dtype=torch.int64, g=1), table),
        lambda: e.backward(i, gpu(3, 8), grads, tok_off=off), lambda: e.backward(i, x, gpu(10, 8), tok_off=off), lambda: e.backward(i, x, [table], tok_off=off),
        lambda: e.backward(i, x, [table, gpu(10, 8, dtype=bf)], tok_off=off), lambda: e.backward(i, x, [table, gpu(9, 8)], tok_off=off), lambda: e.backward(i, x, grads),
        lambda: e.backward(i, x, gpu(2, 10, 8, dtype=torch.float64), tok_off=off), lambda: e.backward(i, x, gpu(10, 2, 8).transpose(0, 1)[:, :, ::1], tok_off=off),
        lambda: n.forward(gpu(4, 7), w), lambda: n.forward(x, gpu(7)), lambda: n.forward(x, w, gpu(8, dtype=bf)), lambda: n.forward(x, w, out=gpu(4, 8, dtype=bf)),
        lambda: n.backward(x, w, f, gpu(3, 8)), lambda: n.backward(x, w, sc.LayerNormOutputs(x, w[:3], w[:4]), x), lambda: n.backward(x, w, f, x, gpu(2, 8, dtype=bf), tok_off=off),
        lambda: n.backward(x, w, f, x, gpu(1, 8), tok_off=off), lambda: n.backward(x, w, f, x, gpu(2, 8)),
        lambda: c.forward(x, gpu(10, 8, dtype=bf), i, tok_off=off), lambda: c.forward(x, table, gpu(5, dtype=torch.int64), tok_off=off), lambda: c.forward(x, table, gpu(4), tok_off=off),
        lambda: c.forward(x, table, i, tok_off=off, weights=[1.0]), lambda: c.forward(x, table, i),
        lambda: c.backward(x, table, i, g, gpu(10, 8), tok_off=off), lambda: c.backward(x, table, i, g, grads, tok_off=off, d_loss=gpu(2)),
        lambda: c.backward(x, table, i, g, grads, tok_off=off, d_x=gpu(4, 9)), lambda: c.backward(x, table, i, sc.CrossEntropyOutputs(w[:4], w[:3], w[:2], w[:2], w[:1]), grads, tok_off=off),
    ]
    for k, call in enumerate(bad):
        with pytest.raises((TypeError, ValueError)):
            call()
            pytest.fail(f"call {k} was not refused")


def test_the_library_and_the_binding_agree(lang):
    """Sizes of the structs that cross the boundary, as the C compiler lays them out."""
    assert ctypes.sizeof(lang.Batch) == 24 and ctypes.sizeof(lang.OrderShape) == 32 and ctypes.sizeof(lang.EmbeddingShape) == 32
    assert ctypes.sizeof(lang.NormShape) == 16 and ctypes.sizeof(lang.CrossEntropyShape) == 24 and ctypes.sizeof(lang.CrossEntropyOut) == 40


def test_oracles_agree_with_other_forms():
    """The plain forms against torch's own in 64 bits."""
    from oracle import language as ol
    rng = np.random.default_rng(1)
    x, w, t = rng.normal(0, 1, (12, 5)), rng.normal(0, 1, (7, 5)), rng.integers(0, 7, 12)
    z, nll, lse, each, share, loss = ol.cross_entropy(x, w, t, [0, 4, 12], np.array([0.25, 0.75]))
    xt, wt = torch.from_numpy(x).requires_grad_(), torch.from_numpy(w).requires_grad_()
    ref = torch.nn.functional.cross_entropy(xt @ wt.T, torch.from_numpy(t), reduction="none")
    assert np.allclose(nll, ref.detach().numpy(), rtol=1e-12) and np.allclose(each, [ref[:4].mean().item(), ref[4:].mean().item()], rtol=1e-12)
    ref[:4].mean().backward(retain_graph=True)
    g, dx, dw = ol.cross_entropy_gradients(x, w, t, [0, 4, 12], z, lse, share)
    assert np.allclose(dw[0], wt.grad.numpy(), atol=1e-14) and np.allclose(dx[:4], xt.grad.numpy()[:4], atol=1e-14)
    g0, b0 = rng.normal(0, 1, 5), rng.normal(0, 1, 5)
    y, mean, rstd, h = ol.layer_norm(x, g0, b0, 1e-3)
    xt = torch.from_numpy(x).requires_grad_()
    gt, bt = torch.from_numpy(g0).requires_grad_(), torch.from_numpy(b0).requires_grad_()
    ref = torch.nn.functional.layer_norm(xt, (5,), gt, bt, 1e-3)
    up = rng.normal(0, 1, (12, 5))
    ref.backward(torch.from_numpy(up))
    d_x, d_w, d_b = ol.layer_norm_gradients(h, rstd, g0, up, [0, 3, 12])
    assert np.allclose(y, ref.detach().numpy(), atol=1e-12) and np.allclose(d_x, xt.grad.numpy(), atol=1e-12)
    assert np.allclose(d_w.sum(axis=0), gt.grad.numpy(), atol=1e-12) and np.allclose(d_b.sum(axis=0), bt.grad.numpy(), atol=1e-12)
    total, _ = ol.embed_gradients(np.array([1, -1, 1, 0]), x[:4], 3, 2.0, [0, 2, 4])
    assert np.allclose(total[0, 1], 2 * x[0]) and np.allclose(total[1, 1], 2 * x[2]) and np.allclose(total[1, 0], 2 * x[3]) and not total[0, 0].any()
    pos, src, bounds = ol.order(np.array([[1, 0], [1, 5], [0, 1]]), 2, [0, 1, 3])
    assert pos.tolist() == [[2, 0], [3, -1], [1, 4]] and src.tolist() == [1, 4, 0, 2, 5, -1] and bounds.tolist() == [0, 1, 2, 3, 5]
