"""What lies between tokens and logits of language models trained on K devices:
tokens sorted by expert and back, beside the router, the embedding, layer norm, and
the cross entropy of the logits without keeping them. Part of the package's
binding (``scadles.h``, "between tokens and logits"): checks of tensors and
marshalling.

The objects hold shapes only. Outputs, and scratch memory that a call needs, are
allocated for the call on its stream, so calls may be made on several streams, in
threads and in several captured graphs at once; what the caller does with a
tensor on other streams is the caller's to order. Outside autograd: outputs have no
history, and gradients are handed on with ``tensor.backward(gradient)``."""
from __future__ import annotations

import ctypes
import math
from dataclasses import dataclass

import numpy as np
import torch

import paper_2301_08897_amd as _sc

_vp, _u64, _u32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32


class Batch(ctypes.Structure):
    """scadles_batch: the rows of the devices."""
    _fields_ = [("tokens", _u64), ("tok_off", ctypes.POINTER(_u64)), ("devices", _u32)]


class OrderShape(ctypes.Structure):
    """scadles_order: the order that rows are moved by."""
    _fields_ = [("tokens", _u64), ("pos", _vp), ("k", _u32), ("dim", _u32), ("type", ctypes.c_int32)]


class EmbeddingShape(ctypes.Structure):
    """scadles_embedding: a table and its types."""
    _fields_ = [("vocab", _u64), ("dim", _u32), ("type", ctypes.c_int32), ("grad_type", ctypes.c_int32),
                ("token_bytes", ctypes.c_int32), ("scale", ctypes.c_float)]


class NormShape(ctypes.Structure):
    """scadles_norm: a layer norm and its types."""
    _fields_ = [("dim", _u32), ("type", ctypes.c_int32), ("weight_type", ctypes.c_int32), ("eps", ctypes.c_float)]


class CrossEntropyShape(ctypes.Structure):
    """scadles_cross_entropy: a linear layer over a vocabulary and its types."""
    _fields_ = [("vocab", _u64), ("dim", _u32), ("type", ctypes.c_int32), ("grad_type", ctypes.c_int32),
                ("target_bytes", ctypes.c_int32)]


class CrossEntropyOut(ctypes.Structure):
    """scadles_cross_entropy_out: what the forward pass writes."""
    _fields_ = [("nll", _vp), ("lse", _vp), ("device_loss", _vp), ("share", _vp), ("loss", _vp)]


_order_ws_bytes = _sc._sig("scadles_order_workspace_bytes", ctypes.c_size_t, _u64, _u32, _u32)
_order_sort = _sc._sig("scadles_order_sort", ctypes.c_int, ctypes.POINTER(Batch), _vp, _u32, _u32, _vp, _vp, _vp, _vp,
                       ctypes.c_size_t, _vp)
_dispatch = _sc._sig("scadles_dispatch", ctypes.c_int, ctypes.POINTER(OrderShape), _vp, _u64, _vp, _u64, _vp)
_combine = _sc._sig("scadles_combine", ctypes.c_int, ctypes.POINTER(OrderShape), _vp, _u64, _vp, _vp, _u64, _vp)
_combine_backward = _sc._sig("scadles_combine_backward", ctypes.c_int, ctypes.POINTER(OrderShape), _vp, _u64, _vp, _u64,
                             _vp, _vp, _u64, _vp, _vp)
_embedding_forward = _sc._sig("scadles_embedding_forward", ctypes.c_int, ctypes.POINTER(EmbeddingShape), _u64, _vp, _vp, _u64,
                              _vp, _u64, _vp)
_embedding_ws_bytes = _sc._sig("scadles_embedding_workspace_bytes", ctypes.c_size_t, _u64, _u64, _u32)
_embedding_backward = _sc._sig("scadles_embedding_backward", ctypes.c_int, ctypes.POINTER(EmbeddingShape),
                               ctypes.POINTER(Batch), _vp, _vp, _u64, ctypes.POINTER(_vp), ctypes.c_int, _vp,
                               ctypes.c_size_t, _vp)
_layer_norm_forward = _sc._sig("scadles_layer_norm_forward", ctypes.c_int, ctypes.POINTER(NormShape), _u64, _vp, _u64, _vp,
                               _vp, _vp, _u64, _vp, _vp, _vp)
_layer_norm_ws_bytes = _sc._sig("scadles_layer_norm_workspace_bytes", ctypes.c_size_t, _u64, _u32)
_layer_norm_backward = _sc._sig("scadles_layer_norm_backward", ctypes.c_int, ctypes.POINTER(NormShape),
                                ctypes.POINTER(Batch), _vp, _u64, _vp, _vp, _vp, _vp, _u64, _vp, _u64,
                                ctypes.POINTER(_vp), ctypes.POINTER(_vp), _vp, ctypes.c_size_t, _vp)
_cross_entropy_ws_bytes = _sc._sig("scadles_cross_entropy_workspace_bytes", ctypes.c_size_t,
                                   ctypes.POINTER(CrossEntropyShape), ctypes.POINTER(Batch), ctypes.c_int)
_cross_entropy_forward = _sc._sig("scadles_cross_entropy_forward", ctypes.c_int, ctypes.POINTER(CrossEntropyShape),
                                  ctypes.POINTER(Batch), ctypes.POINTER(ctypes.c_float), _vp, _u64, _vp, _u64, _vp,
                                  ctypes.POINTER(CrossEntropyOut), _vp, ctypes.c_size_t, _vp)
_cross_entropy_backward = _sc._sig("scadles_cross_entropy_backward", ctypes.c_int, ctypes.POINTER(CrossEntropyShape),
                                   ctypes.POINTER(Batch), ctypes.POINTER(ctypes.c_float), _vp, _u64, _vp, _u64, _vp,
                                   ctypes.POINTER(CrossEntropyOut), _vp, _vp, _u64, ctypes.POINTER(_vp), _vp,
                                   ctypes.c_size_t, _vp)


# ---- arguments --------------------------------------------------------------------------------------

_F32, _I32 = (torch.float32,), (torch.int32,)
_FLOATS, _INTEGERS = (torch.float32, torch.bfloat16), (torch.int32, torch.int64)


def _gpu(t, name, kinds, like):
    """Refuses what is not a GPU tensor of these types, on the GPU of ``like`` if given."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype not in kinds:
        raise TypeError(f"{name} must be {' or '.join(str(d).removeprefix('torch.') for d in kinds)}, not {t.dtype}")
    if like is not None and t.device != like.device:
        raise ValueError(f"{name} must be on {like.device}")


def _rows(t, name, rows, dim, kinds, like=None):
    """(address, elements between rows) of a [rows, dim] tensor whose rows' elements
    are adjacent; any number for None."""
    _gpu(t, name, kinds, like)
    shape = t.shape
    if len(shape) != 2 or (rows is not None and shape[0] != rows) or (dim is not None and shape[1] != dim):
        raise ValueError(f"{name} must be [{'rows' if rows is None else rows}, {'dim' if dim is None else dim}], not {list(shape)}")
    if t.is_contiguous():
        return t.data_ptr(), shape[1]
    ld, step = t.stride()
    if shape[1] > 1 and step != 1:
        raise ValueError(f"{name}: a row's elements must be adjacent")
    if shape[0] < 2:
        ld = shape[1]
    elif ld < shape[1]:
        raise ValueError(f"{name}: rows overlap")
    return t.data_ptr(), ld


def _whole(t, name, entries, kinds, like):
    """The address of a contiguous tensor of so many entries."""
    _gpu(t, name, kinds, like)
    if t.numel() != entries or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous and have {entries} entries")
    return t.data_ptr()


def _type_of(t):
    return 1 if t.dtype == torch.bfloat16 else 0


def _batch(tokens, tok_off, devices):
    """scadles_batch of the rows; None: all of them the first device's."""
    if tok_off is None:
        if devices != 1:
            raise ValueError(f"tok_off is needed for {devices} devices")
        return Batch(tokens, (_u64 * 2)(0, tokens), 1)
    if len(tok_off) != devices + 1:
        raise ValueError(f"tok_off must have {devices + 1} entries")
    off = [int(x) for x in tok_off]
    if min(off) < 0:
        raise ValueError("tok_off must not be negative")
    return Batch(tokens, (_u64 * (devices + 1))(*off), devices)


def _run(call, *args, like, stream):
    """A library call on the tensor's GPU, with the stream's address as its last argument."""
    gpu = like.get_device()
    if stream is None:
        p = torch._C._cuda_getCurrentRawStream(gpu)
    elif stream.device_index != gpu:
        raise ValueError(f"the stream must be one of cuda:{gpu}")
    else:
        p = stream.cuda_stream
    if torch.cuda.current_device() == gpu:
        return _sc._check(call(*args, p))
    with torch.cuda.device(gpu):
        _sc._check(call(*args, p))


def _new(shape, dtype, like, stream):
    """Uninitialised memory that belongs to the stream (the current one for None)."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    if stream.device_index != like.get_device():
        raise ValueError(f"the stream must be one of {like.device}")
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


def _scratch(size, like, stream):
    """A workspace of the call's: memory of its stream, which the allocator gives to
    others only behind the call there."""
    return _new((max(size, 256),), torch.uint8, like, stream)


def _output(t, name, rows, dim, kind, like, stream):
    """The tensor that a result goes to, new for None: (tensor, address, elements between rows)."""
    if t is None:
        t = _new((rows, dim), kind, like, stream)
        return t, t.data_ptr(), dim
    return (t,) + _rows(t, name, rows, dim, (kind,), like)


def _each(tensors, name, devices, shape, kinds, like):
    """(the tensors, their type, their addresses): one contiguous tensor of the shape for each
    device, as a list or as a tensor [devices, ...] (without that for one device)."""
    n = math.prod(shape)
    if isinstance(tensors, torch.Tensor):
        given = tuple(tensors.shape)
        if given == (devices,) + shape or (devices == 1 and given == shape):
            p, size = _whole(tensors, name, devices * n, kinds, like), n * tensors.element_size()
            return (tensors,), tensors.dtype, (_vp * devices)(*range(p, p + devices * size, size))
        each = list(tensors.unbind(0)) if tensors.dim() else []
    else:
        each = list(tensors)
    if len(each) != devices:
        raise ValueError(f"{name} must be a tensor of {list(shape)} for each of {devices} devices")
    at = [_whole(t, f"{name}[{i}]", n, kinds, like) for i, t in enumerate(each)]
    if any(t.dtype != each[0].dtype for t in each):
        raise TypeError(f"{name} must be of one type")
    return tuple(each), each[0].dtype, (_vp * devices)(*at)


def _wrote(*tensors):
    """Tells autograd that the caller's tensors have been written."""
    given = tuple(t for t in tensors if t is not None and not t.is_inference())
    if given:
        _sc._written(given)


# ---- tokens sorted by expert ----------------------------------------------------------------------------

@dataclass
class ExpertRows:
    """What ``ExpertOrder.sort`` returns (scadles_order_sort)."""
    pos: object          # int32 [T, k]: the row of each choice, -1 where there is none
    src: object          # int32 [T * k]: t * k + c of the choice in each row, -1 behind the last
    bounds: object       # int32 [experts * devices + 1]: first rows by expert and device


class ExpertOrder:
    """Tokens of K devices in the order of the experts that they go to, and back: what
    is needed between ``Router`` and the experts' products. Expert e's rows are
    ``bounds[e * devices]`` to ``bounds[(e + 1) * devices]``, those of device d among
    them ``bounds[e * devices + d]`` to ``bounds[e * devices + d + 1]``. Rows are
    float32 or bfloat16; there is room for all T * k of them, and those behind the last
    (as many as choices are missing) are left as they were."""

    def __init__(self, experts: int, k: int, *, devices: int = 1):
        self.experts, self.k, self.devices = int(experts), int(k), int(devices)
        if int(_order_ws_bytes(1, max(self.experts, 0), max(self.k, 0))) == 0 or not 1 <= self.devices <= _sc.MAX_DEVICES:
            raise _sc.ScadlesError(1, f"invalid experts={experts}, k={k} or devices={devices}")

    def sort(self, idx, *, tok_off=None, stream=None) -> ExpertRows:
        """``idx`` int32 [T, k] as ``Router.forward`` gives it (an index outside the
        experts is a missing choice); rows ``tok_off[d]`` to ``tok_off[d + 1]`` are those
        of device d."""
        _gpu(idx, "idx", _I32, None)
        if idx.dim() != 2 or idx.shape[1] != self.k or not idx.is_contiguous():
            raise ValueError(f"idx must be contiguous [tokens, {self.k}]")
        T, n, cells = idx.shape[0], idx.numel(), self.experts * self.devices + 1
        batch = _batch(T, tok_off, self.devices)
        need = _order_ws_bytes(T, self.experts, self.k)
        space = -(-need // 256) * 64               # the workspace before the results, in their memory
        buf = _new((space + 2 * n + cells,), torch.int32, idx, stream)
        _, pos, src, bounds = buf.split((space, n, n, cells))
        p = buf.data_ptr()
        q = p + 4 * space
        _run(_order_sort, batch, idx.data_ptr(), self.experts, self.k, q, q + 4 * n, q + 8 * n, p, need, like=idx, stream=stream)
        return ExpertRows(pos.view(T, self.k), src, bounds)

    def _shape(self, order, x, T):
        pos = order.pos
        if pos.device != x.device:
            raise ValueError(f"the order must be on {x.device}")
        if pos.dtype != torch.int32 or pos.shape != (T, self.k) or not pos.is_contiguous():
            raise ValueError(f"the order is not one of {T} tokens with {self.k} choices")
        return OrderShape(T, pos.data_ptr(), self.k, x.shape[1], _type_of(x))

    def dispatch(self, x, order: ExpertRows, *, out=None, stream=None):
        """The experts' input rows [T * k, dim]: row ``pos[t, c]`` is ``x[t]``."""
        p, ld = _rows(x, "x", None, None, _FLOATS)
        T, dim = x.shape
        shape = self._shape(order, x, T)
        rows, q, ld_rows = _output(out, "out", T * self.k, dim, x.dtype, x, stream)
        _run(_dispatch, shape, p, ld, q, ld_rows, like=x, stream=stream)
        _wrote(out)
        return rows

    def dispatch_backward(self, d_rows, order: ExpertRows, *, d_x=None, stream=None):
        """The gradient of ``x`` [T, dim]: the sum of its rows' gradients."""
        return self._combine(d_rows, "d_rows", None, order, d_x, "d_x", stream)

    def combine(self, rows, gate, order: ExpertRows, *, out=None, stream=None):
        """The tokens' sums [T, dim] of their experts' outputs ``rows`` [T * k, dim] times
        the gates, float32 [T, k]. Gates and rows of missing choices are not read."""
        _whole(gate, "gate", order.pos.numel(), _F32, rows)
        return self._combine(rows, "rows", gate.data_ptr(), order, out, "out", stream)

    def _combine(self, rows, name, gate, order, out, out_name, stream):
        T = order.pos.shape[0]
        p, ld = _rows(rows, name, T * self.k, None, _FLOATS)
        shape = self._shape(order, rows, T)
        sums, q, ld_out = _output(out, out_name, T, rows.shape[1], rows.dtype, rows, stream)
        _run(_combine, shape, p, ld, gate, q, ld_out, like=rows, stream=stream)
        _wrote(out)
        return sums

    def combine_backward(self, d_out, rows, gate, order: ExpertRows, *, d_rows=None, stream=None):
        """Gradients of ``rows`` [T * k, dim] (in ``d_rows`` if given, which may be ``rows``
        itself) and of the gates, float32 [T, k], 0 where a choice is missing."""
        T = order.pos.shape[0]
        p, ld = _rows(rows, "rows", T * self.k, None, _FLOATS)
        up, ld_up = _rows(d_out, "d_out", T, rows.shape[1], (rows.dtype,), rows)
        g = _whole(gate, "gate", T * self.k, _F32, rows)
        shape = self._shape(order, rows, T)
        to, q, ld_to = _output(d_rows, "d_rows", T * self.k, rows.shape[1], rows.dtype, rows, stream)
        d_gate = _new((T, self.k), torch.float32, rows, stream)
        _run(_combine_backward, shape, up, ld_up, p, ld, g, q, ld_to, d_gate.data_ptr(), like=rows, stream=stream)
        _wrote(d_rows)
        return to, d_gate


# ---- embedding ------------------------------------------------------------------------------------------

class Embedding:
    """Rows of a table [vocab, dim] by token, times ``scale``, and the table's gradients
    by sorted tokens, one for each device (scadles_embedding_forward, _backward). Tokens
    outside the vocabulary are padding: rows of zeros, without gradient."""

    def __init__(self, vocab: int, dim: int, *, scale: float = 1.0, devices: int = 1):
        self.vocab, self.dim, self.scale, self.devices = int(vocab), int(dim), float(scale), int(devices)
        if not 1 <= self.devices <= _sc.MAX_DEVICES or not 1 <= self.dim < 2**24 or not 1 <= self.vocab * self.devices < 2**32 - 1 \
                or not np.isfinite(np.float32(self.scale)):
            raise _sc.ScadlesError(1, f"invalid vocab={vocab}, dim={dim}, scale={scale} or devices={devices}")

    def _tokens(self, tokens, like):
        _gpu(tokens, "tokens", _INTEGERS, like)
        return _whole(tokens, "tokens", tokens.numel(), _INTEGERS, like)

    def _shape(self, tokens, x, grad=0):
        return EmbeddingShape(self.vocab, self.dim, _type_of(x), grad, tokens.element_size(), self.scale)

    def forward(self, tokens, weight, *, out=None, stream=None):
        """``tokens`` int32 or int64, contiguous, of any shape; ``weight`` [vocab, dim]
        float32 or bfloat16. Returns [tokens, dim] of the weight's type."""
        p, ld = _rows(weight, "weight", self.vocab, self.dim, _FLOATS)
        ids, T = self._tokens(tokens, weight), tokens.numel()
        rows, q, ld_out = _output(out, "out", T, self.dim, weight.dtype, weight, stream)
        _run(_embedding_forward, self._shape(tokens, weight), T, ids, p, ld, q, ld_out, like=weight, stream=stream)
        _wrote(out)
        return rows

    def backward(self, tokens, d_out, d_weight, *, tok_off=None, accumulate: bool = False, stream=None):
        """Writes the table's gradients under ``d_out`` [tokens, dim] into ``d_weight``: a
        contiguous tensor of vocab * dim elements for each device, float32 or bfloat16 (a
        part of its flat gradient will do, at any offset), or one tensor [devices, vocab,
        dim]. ``accumulate`` adds to what is there (a table that the logits use too). Tokens
        ``tok_off[d]`` to ``tok_off[d + 1]`` are device d's. Returns ``d_weight``."""
        p, ld = _rows(d_out, "d_out", None, self.dim, _FLOATS)
        T = d_out.shape[0]
        ids = self._tokens(tokens, d_out)
        if tokens.numel() != T:
            raise ValueError(f"tokens must have {T} entries")
        batch = _batch(T, tok_off, self.devices)
        each, kind, at = _each(d_weight, "d_weight", self.devices, (self.vocab, self.dim), _FLOATS, d_out)
        ws = _scratch(_embedding_ws_bytes(T, self.vocab, self.dim), d_out, stream)
        _run(_embedding_backward, self._shape(tokens, d_out, 1 if kind == torch.bfloat16 else 0), batch, ids, p, ld, at, int(bool(accumulate)),
             ws.data_ptr(), ws.numel(), like=d_out, stream=stream)
        _wrote(*each)
        return d_weight


# ---- layer norm -----------------------------------------------------------------------------------------

@dataclass
class LayerNormOutputs:
    """What ``LayerNorm.forward`` returns."""
    y: object            # [T, dim]
    mean: object         # float32 [T]
    rstd: object         # float32 [T]: 1 / sqrt(variance + eps)


class LayerNorm:
    """Layer norm over rows of ``dim`` elements, float32 or bfloat16, and its gradients,
    those of the weights one for each device (scadles_layer_norm_forward, _backward).
    Weight and bias are both float32 or both bfloat16."""

    def __init__(self, dim: int, *, eps: float = 1e-5, devices: int = 1):
        self.dim, self.eps, self.devices = int(dim), float(eps), int(devices)
        if not 1 <= self.dim < 2**24 or not 1 <= self.devices <= _sc.MAX_DEVICES or not 0 <= np.float32(self.eps) < np.inf:
            raise _sc.ScadlesError(1, f"invalid dim={dim}, eps={eps} or devices={devices}")

    def _shape(self, x, weight):
        return NormShape(self.dim, _type_of(x), _type_of(weight), self.eps)

    def forward(self, x, weight, bias=None, *, out=None, stream=None) -> LayerNormOutputs:
        """``x`` [T, dim]; ``y`` is of its type."""
        p, ld = _rows(x, "x", None, self.dim, _FLOATS)
        w = _whole(weight, "weight", self.dim, _FLOATS, x)
        b = None if bias is None else _whole(bias, "bias", self.dim, (weight.dtype,), x)
        T = x.shape[0]
        y, q, ld_y = _output(out, "out", T, self.dim, x.dtype, x, stream)
        both = _new((2, T), torch.float32, x, stream)
        m = both.data_ptr()
        _run(_layer_norm_forward, self._shape(x, weight), T, p, ld, w, b, q, ld_y, m, m + 4 * T, like=x, stream=stream)
        _wrote(out)
        return LayerNormOutputs(y, *both.unbind(0))

    def backward(self, x, weight, out: LayerNormOutputs, d_y, d_weight=None, d_bias=None, *, tok_off=None, d_x=None, stream=None):
        """The gradient of ``x`` [T, dim] (in ``d_x`` if given) under ``d_y``, and those of
        weight and bias into ``d_weight`` and ``d_bias``: a contiguous float32 tensor of
        dim elements for each device (a part of its flat gradient will do), or one tensor
        [devices, dim]; None where they are not wanted. ``out`` is the forward pass's
        (its mean and rstd are read); rows ``tok_off[d]`` to ``tok_off[d + 1]`` are device d's."""
        p, ld = _rows(x, "x", None, self.dim, _FLOATS)
        T = x.shape[0]
        w = _whole(weight, "weight", self.dim, _FLOATS, x)
        g, ld_g = _rows(d_y, "d_y", T, self.dim, (x.dtype,), x)
        mean, rstd = _whole(out.mean, "mean", T, _F32, x), _whole(out.rstd, "rstd", T, _F32, x)
        if tok_off is None and d_weight is None and d_bias is None:
            batch = _batch(T, None, 1)
        else:
            batch = _batch(T, tok_off, self.devices)
        given, at = (d_x,), []
        for t, name in ((d_weight, "d_weight"), (d_bias, "d_bias")):
            each, _, where = ((), None, None) if t is None else _each(t, name, self.devices, (self.dim,), _F32, x)
            given += each
            at.append(where)
        dx, q, ld_dx = _output(d_x, "d_x", T, self.dim, x.dtype, x, stream)
        ws = _scratch(_layer_norm_ws_bytes(T, self.dim), x, stream)
        _run(_layer_norm_backward, self._shape(x, weight), batch, p, ld, w, mean, rstd, g, ld_g, q, ld_dx, at[0], at[1],
             ws.data_ptr(), ws.numel(), like=x, stream=stream)
        _wrote(*given)
        return dx


# ---- cross entropy of a linear layer ----------------------------------------------------------------------

@dataclass
class CrossEntropyOutputs:
    """What ``LinearCrossEntropy.forward`` returns, all float32."""
    nll: object          # [T]: 0 where the target is outside the vocabulary
    lse: object          # [T]: log sum exp of the logits, 0 alike
    device_loss: object  # [devices]: mean of nll over the device's counted rows
    share: object        # [devices]: 1 / counted rows
    loss: object         # [1]: the devices' losses with their weights


class LinearCrossEntropy:
    """The cross entropy of a linear layer ``x @ weight.T`` over a vocabulary, without its
    logits being kept, and the gradients, those of the weight one for each device
    (scadles_cross_entropy_forward, _backward). ``x`` [T, dim] and ``weight`` [vocab, dim]
    are both float32 or both bfloat16; ``target`` int32 or int64 [T], outside the
    vocabulary for rows that are not counted."""

    def __init__(self, vocab: int, dim: int, *, devices: int = 1):
        self.vocab, self.dim, self.devices = int(vocab), int(dim), int(devices)
        if not 1 <= self.vocab <= 2**22 or not 1 <= self.dim <= 65536 or not 1 <= self.devices <= _sc.MAX_DEVICES:
            raise _sc.ScadlesError(1, f"invalid vocab={vocab}, dim={dim} or devices={devices}")

    def _arguments(self, x, weight, target, tok_off, grad):
        p, ld = _rows(x, "x", None, self.dim, _FLOATS)
        w, ld_w = _rows(weight, "weight", self.vocab, self.dim, (x.dtype,), x)
        T = x.shape[0]
        ids = _whole(target, "target", T, _INTEGERS, x)
        batch = _batch(T, tok_off, self.devices)
        return T, CrossEntropyShape(self.vocab, self.dim, _type_of(x), grad, target.element_size()), batch, (p, ld, w, ld_w, ids)

    def _weights(self, weights):
        if len(weights) != self.devices:
            raise ValueError(f"weights must have {self.devices} entries")
        return (ctypes.c_float * self.devices)(*[float(w) for w in weights])

    def forward(self, x, weight, target, *, tok_off=None, weights=None, stream=None) -> CrossEntropyOutputs:
        """Rows ``tok_off[d]`` to ``tok_off[d + 1]`` are device d's. ``weights``: Eqn 4a, by
        default the devices' shares of the rows."""
        T, shape, batch, args = self._arguments(x, weight, target, tok_off, 0)
        if weights is None:
            weights = [(batch.tok_off[d + 1] - batch.tok_off[d]) / T if T else 1.0 / self.devices for d in range(self.devices)]
        weights, K = self._weights(weights), self.devices
        buf = _new((2 * T + 2 * K + 1,), torch.float32, x, stream)
        q = buf.data_ptr()
        at = CrossEntropyOut(q, q + 4 * T, q + 8 * T, q + 8 * T + 4 * K, q + 8 * T + 8 * K)
        ws = _scratch(_cross_entropy_ws_bytes(shape, batch, 0), x, stream)
        _run(_cross_entropy_forward, shape, batch, weights, *args, at, ws.data_ptr(), ws.numel(), like=x, stream=stream)
        return CrossEntropyOutputs(*buf.split((T, T, K, K, 1)))

    def backward(self, x, weight, target, out: CrossEntropyOutputs, d_weight=None, *, tok_off=None, weights=None, d_loss=None, d_x=None,
                 stream=None):
        """The gradient of ``x`` [T, dim] (in ``d_x`` if given), and those of the weight into
        ``d_weight``: a contiguous tensor of vocab * dim elements for each device, float32
        or bfloat16 (a part of its flat gradient will do, at any offset), or one tensor
        [devices, vocab, dim]; None where they are not wanted. ``out`` is the forward
        pass's (its lse and share are read). ``weights``: by default ones, so that every
        device has the gradient of its own loss, before the aggregation weights it; the
        forward pass's give the gradient of its ``loss``. All of it times ``d_loss``, one
        float32 on the GPU, if given. With bfloat16 ``x`` and ``d_weight`` the softmax's part is
        rounded to bfloat16 before it is multiplied; float32 gradients keep it whole."""
        _gpu(x, "x", _FLOATS, None)
        each, kind, where = (), x.dtype, None
        if d_weight is not None:
            each, kind, where = _each(d_weight, "d_weight", self.devices, (self.vocab, self.dim), _FLOATS, x)
        T, shape, batch, args = self._arguments(x, weight, target, tok_off, 1 if kind == torch.bfloat16 else 0)
        lse, share = _whole(out.lse, "lse", T, _F32, x), _whole(out.share, "share", self.devices, _F32, x)
        d = None if d_loss is None else _whole(d_loss, "d_loss", 1, _F32, x)
        weights = None if weights is None else self._weights(weights)
        dx, q, ld_dx = _output(d_x, "d_x", T, self.dim, x.dtype, x, stream)
        ws = _scratch(_cross_entropy_ws_bytes(shape, batch, 1), x, stream)
        _run(_cross_entropy_backward, shape, batch, weights, *args,
             CrossEntropyOut(None, lse, None, share, None), d, q, ld_dx, where, ws.data_ptr(), ws.numel(), like=x, stream=stream)
        _wrote(d_x, *each)
        return dx
