"""What lies between tokens and logits of language models trained on K devices:
tokens sorted by expert and back, beside the router. Part of the package's
binding (``scadles.h``, "between tokens and logits"): checks of tensors and
marshalling.

The objects hold shapes only. Outputs, and scratch memory that a call needs, are
allocated for the call on its stream, so calls may be made on several streams, in
threads and in several captured graphs at once; what the caller does with a
tensor on other streams is the caller's to order. Outside autograd: outputs have no
history, and gradients are handed on with ``tensor.backward(gradient)``."""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

import numpy as np

import paper_2301_08897_amd as _sc

_vp, _u64, _u32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32


class Batch(ctypes.Structure):
    """scadles_batch: the rows of the devices."""
    _fields_ = [("tokens", _u64), ("tok_off", ctypes.POINTER(_u64)), ("devices", _u32)]


class OrderShape(ctypes.Structure):
    """scadles_order: the order that rows are moved by."""
    _fields_ = [("tokens", _u64), ("pos", _vp), ("k", _u32), ("dim", _u32), ("type", ctypes.c_int32)]


_order_ws_bytes = _sc._sig("scadles_order_workspace_bytes", ctypes.c_size_t, _u64, _u32, _u32)
_order_sort = _sc._sig("scadles_order_sort", ctypes.c_int, ctypes.POINTER(Batch), _vp, _u32, _u32, _vp, _vp, _vp, _vp,
                       ctypes.c_size_t, _vp)
_dispatch = _sc._sig("scadles_dispatch", ctypes.c_int, ctypes.POINTER(OrderShape), _vp, _u64, _vp, _u64, _vp)
_combine = _sc._sig("scadles_combine", ctypes.c_int, ctypes.POINTER(OrderShape), _vp, _u64, _vp, _vp, _u64, _vp)
_combine_backward = _sc._sig("scadles_combine_backward", ctypes.c_int, ctypes.POINTER(OrderShape), _vp, _u64, _vp, _u64,
                             _vp, _vp, _u64, _vp, _vp)


# ---- arguments --------------------------------------------------------------------------------------

def _gpu(t, name, *dtypes):
    torch = _sc._torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(str(d).removeprefix('torch.') for d in dtypes)}, not {t.dtype}")
    return t


def _rows(t, name, rows, dim, *dtypes, like=None):
    """(address, elements between rows) of a [rows, dim] tensor whose rows' elements
    are adjacent; any number of rows for None."""
    _gpu(t, name, *dtypes)
    if like is not None and t.device != like.device:
        raise ValueError(f"{name} must be on {like.device}")
    if t.dim() != 2 or t.shape[1] != dim or (rows is not None and t.shape[0] != rows):
        raise ValueError(f"{name} must be [{'rows' if rows is None else rows}, {dim}], not {list(t.shape)}")
    ld, step = t.stride()
    if dim > 1 and step != 1:
        raise ValueError(f"{name}: a row's elements must be adjacent")
    if t.shape[0] < 2:
        ld = dim
    elif ld < dim:
        raise ValueError(f"{name}: rows overlap")
    return t.data_ptr(), ld


def _whole(t, name, entries, *dtypes, like):
    """The address of a contiguous tensor of so many entries."""
    _gpu(t, name, *dtypes)
    if t.device != like.device:
        raise ValueError(f"{name} must be on {like.device}")
    if t.numel() != entries or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous and have {entries} entries")
    return t.data_ptr()


def _types():
    torch = _sc._torch()
    return torch.float32, torch.bfloat16


def _type_of(t):
    return 1 if t.dtype == _sc._torch().bfloat16 else 0


def _batch(tokens, tok_off, devices):
    """scadles_batch of the rows; None: all of them the first device's."""
    off = (_u64 * (devices + 1))()
    if tok_off is None:
        if devices != 1:
            raise ValueError(f"tok_off is needed for {devices} devices")
        off[1] = tokens
    else:
        if len(tok_off) != devices + 1:
            raise ValueError(f"tok_off must have {devices + 1} entries")
        for i, x in enumerate(tok_off):
            if x < 0:
                raise ValueError("tok_off must not be negative")
            off[i] = int(x)
    return Batch(tokens, off, devices)


def _stream_of(gpu, stream):
    if stream is None:
        return _sc._torch()._C._cuda_getCurrentRawStream(gpu)
    if stream.device_index != gpu:
        raise ValueError(f"the stream must be one of cuda:{gpu}")
    return stream.cuda_stream


def _run(call, *args, like, stream):
    """A library call on the tensor's GPU, with the stream's address as its last argument."""
    torch, gpu = _sc._torch(), like.device.index
    p = _stream_of(gpu, stream)
    if torch.cuda.current_device() == gpu:
        return _sc._check(call(*args, p))
    with torch.cuda.device(gpu):
        _sc._check(call(*args, p))


def _new(shape, dtype, like, stream):
    return _sc._empty(shape, dtype, like.device, stream)


def _scratch(size, like, stream):
    """A workspace of the call's: memory of its stream, which the allocator gives to
    others only behind the call there."""
    return _sc._empty((max(int(size), 256),), _sc._torch().uint8, like.device, stream)


def _output(t, name, rows, dim, dtype, like, stream):
    """The tensor that a result goes to, new for None: (tensor, address, elements between rows)."""
    if t is None:
        t = _new((rows, dim), dtype, like, stream)
        return t, t.data_ptr(), dim
    return (t,) + _rows(t, name, rows, dim, dtype, like=like)


def _wrote(*tensors):
    """Tells autograd that the caller's tensors have been written."""
    given = [t for t in tensors if t is not None and not t.is_inference()]
    if given:
        _sc._written(tuple(given))


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
        i32 = _sc._torch().int32
        _gpu(idx, "idx", i32)
        if idx.dim() != 2 or idx.shape[1] != self.k or not idx.is_contiguous():
            raise ValueError(f"idx must be contiguous [tokens, {self.k}]")
        T, n, cells = idx.shape[0], idx.numel(), self.experts * self.devices + 1
        batch = _batch(T, tok_off, self.devices)
        need = int(_order_ws_bytes(T, self.experts, self.k))
        buf = _new((2 * n + cells,), i32, idx, stream)
        pos, src, bounds = buf[:n].view(T, self.k), buf[n:2 * n], buf[2 * n:]
        ws = _scratch(need, idx, stream)
        p = buf.data_ptr()
        _run(_order_sort, batch, idx.data_ptr(), self.experts, self.k, p, p + 4 * n, p + 8 * n, ws.data_ptr(), ws.numel(),
             like=idx, stream=stream)
        return ExpertRows(pos, src, bounds)

    def _shape(self, order, x, T):
        pos = order.pos
        if pos.device != x.device:
            raise ValueError(f"the order must be on {x.device}")
        if pos.dtype != _sc._torch().int32 or tuple(pos.shape) != (T, self.k) or not pos.is_contiguous():
            raise ValueError(f"the order is not one of {T} tokens with {self.k} choices")
        return OrderShape(T, pos.data_ptr(), self.k, x.shape[1], _type_of(x))

    def dispatch(self, x, order: ExpertRows, *, out=None, stream=None):
        """The experts' input rows [T * k, dim]: row ``pos[t, c]`` is ``x[t]``."""
        p, ld = _rows(x, "x", None, x.shape[-1], *_types())
        T, dim = x.shape
        rows, q, ld_rows = _output(out, "out", T * self.k, dim, x.dtype, x, stream)
        _run(_dispatch, self._shape(order, x, T), p, ld, q, ld_rows, like=x, stream=stream)
        _wrote(out)
        return rows

    def dispatch_backward(self, d_rows, order: ExpertRows, *, d_x=None, stream=None):
        """The gradient of ``x`` [T, dim]: the sum of its rows' gradients."""
        return self._combine(d_rows, "d_rows", None, order, d_x, "d_x", stream)

    def combine(self, rows, gate, order: ExpertRows, *, out=None, stream=None):
        """The tokens' sums [T, dim] of their experts' outputs ``rows`` [T * k, dim] times
        the gates, float32 [T, k]. Gates and rows of missing choices are not read."""
        _whole(gate, "gate", order.pos.numel(), _types()[0], like=rows)
        return self._combine(rows, "rows", gate.data_ptr(), order, out, "out", stream)

    def _combine(self, rows, name, gate, order, out, out_name, stream):
        T = order.pos.shape[0]
        p, ld = _rows(rows, name, T * self.k, rows.shape[-1], *_types())
        sums, q, ld_out = _output(out, out_name, T, rows.shape[1], rows.dtype, rows, stream)
        _run(_combine, self._shape(order, rows, T), p, ld, gate, q, ld_out, like=rows, stream=stream)
        _wrote(out)
        return sums

    def combine_backward(self, d_out, rows, gate, order: ExpertRows, *, d_rows=None, stream=None):
        """Gradients of ``rows`` [T * k, dim] (in ``d_rows`` if given, which may be ``rows``
        itself) and of the gates, float32 [T, k], 0 where a choice is missing."""
        T, f32 = order.pos.shape[0], _types()[0]
        p, ld = _rows(rows, "rows", T * self.k, rows.shape[-1], *_types())
        up, ld_up = _rows(d_out, "d_out", T, rows.shape[1], rows.dtype, like=rows)
        g = _whole(gate, "gate", T * self.k, f32, like=rows)
        to, q, ld_to = _output(d_rows, "d_rows", T * self.k, rows.shape[1], rows.dtype, rows, stream)
        d_gate = _new((T, self.k), f32, rows, stream)
        _run(_combine_backward, self._shape(order, rows, T), up, ld_up, p, ld, g, q, ld_to, d_gate.data_ptr(), like=rows, stream=stream)
        _wrote(d_rows)
        return to, d_gate
