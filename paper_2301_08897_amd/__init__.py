"""ScaDLES hot path on MI355X: Top-k sparsification, streaming-rate-weighted
aggregation and SGD in hand-written HIP kernels for gfx950.

This package is a thin ctypes binding over ``libscadles.so`` (C ABI in
``include/scadles.h``). It only marshals arguments: every step runs in the HIP
kernels. PyTorch supplies device memory and the stream. Importing fails
loudly when the library has not been built (``__graft_entry__.build()``).
"""
from __future__ import annotations

import ctypes
import math
import os
import weakref
from dataclasses import dataclass
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libscadles.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() first "
                      "(there is no fallback implementation)")

# torch bundles its own HIP runtime under the same soname as the system one.
# Loading torch first makes libscadles bind to that runtime, so the process has
# exactly one HIP/HSA runtime (two would each try to own the GPU).
import torch as _torch_for_runtime  # noqa: E402,F401

_lib = ctypes.CDLL(LIB_PATH)

MAX_DEVICES = 64
MOMENT_BLOCK = 256                     # SCADLES_MOMENT_BLOCK
ROUTER_MAX_EXPERTS, ROUTER_MAX_K = 1024, 16
NOALLOC_SCRATCH_BYTES = 128 << 20      # SCADLES_NOALLOC_SCRATCH_BYTES
PROFILE_STAGES = 5
STAGE_NAMES = ("bracket", "main_select", "post_select", "aggregate", "total")

_vp = ctypes.c_void_p
_u64 = ctypes.c_uint64
_u32 = ctypes.c_uint32


class Sparse(ctypes.Structure):
    _fields_ = [("idx", _vp), ("val", _vp), ("k", _u64)]


class StepOptions(ctypes.Structure):
    """scadles_step_options (momentum SGD, moving-average adaptive rule, accounting)."""
    _fields_ = [("momentum_buf", _vp), ("momentum", ctypes.c_float), ("weight_decay", ctypes.c_float),
                ("ewma", _vp), ("ewma_beta", ctypes.c_double), ("counters", _vp)]


class Stream(ctypes.Structure):
    """scadles_stream: one device's stream buffer."""
    _fields_ = [("rate", _u64), ("elapsed_us", _u64), ("queued", _u64), ("trained", _u64), ("dropped", _u64)]


class AdamWTensor(ctypes.Structure):
    """scadles_adamw_tensor: one tensor of an AdamW plan."""
    _fields_ = [("param", _vp), ("grad", _vp), ("m", _vp), ("v", _vp), ("tops", _vp), ("copy", _vp), ("n", _u64),
                ("weight_decay", ctypes.c_float)]


class AdamWPlan(ctypes.Structure):
    """scadles_adamw_plan: the handle of a plan (its fields are the library's)."""
    _fields_ = [("table", _vp), ("chunks_at", _u64), ("chunks", _u64), ("n", _u64), ("moment_bits", _u32),
                ("grad_type", _u32), ("magic", _u32), ("reserved", _u32)]


class AdamWOptions(ctypes.Structure):
    """scadles_adamw_options: a step's hyperparameters and its number."""
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", _u64)]


class RouterShape(ctypes.Structure):
    """scadles_router: the shape of a router call."""
    _fields_ = [("tokens", _u64), ("ld", _u64), ("tok_off", ctypes.POINTER(_u64)),
                ("weights", ctypes.POINTER(ctypes.c_float)), ("experts", _u32), ("k", _u32), ("devices", _u32),
                ("logits_type", ctypes.c_int32), ("renormalise", ctypes.c_int32)]


class RouterOut(ctypes.Structure):
    """scadles_router_out: what the router's forward pass writes."""
    _fields_ = [("idx", _vp), ("gate", _vp), ("lse", _vp), ("counts", _vp), ("load", _vp), ("share", _vp),
                ("loss", _vp)]


def _sig(name, restype, *argtypes):
    f = getattr(_lib, name)
    f.restype = restype
    f.argtypes = list(argtypes)
    return f


_topk_k = _sig("scadles_topk_k", _u64, _u64, ctypes.c_double)
_ws_bytes = _sig("scadles_workspace_bytes", ctypes.c_size_t, _u32, _u64, ctypes.POINTER(ctypes.c_double))
_agg_ws_bytes = _sig("scadles_aggregate_workspace_bytes", ctypes.c_size_t, _u32, _u64)
_topk_select = _sig("scadles_topk_select", ctypes.c_int, _vp, _u64, ctypes.c_double, _vp, _vp, _vp, _vp,
                    ctypes.c_size_t, _vp)
_topk_select_noalloc = _sig("scadles_topk_select_noalloc", ctypes.c_int, _vp, _u64, ctypes.c_double, _vp, _vp,
                            _vp, _vp)
_layers_k = _sig("scadles_layers_k", _u64, ctypes.POINTER(_u64), _u32, ctypes.c_double)
_layers_ws_bytes = _sig("scadles_layers_workspace_bytes", ctypes.c_size_t, _u32, ctypes.POINTER(_u64), _u32,
                        ctypes.POINTER(ctypes.c_double))
_topk_select_layers = _sig("scadles_topk_select_layers", ctypes.c_int, ctypes.POINTER(_vp), _u32,
                           ctypes.POINTER(_u64), _u32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_vp),
                           ctypes.POINTER(_vp), _vp, _vp, ctypes.c_size_t, _vp)
_weighted_aggregate = _sig("scadles_weighted_aggregate", ctypes.c_int, ctypes.POINTER(Sparse),
                           ctypes.POINTER(ctypes.c_float), _u32, _u64, _vp, _vp, ctypes.c_size_t, _vp)
_apply_sgd = _sig("scadles_apply_sgd", ctypes.c_int, _vp, _vp, _u64, ctypes.c_float, _vp)
_apply_momentum_sgd = _sig("scadles_apply_momentum_sgd", ctypes.c_int, _vp, _vp, _vp, _u64, ctypes.c_float,
                           ctypes.c_float, ctypes.c_float, _vp)
_step_fused = _sig("scadles_step_fused", ctypes.c_int, ctypes.POINTER(_vp), _u32, _u64,
                   ctypes.POINTER(ctypes.c_double), ctypes.c_double, ctypes.POINTER(ctypes.c_float),
                   ctypes.POINTER(_vp), ctypes.POINTER(_vp), _vp, _vp, _vp, _vp, ctypes.c_float, _vp,
                   ctypes.c_size_t, _vp)
_step_fused_ex = _sig("scadles_step_fused_ex", ctypes.c_int, ctypes.POINTER(_vp), _u32, _u64,
                      ctypes.POINTER(ctypes.c_double), ctypes.c_double, ctypes.POINTER(ctypes.c_float),
                      ctypes.POINTER(_vp), ctypes.POINTER(_vp), _vp, _vp, _vp, _vp, ctypes.c_float,
                      ctypes.POINTER(StepOptions), _vp, ctypes.c_size_t, _vp)
_stream_weights = _sig("scadles_stream_weights", ctypes.c_int, ctypes.POINTER(ctypes.c_double), _u32,
                       ctypes.c_double, ctypes.c_double, ctypes.c_double, ctypes.POINTER(ctypes.c_float),
                       ctypes.POINTER(ctypes.c_double))
_step_layers_ws_bytes = _sig("scadles_step_layers_workspace_bytes", ctypes.c_size_t, _u32, ctypes.POINTER(_u64),
                             _u32, ctypes.POINTER(ctypes.c_double))
_step_fused_layers = _sig("scadles_step_fused_layers", ctypes.c_int, ctypes.POINTER(_vp), _u32, ctypes.POINTER(_u64),
                          _u32, ctypes.POINTER(ctypes.c_double), ctypes.c_double, ctypes.POINTER(ctypes.c_float),
                          ctypes.POINTER(_vp), ctypes.POINTER(_vp), _vp, _vp, _vp, _vp, ctypes.c_float,
                          ctypes.POINTER(StepOptions), _vp, ctypes.c_size_t, _vp)
_stream_init = _sig("scadles_stream_init", ctypes.c_int, _u32, ctypes.POINTER(_u64), ctypes.POINTER(Stream))
_stream_iteration = _sig("scadles_stream_iteration", ctypes.c_int, _u32, ctypes.POINTER(Stream), ctypes.POINTER(_u64),
                         _u64, _u64, ctypes.c_int, ctypes.c_double, ctypes.POINTER(_u64),
                         ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_double))
_stream_simulate = _sig("scadles_stream_simulate", ctypes.c_int, _u32, ctypes.POINTER(_u64), ctypes.POINTER(_u64), _u64,
                        _u64, ctypes.c_int, _u64, ctypes.POINTER(_u64), ctypes.POINTER(_u64), ctypes.POINTER(_u64))
_adamw_plan_bytes = _sig("scadles_adamw_plan_bytes", ctypes.c_size_t, ctypes.POINTER(AdamWTensor), _u32)
_adamw_plan_build = _sig("scadles_adamw_plan_build", ctypes.c_int, ctypes.POINTER(AdamWTensor), _u32, ctypes.c_int,
                         ctypes.c_int, _vp, ctypes.c_size_t, ctypes.POINTER(AdamWPlan), _vp)
_grad_norm = _sig("scadles_grad_norm", ctypes.c_int, ctypes.POINTER(AdamWPlan), ctypes.c_double, _vp, _vp)
_adamw_step = _sig("scadles_adamw_step", ctypes.c_int, ctypes.POINTER(AdamWPlan), ctypes.POINTER(AdamWOptions), _vp,
                   _vp)
_adamw_get_moments = _sig("scadles_adamw_get_moments", ctypes.c_int, ctypes.POINTER(AdamWPlan), _vp, _vp, _vp)
_adamw_set_moments = _sig("scadles_adamw_set_moments", ctypes.c_int, ctypes.POINTER(AdamWPlan), _vp, _vp, _u64, _vp)
_router_ws_bytes = _sig("scadles_router_workspace_bytes", ctypes.c_size_t, _u64, _u32, _u32)
_router_forward = _sig("scadles_router_forward", ctypes.c_int, ctypes.POINTER(RouterShape), _vp, _vp,
                       ctypes.POINTER(RouterOut), _vp, ctypes.c_size_t, _vp)
_router_backward = _sig("scadles_router_backward", ctypes.c_int, ctypes.POINTER(RouterShape), _vp,
                        ctypes.POINTER(RouterOut), _vp, _vp, _vp, _u64, _vp)
_last_error = _sig("scadles_last_error", ctypes.c_char_p)
_set_option = _sig("scadles_set_option", ctypes.c_int, ctypes.c_char_p, ctypes.c_int64)
_profile_enable = _sig("scadles_profile_enable", ctypes.c_int, ctypes.c_int)
_profile_read = _sig("scadles_profile_read", ctypes.c_int, ctypes.POINTER(ctypes.c_double),
                     ctypes.POINTER(_u32))

STATUS = {0: "SCADLES_OK", 1: "SCADLES_EINVAL", 2: "SCADLES_EWORKSPACE", 3: "SCADLES_EHIP",
          4: "SCADLES_EUNSORTED", 5: "SCADLES_EINTERNAL"}


class ScadlesError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{STATUS.get(code, code)}: {msg}")
        self.code = code


def _check(code: int):
    if code != 0:
        raise ScadlesError(code, _last_error().decode(errors="replace"))


def _torch():
    import torch
    return torch


def _stream_ptr(stream) -> Optional[int]:
    torch = _torch()
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _dev_f32(t, name, device=None):
    torch = _torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype != torch.float32 or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous float32 tensor")
    if device is not None and t.device != device:
        raise ValueError(f"{name} must be on {device}")
    return t.data_ptr()


def library_path() -> str:
    return LIB_PATH


# ---- host-side rules ----------------------------------------------------------------------

def topk_k(n: int, ratio: float) -> int:
    """k = clamp(floor(ratio * n), 1, n) (0 for invalid input)."""
    return int(_topk_k(int(n), float(ratio)))


def workspace_bytes(K: int, n: int, ratios: Sequence[float]) -> int:
    r = (ctypes.c_double * K)(*[float(x) for x in ratios])
    return int(_ws_bytes(K, int(n), r))


def _seg_array(seg_off):
    off = [int(x) for x in seg_off]
    return (_u64 * len(off))(*off), len(off) - 1


def layers_k(seg_off: Sequence[int], ratio: float) -> int:
    """Entries kept by the per-layer Top-k over layers [seg_off[l], seg_off[l+1])
    (0 for invalid input)."""
    arr, L = _seg_array(seg_off)
    return int(_layers_k(arr, max(L, 0), float(ratio))) if L >= 1 else 0


def layers_workspace_bytes(K: int, seg_off: Sequence[int], ratios: Sequence[float]) -> int:
    arr, L = _seg_array(seg_off)
    r = (ctypes.c_double * K)(*[float(x) for x in ratios])
    return int(_layers_ws_bytes(K, arr, L, r)) if L >= 1 else 0


def aggregate_workspace_bytes(K: int, n: int) -> int:
    return int(_agg_ws_bytes(K, int(n)))


def stream_weights(rates, b_min: float = 0.0, b_max: float = math.inf, base_batch: Optional[float] = None):
    """Eqn 4a weights (float32[K]) and, if base_batch is given, the linear-scaling gamma."""
    r = np.ascontiguousarray(rates, dtype=np.float64)
    K = r.size
    w = np.empty(K, dtype=np.float32)
    g = ctypes.c_double()
    _check(_stream_weights(r.ctypes.data_as(ctypes.POINTER(ctypes.c_double)), K, float(b_min), float(b_max),
                           float(base_batch) if base_batch is not None else 0.0,
                           w.ctypes.data_as(ctypes.POINTER(ctypes.c_float)),
                           ctypes.byref(g) if base_batch is not None else None))
    return (w, g.value) if base_batch is not None else (w, None)


PERSISTENCE, TRUNCATION = 0, 1
NO_BOUND = 2**64 - 1
_POLICIES = {"persistence": PERSISTENCE, "truncation": TRUNCATION, PERSISTENCE: PERSISTENCE,
             TRUNCATION: TRUNCATION}


def _u64_array(x, n=None):
    a = np.ascontiguousarray(x, dtype=np.uint64)
    if n is not None and a.size != n:
        raise ValueError(f"expected {n} values")
    return a


def _p64(a):
    return a.ctypes.data_as(ctypes.POINTER(_u64))


class StreamBuffers:
    """The stream buffers of K devices (persistence or truncation) and, per
    training iteration, the batch each device trains on with the Eqn 4a
    weights and learning-rate scale that follow from them. Host only."""

    def __init__(self, rates, *, b_min: int = 0, b_max: int = NO_BOUND, policy="persistence",
                 base_batch: Optional[float] = None):
        r = _u64_array(rates)
        self.K = r.size
        self.b_min, self.b_max = int(b_min), int(b_max)
        self.policy = _POLICIES[policy]
        self.base_batch = base_batch
        self.state = (Stream * self.K)()
        _check(_stream_init(self.K, _p64(r), self.state))

    def iteration(self, iter_us):
        """One iteration of iter_us microseconds per device (scalar or per device).
        Returns (batch uint64[K], weights float32[K], gamma or None)."""
        t = _u64_array(np.broadcast_to(np.asarray(iter_us, dtype=np.uint64), (self.K,)), self.K)
        batch = np.empty(self.K, dtype=np.uint64)
        w = np.empty(self.K, dtype=np.float32)
        g = ctypes.c_double()
        _check(_stream_iteration(self.K, self.state, _p64(t), self.b_min, self.b_max, self.policy,
                                 float(self.base_batch) if self.base_batch is not None else 0.0, _p64(batch),
                                 w.ctypes.data_as(ctypes.POINTER(ctypes.c_float)),
                                 ctypes.byref(g) if self.base_batch is not None else None))
        return batch, w, (g.value if self.base_batch is not None else None)

    def field(self, name: str) -> np.ndarray:
        return np.array([getattr(s, name) for s in self.state], dtype=np.uint64)


def stream_simulate(rates, iter_us, b_min: int, b_max: int, policy, T: int):
    """T iterations from fresh buffers: (queued uint64[T+1, K], batch uint64[T, K], dropped uint64[K])."""
    r = _u64_array(rates)
    K = r.size
    t = _u64_array(iter_us, K)
    queued = np.empty((T + 1, K), dtype=np.uint64)
    batch = np.empty((max(T, 1), K), dtype=np.uint64)
    dropped = np.empty(K, dtype=np.uint64)
    _check(_stream_simulate(K, _p64(r), _p64(t), int(b_min), int(b_max), _POLICIES[policy], int(T), _p64(queued),
                            _p64(batch), _p64(dropped)))
    return queued, batch[:T], dropped


def set_option(name: str, value: int):
    _check(_set_option(name.encode(), int(value)))


def profile_enable(on: bool = True):
    _check(_profile_enable(1 if on else 0))


def profile_read():
    """(dict stage -> summed ms, number of calls) since the last read; syncs the events."""
    ms = (ctypes.c_double * PROFILE_STAGES)()
    calls = _u32()
    _check(_profile_read(ms, ctypes.byref(calls)))
    return dict(zip(STAGE_NAMES, list(ms))), int(calls.value)


def _workspace(nbytes: int, device):
    torch = _torch()
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


# ---- the three calls of the hot path -----------------------------------------------------------

def topk_select(grad, ratio: float, *, workspace=None, energies: bool = False, stream=None):
    """Top-k of one gradient. Returns (idx uint32[k], val float32[k]) or, with
    energies=True, (idx, val, float64[2] = (sum g^2, sum kept g^2))."""
    torch = _torch()
    gp = _dev_f32(grad, "grad")
    n = grad.numel()
    k = topk_k(n, ratio)
    if k == 0:
        raise ScadlesError(1, f"invalid n={n} or ratio={ratio}")
    dev = grad.device
    idx = torch.empty(k, dtype=torch.uint32, device=dev)
    val = torch.empty(k, dtype=torch.float32, device=dev)
    en = torch.empty(2, dtype=torch.float64, device=dev) if energies else None
    need = workspace_bytes(1, n, [ratio])
    ws = workspace if workspace is not None else _workspace(need, dev)
    _check(_topk_select(gp, n, float(ratio), idx.data_ptr(), val.data_ptr(),
                        en.data_ptr() if en is not None else None, ws.data_ptr(), ws.numel(),
                        _stream_ptr(stream)))
    return (idx, val, en) if energies else (idx, val)


def topk_select_noalloc(grad, ratio: float, idx, val, energies=None, *, stream=None):
    """Top-k of one gradient into caller-given outputs (idx uint32[k], val
    float32[k], energies float64[2] or None) using the library's static
    scratch: the call allocates nothing (scadles_topk_select_noalloc)."""
    torch = _torch()
    gp = _dev_f32(grad, "grad")
    n = grad.numel()
    k = topk_k(n, ratio)
    if k == 0:
        raise ScadlesError(1, f"invalid n={n} or ratio={ratio}")
    if idx.numel() < k or val.numel() < k or not idx.is_cuda or not idx.is_contiguous():
        raise ValueError(f"idx and val must be contiguous GPU tensors of at least k={k} entries")
    if idx.dtype not in (torch.uint32, torch.int32):
        raise TypeError("idx must be uint32")
    if energies is not None and (energies.dtype != torch.float64 or energies.numel() < 2 or not energies.is_cuda):
        raise TypeError("energies must be a float64 GPU tensor of 2 entries")
    _check(_topk_select_noalloc(gp, n, float(ratio), idx.data_ptr(), _dev_f32(val, "val"),
                                energies.data_ptr() if energies is not None else None, _stream_ptr(stream)))
    return idx, val, energies


def weighted_aggregate(sets, weights, n: int, *, out=None, workspace=None, stream=None):
    """Eqn 4b. ``sets``: list of (idx uint32 tensor or None for dense, val float32 tensor)."""
    torch = _torch()
    K = len(sets)
    w = np.ascontiguousarray(weights, dtype=np.float32)
    if w.size != K:
        raise ValueError("one weight per set")
    arr = (Sparse * K)()
    dev = None
    for j, (idx, val) in enumerate(sets):
        vp = _dev_f32(val, f"sets[{j}].val")
        dev = val.device
        if idx is None:
            arr[j] = Sparse(None, vp, val.numel())
        else:
            if idx.dtype not in (torch.uint32, torch.int32) or not idx.is_cuda or not idx.is_contiguous():
                raise TypeError(f"sets[{j}].idx must be a contiguous uint32 GPU tensor")
            if idx.numel() != val.numel():
                raise ValueError(f"sets[{j}]: idx and val differ in length")
            arr[j] = Sparse(idx.data_ptr(), vp, idx.numel())
    if out is None:
        out = torch.empty(n, dtype=torch.float32, device=dev)
    ws = workspace if workspace is not None else _workspace(aggregate_workspace_bytes(K, n), dev)
    _check(_weighted_aggregate(arr, w.ctypes.data_as(ctypes.POINTER(ctypes.c_float)), K, int(n),
                               _dev_f32(out, "out"), ws.data_ptr(), ws.numel(), _stream_ptr(stream)))
    return out


def apply_sgd(params, grad, lr: float, *, stream=None):
    """Eqn 4c in place on ``params``."""
    _check(_apply_sgd(_dev_f32(params, "params"), _dev_f32(grad, "grad"), params.numel(), float(lr),
                      _stream_ptr(stream)))
    return params


def apply_momentum_sgd(params, momentum_buf, grad, lr: float, momentum: float, weight_decay: float, *,
                       stream=None):
    """Momentum SGD with weight decay (§V training setup) in place on ``params``
    and ``momentum_buf``."""
    if not (params.numel() == momentum_buf.numel() == grad.numel()):
        raise ValueError("params, momentum_buf and grad must have the same size")
    _check(_apply_momentum_sgd(_dev_f32(params, "params"), _dev_f32(momentum_buf, "momentum_buf"),
                               _dev_f32(grad, "grad"), params.numel(), float(lr), float(momentum),
                               float(weight_decay), _stream_ptr(stream)))
    return params, momentum_buf


class LayerSelect:
    """Per-layer Top-k of K gradients that share one layer layout (every layer
    keeps its own top fraction): outputs and workspace allocated once, ``run``
    only marshals pointers. ``seg_off`` = [0, ..., n] are the layer bounds."""

    def __init__(self, grads, seg_off: Sequence[int], ratios: Sequence[float]):
        torch = _torch()
        if isinstance(grads, torch.Tensor) and grads.dim() == 2:
            grads = [grads[j] for j in range(grads.shape[0])]
        self.grads = list(grads)
        self.K = len(self.grads)
        if not 1 <= self.K <= MAX_DEVICES:
            raise ValueError(f"K must be in [1, {MAX_DEVICES}]")
        self.seg_off = [int(x) for x in seg_off]
        self.n = self.seg_off[-1] if self.seg_off else 0
        for j, g in enumerate(self.grads):
            _dev_f32(g, f"grads[{j}]")
            if g.numel() != self.n:
                raise ValueError("every gradient must have seg_off[-1] elements")
        self.ratios = [float(r) for r in ratios]
        if len(self.ratios) != self.K:
            raise ValueError("one ratio per device")
        self.k = [layers_k(self.seg_off, r) for r in self.ratios]
        if min(self.k) == 0:
            raise ScadlesError(1, "invalid layer bounds or ratio")
        dev = self.grads[0].device
        self.idx = [torch.empty(k, dtype=torch.uint32, device=dev) for k in self.k]
        self.val = [torch.empty(k, dtype=torch.float32, device=dev) for k in self.k]
        self.energies = torch.empty(2 * self.K, dtype=torch.float64, device=dev)
        self.ws = _workspace(layers_workspace_bytes(self.K, self.seg_off, self.ratios), dev)
        self._seg, self._L = _seg_array(self.seg_off)
        self._ratios = (ctypes.c_double * self.K)(*self.ratios)
        self._grad_ptrs = (_vp * self.K)(*[g.data_ptr() for g in self.grads])
        self._idx_ptrs = (_vp * self.K)(*[t.data_ptr() for t in self.idx])
        self._val_ptrs = (_vp * self.K)(*[t.data_ptr() for t in self.val])

    def run(self, *, stream=None):
        """Select every device's kept set; returns (idx list, val list, energies float64[2K])."""
        _check(_topk_select_layers(self._grad_ptrs, self.K, self._seg, self._L, self._ratios, self._idx_ptrs,
                                   self._val_ptrs, self.energies.data_ptr(), self.ws.data_ptr(), self.ws.numel(),
                                   _stream_ptr(stream)))
        return self.idx, self.val, self.energies


# ---- the fused step -----------------------------------------------------------------------------

@dataclass
class StepOutputs:
    idx: list
    val: list
    dense: object
    energies: object
    compressed: object


class FusedStep:
    """One hot-path step for K devices of n elements (Top-k + energies + adaptive
    rule + Eqn 4b aggregation + optional Eqn 4c update), with every output and
    the workspace allocated once so that ``run`` only marshals pointers."""

    def __init__(self, grads, ratios: Sequence[float], *, delta: float = math.inf, params=None,
                 momentum_buf=None, momentum: float = 0.0, weight_decay: float = 0.0,
                 ewma_beta: Optional[float] = None, track: bool = False, seg_off: Optional[Sequence[int]] = None):
        torch = _torch()
        if isinstance(grads, torch.Tensor) and grads.dim() == 2:
            grads = [grads[j] for j in range(grads.shape[0])]
        self.K = len(grads)
        if not 1 <= self.K <= MAX_DEVICES:
            raise ValueError(f"K must be in [1, {MAX_DEVICES}]")
        self.n = grads[0].numel()
        # per-layer Top-k over layers [seg_off[l], seg_off[l+1]) when given
        self.seg_off = None if seg_off is None else [int(x) for x in seg_off]
        if self.seg_off is not None:
            if len(self.seg_off) < 2 or self.seg_off[-1] != self.n:
                raise ValueError("seg_off must run from 0 to the gradients' size")
            self._seg, self._L = _seg_array(self.seg_off)
        self.grads = list(grads)
        for j, g in enumerate(self.grads):
            _dev_f32(g, f"grads[{j}]")
            if g.numel() != self.n:
                raise ValueError("all gradients must have n elements")
        dev = self.grads[0].device
        self.device = dev
        self.params = params
        # momentum SGD with weight decay in place of Eqn 4c when a buffer is given
        self.momentum_buf = momentum_buf
        self.momentum = float(momentum)
        self.weight_decay = float(weight_decay)
        if momentum_buf is not None:
            if params is None:
                raise ValueError("momentum_buf needs params")
            _dev_f32(momentum_buf, "momentum_buf")
            if momentum_buf.numel() != self.n or params.numel() != self.n:
                raise ValueError("params and momentum_buf must have n elements")
        self.delta = float(delta)
        self.set_ratios(ratios)
        # §IV moving average of the energies (state zero-filled: no history) and
        # §V-G accounting, both kept on the device across run() calls
        self.ewma_beta = None if ewma_beta is None else float(ewma_beta)
        self.ewma = (torch.zeros(2 * self.K, dtype=torch.float64, device=dev)
                     if ewma_beta is not None else None)
        self.counters = torch.zeros(3 * self.K, dtype=torch.int64, device=dev) if track else None
        self._opts = StepOptions(
            momentum_buf.data_ptr() if momentum_buf is not None else None, self.momentum, self.weight_decay,
            self.ewma.data_ptr() if self.ewma is not None else None,
            self.ewma_beta if self.ewma_beta is not None else 0.0,
            self.counters.data_ptr() if self.counters is not None else None)
        self.dense = torch.empty(self.n, dtype=torch.float32, device=dev)
        self.energies = torch.empty(2 * self.K, dtype=torch.float64, device=dev)
        self.compressed = torch.empty(self.K, dtype=torch.uint8, device=dev)
        self._grad_ptrs = (_vp * self.K)(*[g.data_ptr() for g in self.grads])
        self._w = (ctypes.c_float * self.K)()

    def set_grads(self, grads):
        """Point the step at other gradients of the same shape (marshalling only)."""
        torch = _torch()
        if isinstance(grads, torch.Tensor) and grads.dim() == 2:
            grads = [grads[j] for j in range(grads.shape[0])]
        if len(grads) != self.K:
            raise ValueError("one gradient per device")
        for j, g in enumerate(grads):
            _dev_f32(g, f"grads[{j}]")
            if g.numel() != self.n:
                raise ValueError("all gradients must have n elements")
        self.grads = list(grads)
        self._grad_ptrs = (_vp * self.K)(*[g.data_ptr() for g in self.grads])

    def set_ratios(self, ratios):
        torch = _torch()
        ratios = [float(r) for r in ratios]
        if len(ratios) != self.K:
            raise ValueError("one ratio per device")
        self.ratios = ratios
        if self.seg_off is not None:
            self.k = [layers_k(self.seg_off, r) for r in ratios]
        else:
            self.k = [topk_k(self.n, r) for r in ratios]
        if min(self.k) == 0:
            raise ScadlesError(1, "ratio outside (0, 1]")
        self.idx = [torch.empty(k, dtype=torch.uint32, device=self.device) for k in self.k]
        self.val = [torch.empty(k, dtype=torch.float32, device=self.device) for k in self.k]
        self._ratios = (ctypes.c_double * self.K)(*ratios)
        self._idx_ptrs = (_vp * self.K)(*[t.data_ptr() for t in self.idx])
        self._val_ptrs = (_vp * self.K)(*[t.data_ptr() for t in self.val])
        if self.seg_off is not None:
            need = int(_step_layers_ws_bytes(self.K, self._seg, self._L, self._ratios))
        else:
            need = workspace_bytes(self.K, self.n, ratios)
        if need == 0:
            raise ScadlesError(1, "workspace query rejected the arguments")
        if getattr(self, "ws", None) is None or self.ws.numel() < need:
            self.ws = _workspace(need, self.device)

    def run(self, weights, lr: float = 0.0, *, stream=None) -> StepOutputs:
        w = np.ascontiguousarray(weights, dtype=np.float32)
        for j in range(self.K):
            self._w[j] = float(w[j])
        pp = _dev_f32(self.params, "params") if self.params is not None else None
        opts = self.momentum_buf is not None or self.ewma is not None or self.counters is not None
        if self.seg_off is not None:
            _check(_step_fused_layers(self._grad_ptrs, self.K, self._seg, self._L, self._ratios, self.delta, self._w,
                                      self._idx_ptrs, self._val_ptrs, self.dense.data_ptr(),
                                      self.energies.data_ptr(), self.compressed.data_ptr(), pp, float(lr),
                                      ctypes.byref(self._opts) if opts else None, self.ws.data_ptr(),
                                      self.ws.numel(), _stream_ptr(stream)))
        elif opts:
            _check(_step_fused_ex(self._grad_ptrs, self.K, self.n, self._ratios, self.delta, self._w,
                                  self._idx_ptrs, self._val_ptrs, self.dense.data_ptr(), self.energies.data_ptr(),
                                  self.compressed.data_ptr(), pp, float(lr), ctypes.byref(self._opts),
                                  self.ws.data_ptr(), self.ws.numel(), _stream_ptr(stream)))
        else:
            _check(_step_fused(self._grad_ptrs, self.K, self.n, self._ratios, self.delta, self._w,
                               self._idx_ptrs, self._val_ptrs, self.dense.data_ptr(), self.energies.data_ptr(),
                               self.compressed.data_ptr(), pp, float(lr), self.ws.data_ptr(), self.ws.numel(),
                               _stream_ptr(stream)))
        return StepOutputs(self.idx, self.val, self.dense, self.energies, self.compressed)

    def accounting(self):
        """The counters of ``track=True`` as uint64[K, 3]: per device the iterations
        that sent Top-k, the iterations, and the floats sent (§V-G)."""
        if self.counters is None:
            raise ValueError("construct with track=True")
        return self.counters.cpu().numpy().reshape(self.K, 3).astype(np.uint64)


def step_fused(grads, ratios, weights, *, delta: float = math.inf, params=None, lr: float = 0.0,
               stream=None) -> StepOutputs:
    """One-shot convenience wrapper around FusedStep."""
    return FusedStep(grads, ratios, delta=delta, params=params).run(weights, lr, stream=stream)


# ---- AdamW ----------------------------------------------------------------------------------------

def _empty(shape, dtype, device, stream):
    """Uninitialised memory that belongs to the stream (the current one for None)."""
    torch = _torch()
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _wholes(tensors):
    """The tensors that these are, or are parts of: parts share their version counter."""
    return tuple({id(x): x for x in (t if t._base is None else t._base for t in tensors)}.values())


def _written(tensors):
    """Tells autograd, by their version counters, that the library has written the tensors."""
    _torch().autograd.graph.increment_version(tensors)


def _capturing(stream):
    torch = _torch()
    if stream.cuda_stream == 0:                # the default stream cannot be captured
        return False
    with torch.cuda.stream(stream):
        return torch.cuda.is_current_stream_capturing()


class _Order:
    """Runs an object's calls in the order in which they are made, whatever streams
    they are given, and tells the allocator which streams use its buffers: every
    call reads and writes memory of the object, so that none may overtake another.
    A call on another stream than the last one's waits for that one; a call that
    is captured waits for captured ones only, a call that is not for those that
    are not. The calls are made with the buffers' GPU as the current one, whose
    default stream the address 0 means."""

    def __init__(self, stream, buffers):
        """The buffers belong to the stream."""
        torch = _torch()
        self.gpu, self.cuda = buffers[0].device.index, torch.cuda
        # the current stream's address without the object around it: a fifth of the time
        self.current_device, self.raw = torch.cuda.current_device, torch._C._cuda_getCurrentRawStream
        self.stream = self.launched = self.on(stream)      # of the last call, and of the last that was not captured
        self.address, self.seen, self.buffers = stream.cuda_stream, {stream.cuda_stream}, buffers
        self.event = torch.cuda.Event()

    def on(self, stream):
        """The stream to run on: the GPU's current one for None."""
        if stream is None:
            return self.cuda.current_stream(self.gpu)
        if stream.device_index != self.gpu:
            raise ValueError(f"the stream must be one of cuda:{self.gpu}")
        return stream

    def enter(self, stream):
        """The address of the stream to run on."""
        if stream is None and self.raw(self.gpu) == self.address:
            return self.address
        stream = self.on(stream)
        if stream.cuda_stream != self.address:
            self._change(stream)
        return stream.cuda_stream

    def run(self, call, *args, stream):
        """A library call, with the stream's address as its last argument."""
        p = self.enter(stream)
        if self.current_device() == self.gpu:
            return _check(call(*args, p))
        with self.cuda.device(self.gpu):
            _check(call(*args, p))

    def _change(self, stream):
        p, captured = stream.cuda_stream, _capturing(stream)
        last = self.launched if not captured else self.stream if _capturing(self.stream) else stream
        if last.cuda_stream != p:
            self.event.record(last)
            stream.wait_event(self.event)
        if p not in self.seen:
            for x in self.buffers:
                x.record_stream(stream)
            self.seen.add(p)
        self.stream = stream
        if captured:
            self.address = None                # whether the next call is captured too has to be asked
        else:
            self.launched, self.address = stream, p


class AdamW:
    """AdamW over many tensors at once, one launch per step, with moments in 32
    bits or in blocks of 8-bit codes (format: scadles.h).

    ``params``: contiguous float32 tensors, updated in place, no two overlapping (a
    tensor used twice is listed once); ``grads``: as many contiguous tensors of the
    same sizes, all float32 or all bfloat16, read at every step where they are (a
    part of a flat gradient will do, at any offset). ``weight_decay``: one value,
    or one per tensor. ``copies``: bfloat16 tensors that receive the updated
    parameters, or None.

    Calls may be given any streams: they run in the order in which they are made (a
    stream has to exist until the call after its last one is made). What the caller
    does with the tensors on other streams is the caller's to order.

    The moments start at zero and belong to the object: ``m`` and ``v`` (float32
    [n], the tensors packed in order; with ``state_bits=8`` uint8 [blocks, 256],
    every tensor starting a block) and ``tops`` (int32 [blocks] or None), ``t``
    the number of steps made."""

    def __init__(self, params, grads, *, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.01,
                 state_bits: int = 32, copies=None, stream=None):
        torch = _torch()
        self.params = list(params)
        if not self.params:
            raise ValueError("params is empty")
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 32 or 8")
        for i, p in enumerate(self.params):
            _dev_f32(p, f"params[{i}]", self.params[0].device if i else None)
        self.device = self.params[0].device
        self.sizes = [p.numel() for p in self.params]
        self.n = sum(self.sizes)
        self.betas, self.eps, self.state_bits = (float(betas[0]), float(betas[1])), float(eps), int(state_bits)
        L = len(self.params)
        decay = [float(weight_decay)] * L if isinstance(weight_decay, (int, float)) else [float(w) for w in weight_decay]
        self.copies = None if copies is None else list(copies)
        if len(decay) != L or (self.copies is not None and len(self.copies) != L):
            raise ValueError("one weight_decay and one copy per tensor")
        for i, c in enumerate(self.copies or []):
            if not isinstance(c, torch.Tensor) or c.dtype != torch.bfloat16 or not c.is_contiguous():
                raise TypeError(f"copies[{i}] must be a contiguous bfloat16 GPU tensor")
            if c.device != self.device or c.numel() != self.sizes[i]:
                raise ValueError(f"copies[{i}] must be on the parameters' GPU and of their size")
        self._tensors = (AdamWTensor * L)()
        self._plan, self._options = AdamWPlan(), AdamWOptions(0.0, self.betas[0], self.betas[1], self.eps, 0)
        self.t = 0
        stream = torch.cuda.current_stream(self.device) if stream is None else stream
        with torch.cuda.stream(stream):
            if self.state_bits == 8:
                blocks = [-(-x // MOMENT_BLOCK) for x in self.sizes]
                self.m = torch.zeros((sum(blocks), MOMENT_BLOCK), dtype=torch.uint8, device=self.device)
                self.v = torch.zeros_like(self.m)
                self.tops = torch.zeros(sum(blocks), dtype=torch.int32, device=self.device)
            else:
                self.m = torch.zeros(self.n, dtype=torch.float32, device=self.device)
                self.v = torch.zeros_like(self.m)
                self.tops = None
            at = 0
            m, v, tops = self.m.data_ptr(), self.v.data_ptr(), None if self.tops is None else self.tops.data_ptr()
            for i, p in enumerate(self.params):
                x = self._tensors[i]
                x.param, x.n, x.weight_decay = p.data_ptr(), self.sizes[i], decay[i]
                x.copy = None if self.copies is None else self.copies[i].data_ptr()
                if self.state_bits == 8:
                    x.m, x.v, x.tops = m + at * MOMENT_BLOCK, v + at * MOMENT_BLOCK, tops + at * 4
                    at += blocks[i]
                else:
                    x.m, x.v = m + at * 4, v + at * 4
                    at += self.sizes[i]
            self._table = _workspace(int(_adamw_plan_bytes(self._tensors, L)), self.device)
            self.clip = torch.zeros(2, dtype=torch.float32, device=self.device)
        self._order = _Order(stream, [x for x in (self.m, self.v, self.tops, self._table, self.clip) if x is not None])
        moments = [x for x in (self.m, self.v, self.tops) if x is not None]
        self._moments, self._steps = _wholes(moments), _wholes(self.params + (self.copies or []) + moments)
        self.set_grads(grads, stream=stream)

    def set_grads(self, grads, *, stream=None):
        """Point the optimizer at other gradients of the same sizes (writes the plan
        anew). Needed before the next step whenever gradients were allocated anew:
        the object keeps the ones it has, and a step goes on reading them."""
        torch = _torch()
        grads = list(grads)
        if len(grads) != len(self.params):
            raise ValueError("one gradient per parameter")
        for i, g in enumerate(grads):
            if not isinstance(g, torch.Tensor) or not g.is_cuda or not g.is_contiguous():
                raise TypeError(f"grads[{i}] must be a contiguous GPU tensor")
            if g.dtype not in (torch.float32, torch.bfloat16) or g.dtype != grads[0].dtype:
                raise TypeError("grads must be all float32 or all bfloat16")
            if g.device != self.device or g.numel() != self.sizes[i]:
                raise ValueError(f"grads[{i}] must be on the parameters' GPU and of their size")
            self._tensors[i].grad = g.data_ptr()
        self._order.run(_adamw_plan_build, self._tensors, len(grads), self.state_bits,
                        1 if grads[0].dtype == torch.bfloat16 else 0, self._table.data_ptr(), self._table.numel(),
                        self._plan, stream=stream)
        self.grads = grads

    def grad_norm(self, max_norm: float = math.inf, *, stream=None):
        """float32[2] = (global norm of the gradients, factor that clips it to
        ``max_norm``), for ``step``; the factor is NaN when the norm is not
        finite. The tensor is the object's own and overwritten by the next call."""
        self._order.run(_grad_norm, self._plan, float(max_norm), self.clip.data_ptr(), stream=stream)
        _written((self.clip,))
        return self.clip

    def step(self, lr: float, *, clip=None, stream=None):
        """One step, with the gradients times clip[1] when given (as from
        ``grad_norm``; a NaN there leaves everything but ``t`` as it is)."""
        o = self._options
        o.lr, o.step = float(lr), self.t + 1
        if clip is not None and clip.numel() != 2:
            raise ValueError("clip must have two entries")
        self._order.run(_adamw_step, self._plan, o, None if clip is None else _dev_f32(clip, "clip", self.device),
                        stream=stream)
        _written(self._steps)
        self.t += 1

    def moments(self, *, stream=None):
        """(m, v) as float32 [n], the tensors packed in order: the 32-bit moments
        themselves, or what the 8-bit codes stand for."""
        if self.state_bits == 32:
            self._order.enter(stream)
            return self.m, self.v
        m, v = (_empty(self.n, _torch().float32, self.device, stream) for _ in range(2))
        self._order.run(_adamw_get_moments, self._plan, m.data_ptr(), v.data_ptr(), stream=stream)
        return m, v

    def load(self, t: int, m, v, *, tops=None, stream=None):
        """Continue from step ``t`` with these moments: the values as ``moments``
        gives them, or the codes ``m``, ``v`` with ``tops``."""
        torch = _torch()
        if t < 0:
            raise ValueError("t must not be negative")
        stream = self._order.on(stream)
        if tops is not None:
            if self.state_bits != 8:
                raise ValueError("tops belongs to 8-bit moments")
            for x, mine, name in ((m, self.m, "m"), (v, self.v, "v"), (tops, self.tops, "tops")):
                if x.dtype != mine.dtype or x.shape != mine.shape:
                    raise ValueError(f"{name} must be {mine.dtype} of shape {tuple(mine.shape)}")
            self._order.enter(stream)
            with torch.cuda.stream(stream):
                for x, mine in ((m, self.m), (v, self.v), (tops, self.tops)):
                    mine.copy_(x)
        else:
            if m.numel() != self.n or v.numel() != self.n:
                raise ValueError("m and v must hold every element")
            self._order.run(_adamw_set_moments, self._plan, _dev_f32(m, "m", self.device), _dev_f32(v, "v", self.device),
                            int(t), stream=stream)
            _written(self._moments)
        self.t = int(t)


# ---- the router of a mixture of experts ---------------------------------------------------------------

@dataclass
class RouterOutputs:
    """What ``Router.forward`` returns: the router's own buffers, overwritten by
    its next forward pass."""
    idx: object          # int32 [T, k], -1 where there is no choice
    gate: object         # float32 [T, k]
    lse: object          # float32 [T]
    counts: object       # int32 [devices, experts]
    load: object         # float32 [experts]
    share: object        # float32 [devices]: 1 / counted rows
    loss: object         # float32 [2]: balance, z
    mark: object = None  # the pass's, for the backward pass's check


class _Mark:
    """A router's pass, held by its outputs: the router sees whether any are left."""
    __slots__ = ("__weakref__",)


def _seen(x):
    """A tensor and its version, without holding it."""
    return weakref.ref(x), 0 if x.is_inference() else x._version


def _same(a, b):
    return a[1] == b[1] and a[0]() is b[0]()


class _Pass:
    """What the library reads of a router's pass: bounds, weights and shapes. The
    backward pass has weights of its own (``w_back``) for when they are given.
    Beside them what tells the pass from others: its logits and mask."""

    def __init__(self, E, k, K, renormalise):
        off, w, w_back = (_u64 * (K + 1))(), (ctypes.c_float * K)(), (ctypes.c_float * K)()
        self.off = np.frombuffer(off, dtype=np.uint64)
        self.w, self.w_back = (np.frombuffer(x, dtype=np.float32) for x in (w, w_back))
        self.shape, self.back = (RouterShape(0, E, off, x, E, k, K, 0, renormalise) for x in (w, w_back))
        self.logits = self.valid = None

    def repeats(self, other):
        """Whether this pass has the inputs of ``other``, so that it writes the same
        once more. A mask that no longer exists is taken for the same one."""
        if not _same(self.logits, other.logits) or (self.valid is None) != (other.valid is None):
            return False
        if self.valid is not None and other.valid[0]() is not None and not _same(self.valid, other.valid):
            return False
        return self.off.tobytes() == other.off.tobytes() and self.w.tobytes() == other.w.tobytes()


class Router:
    """Routes the tokens of K devices to ``experts`` experts, ``k`` each, with the
    balance loss and the z loss over all devices (scadles_router_forward), and
    gives the logits' gradient. Outputs and workspace are allocated once, for up
    to ``max_tokens`` rows. Calls may be given any streams: they run in the order
    in which they are made (a stream has to exist until the call after its last one
    is made). Outside autograd: the outputs have no history, and the gradient that
    ``backward`` returns goes on with ``logits.backward(d_logits)``."""

    def __init__(self, max_tokens: int, experts: int, k: int, *, devices: int = 1, renormalise: bool = False,
                 device=None):
        torch = _torch()
        self.max_tokens, self.experts, self.k, self.devices = int(max_tokens), int(experts), int(k), int(devices)
        self.renormalise = bool(renormalise)
        need = int(_router_ws_bytes(self.max_tokens, self.experts, self.devices)) if self.max_tokens >= 0 else 0
        if need == 0 or not 1 <= self.k <= min(self.experts, ROUTER_MAX_K):
            raise ScadlesError(1, f"invalid max_tokens={max_tokens}, experts={experts}, k={k} or devices={devices}")
        dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        f32 = dict(dtype=torch.float32, device=dev)
        T, E, K = self.max_tokens, self.experts, self.devices
        self.idx = torch.empty((T, self.k), dtype=torch.int32, device=dev)
        self.gate, self.lse = torch.empty((T, self.k), **f32), torch.empty(T, **f32)
        self.counts = torch.empty((K, E), dtype=torch.int32, device=dev)
        self.load, self.share, self.loss = torch.empty(E, **f32), torch.empty(K, **f32), torch.empty(2, **f32)
        self.ws = _workspace(need, dev)
        self._out = RouterOut(*[x.data_ptr() for x in (self.idx, self.gate, self.lse, self.counts, self.load, self.share,
                                                       self.loss)])
        self.device = self.idx.device
        self._order = _Order(torch.cuda.current_stream(self.device), [self.idx, self.gate, self.lse, self.counts,
                                                                      self.load, self.share, self.loss, self.ws])
        self._outs = (self.idx, self.gate, self.lse, self.counts, self.load, self.share, self.loss)
        # the last pass, and the one that takes its place once the library has accepted it
        self._last, self._next = (_Pass(E, self.k, K, self.renormalise) for _ in range(2))
        self._mark = lambda: None                # a weak reference to the last pass's

    def _logits(self, x, name):
        """(address, elements between rows) of a [tokens, experts] tensor."""
        torch = _torch()
        if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dtype not in (torch.float32, torch.bfloat16):
            raise TypeError(f"{name} must be a float32 or bfloat16 GPU tensor")
        if x.device != self.device:
            raise ValueError(f"{name} must be on {self.device}")
        if x.dim() != 2 or x.shape[1] != self.experts:
            raise ValueError(f"{name} must be [tokens, {self.experts}]")
        row, step = x.stride()
        if self.experts > 1 and step != 1:
            raise ValueError(f"{name}: a row's experts must be adjacent")
        if x.shape[0] < 2:
            row = self.experts
        elif row < self.experts:
            raise ValueError(f"{name}: rows overlap")
        return x.data_ptr(), row

    @staticmethod
    def _fill(view, values, name):
        if len(values) != len(view):
            raise ValueError(f"{name} must have {len(view)} entries")
        view[:] = values

    def forward(self, logits, *, tok_off=None, weights=None, valid=None, stream=None) -> RouterOutputs:
        """``logits`` [T, experts] float32 or bfloat16, rows ``tok_off[d]`` to
        ``tok_off[d + 1]`` those of device d (None: one device). ``weights``: Eqn
        4a, by default the devices' shares of the rows. ``valid``: bool [T] or
        None; False marks padding."""
        torch = _torch()
        p, ld = self._logits(logits, "logits")
        T = logits.shape[0]
        if T > self.max_tokens:
            raise ValueError(f"more than max_tokens = {self.max_tokens} rows")
        n = self._next
        self._fill(n.off, (0, T) if tok_off is None else tok_off, "tok_off")
        if weights is None:
            weights = np.diff(n.off.astype(np.int64)) / T if T else [1.0 / self.devices] * self.devices
        self._fill(n.w, weights, "weights")
        if valid is not None:
            if valid.dtype not in (torch.bool, torch.uint8) or not valid.is_cuda or not valid.is_contiguous():
                raise TypeError("valid must be a contiguous bool GPU tensor")
            if valid.numel() != T or valid.device != self.device:
                raise ValueError(f"valid must have one entry per row and be on {self.device}")
        f = n.shape
        f.tokens, f.ld, f.logits_type = T, ld, logits.dtype == torch.bfloat16
        self._order.run(_router_forward, f, p, None if valid is None else valid.data_ptr(), self._out,
                        self.ws.data_ptr(), self.ws.numel(), stream=stream)
        _written(self._outs)
        n.logits, n.valid = _seen(logits), None if valid is None else _seen(valid)
        mark = self._mark()
        if mark is None or not n.repeats(self._last):
            mark = _Mark()
            self._mark = weakref.ref(mark)
        self._last, self._next = n, self._last
        if T == self.max_tokens:
            return RouterOutputs(self.idx, self.gate, self.lse, self.counts, self.load, self.share, self.loss, mark)
        return RouterOutputs(self.idx[:T], self.gate[:T], self.lse[:T], self.counts, self.load, self.share, self.loss, mark)

    def backward(self, logits, out: RouterOutputs, d_gate=None, d_loss=None, *, weights=None, d_logits=None, stream=None):
        """Gradient of ``logits`` under ``d_gate`` [T, k] (or None) of the gates and
        ``d_loss`` [2] (or None) of the losses, both float32; ``out`` is the last
        forward pass's: one that another pass has overwritten is refused.
        ``weights``: as in the forward pass by default; ones give
        each device's own share, before the aggregation weights it. Returned in
        ``d_logits`` if given."""
        torch = _torch()
        p, ld = self._logits(logits, "logits")
        f, T = self._last.shape, logits.shape[0]
        if out.mark is None or out.mark is not self._mark():
            raise ValueError("out is not this router's last forward pass")
        if T != f.tokens or f.logits_type != (logits.dtype == torch.bfloat16):
            raise ValueError("logits are not those of the forward pass")
        if d_gate is not None and d_gate.numel() != T * self.k:
            raise ValueError(f"d_gate must have {T * self.k} entries")
        if d_loss is not None and d_loss.numel() != 2:
            raise ValueError("d_loss must have 2 entries")
        given = d_logits is not None
        if not given:
            d_logits = _empty((T, self.experts), logits.dtype, logits.device, stream)
        q, ld_out = self._logits(d_logits, "d_logits")
        if d_logits.dtype != logits.dtype or d_logits.shape[0] != T:
            raise ValueError("d_logits must be like logits")
        if weights is not None:
            self._fill(self._last.w_back, weights, "weights")
            f = self._last.back
            f.tokens, f.logits_type = T, self._last.shape.logits_type
        f.ld = ld
        self._order.run(_router_backward, f, p, self._out,
                        None if d_gate is None else _dev_f32(d_gate, "d_gate", self.device),
                        None if d_loss is None else _dev_f32(d_loss, "d_loss", self.device), q, ld_out, stream=stream)
        if given:
            _written((d_logits,))
        return d_logits


# ---- between tokens and logits ------------------------------------------------------------------------

from .language import (Batch, CrossEntropyOut, CrossEntropyOutputs, CrossEntropyShape, Embedding,  # noqa: E402,F401
                       EmbeddingShape, ExpertOrder, ExpertRows, LayerNorm, LayerNormOutputs, LinearCrossEntropy,
                       NormShape, OrderShape)
