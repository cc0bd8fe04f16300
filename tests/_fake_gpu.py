"""Stand-ins that let the host side of the training objects run without a GPU:
tensors in host memory that say they are on one, streams and events that write
down what is done with them, and library calls that only return a status."""
from __future__ import annotations

import contextlib
import types

import torch


class Tensor(torch.Tensor):
    """A host tensor that is on ``cuda:gpu`` as far as its attributes say."""
    gpu = 0

    @property
    def device(self):
        return torch.device("cuda", self.gpu)

    @property
    def is_cuda(self):
        return True

    @classmethod
    def __torch_function__(cls, func, kinds, args=(), kwargs=None):
        out = super().__torch_function__(func, kinds, args, kwargs or {})
        if isinstance(out, Tensor):
            out.gpu = next(a.gpu for a in args if isinstance(a, Tensor))
        return out

    def record_stream(self, stream):
        stream.log.append(("use", stream.cuda_stream))


def on(gpu, x):
    t = x.as_subclass(Tensor)
    t.gpu = gpu
    return t


class Stream:
    def __init__(self, log, number, gpu=0):
        self.log, self.cuda_stream, self.device_index, self.device = log, number, gpu, torch.device("cuda", gpu)
        self.capturing = False

    def wait_event(self, event):
        self.log.append(("wait", self.cuda_stream, event.at))


class Event:
    def __init__(self, log):
        self.log, self.at = log, None

    def record(self, stream):
        self.at = (stream.cuda_stream, len(self.log))
        self.log.append(("record", stream.cuda_stream))


class Cuda:
    """torch.cuda of a machine with ``gpus`` GPUs; stream 0 is every GPU's default stream."""

    def __init__(self, log, gpus=2):
        self.log, self.gpu, self.current = log, 0, [Stream(log, 0, g) for g in range(gpus)]

    def Event(self):
        return Event(self.log)

    def current_device(self):
        return self.gpu

    def current_stream(self, device=None):
        if device is None:
            return self.current[self.gpu]
        return self.current[device if isinstance(device, int) else torch.device(device).index or 0]

    def is_current_stream_capturing(self):
        return self.current_stream().capturing

    @contextlib.contextmanager
    def stream(self, s):
        gpu, was = self.gpu, self.current[s.device_index]
        self.gpu, self.current[s.device_index] = s.device_index, s
        yield
        self.gpu, self.current[s.device_index] = gpu, was

    @contextlib.contextmanager
    def device(self, device):
        gpu, self.gpu = self.gpu, device if isinstance(device, int) else device.index
        yield
        self.gpu = gpu


class Torch:
    """The torch module with a machine of ``gpus`` GPUs."""

    def __init__(self, log, gpus=2):
        self.cuda = Cuda(log, gpus)
        self._C = types.SimpleNamespace(_cuda_getCurrentRawStream=lambda gpu: self.cuda.current_stream(gpu).cuda_stream)

    def __getattr__(self, name):
        return getattr(torch, name)

    def _make(self, make, *shape, device=None, **more):
        device = torch.device("cuda" if device is None else device)
        return on(self.cuda.gpu if device.index is None else device.index, make(*shape, **more))

    def empty(self, *shape, **more):
        return self._make(torch.zeros, *shape, **more)

    zeros = empty


class Library:
    """Replaces the package's torch and its library calls on streams by stand-ins.
    ``status`` is what the next calls return; ``log`` holds (call, stream,
    current GPU, arguments) between the streams' entries."""

    CALLS = ("_adamw_plan_build", "_grad_norm", "_adamw_step", "_adamw_get_moments", "_adamw_set_moments", "_router_forward",
             "_router_backward")

    def __init__(self, sc, monkeypatch):
        self.log, self.status = [], 0
        self.torch = Torch(self.log)
        monkeypatch.setattr(sc, "_torch", lambda: self.torch)
        for name in self.CALLS:
            monkeypatch.setattr(sc, name, self._call(name))

    def _call(self, name):
        def call(*args):
            self.log.append((name, args[-1] or 0, self.torch.cuda.gpu, args[:-1]))
            return self.status
        return call

    def stream(self, number, gpu=0):
        return Stream(self.log, number, gpu)

    def calls(self):
        return [x for x in self.log if x[0] in self.CALLS]
