"""The layers' binding on the host: CPU tensors taken for device tensors, and a library that notes its calls."""
import contextlib

import torch


class Library:
    """Answers every call with success; notes (name, arguments) in calls."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 4096 if name.endswith("workspace_bytes") else 0
        return call

    def named(self, name):
        return [args for n, args in self.calls if n == name]


class Stream:
    """A stream object with torch's attributes."""

    def __init__(self, number):
        self.cuda_stream, self.device = number, torch.device("cpu")


class Device:
    """What happened: the current stream, the stream of every allocation by address, recorded uses."""

    def __init__(self, layers, monkeypatch):
        self.library, self.main = Library(), Stream(11)
        self.current, self.allocated, self.recorded = self.main, {}, []
        dev = self

        @contextlib.contextmanager
        def stream(s):
            before, dev.current = dev.current, s
            yield
            dev.current = before

        def allocating(f):
            def call(*args, **kw):
                t = f(*args, **kw)
                dev.allocated[t.data_ptr()] = dev.current
                return t
            return call

        monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
        monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: dev.recorded.append((t.data_ptr(), s)))
        monkeypatch.setattr(torch.Tensor, "new_empty", allocating(torch.Tensor.new_empty))
        monkeypatch.setattr(torch.Tensor, "clone", allocating(torch.Tensor.clone))
        for name in ("empty", "empty_like"):
            monkeypatch.setattr(torch, name, allocating(getattr(torch, name)))
        monkeypatch.setattr(torch.cuda, "stream", stream)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: dev.current)
        monkeypatch.setattr(layers, "_current_stream", lambda *a: dev.current.cuda_stream)
        monkeypatch.setattr(layers, "_device_of", torch.Tensor.get_device)
        monkeypatch.setattr(layers, "lib", lambda: self.library)
