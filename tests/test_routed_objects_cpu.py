"""The objects of paper_2608_14575_amd/routed.py without a device: what is ordered against
what, on stand-ins for streams and contexts that write down the calls."""
import contextlib

import pytest

from paper_2608_14575_amd import routed

torch = pytest.importorskip("torch")


class Stream:
    def __init__(self, number, log):
        self.cuda_stream, self.log = number, log

    def wait_stream(self, other):
        self.log.append(("wait", self.cuda_stream, other.cuda_stream))

    def synchronize(self):
        self.log.append(("synchronize", self.cuda_stream))


@pytest.fixture
def log():
    return []


@pytest.fixture
def caller(monkeypatch, log):
    """The stream that is torch's current one."""
    s = Stream(7, log)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: s)
    return s


def noting(log, fn):
    def call(*a, **kw):
        log.append(("fill",))
        return fn(*a, **kw)
    return call


class Ops:
    """A context that notes its calls."""

    def __init__(self, log, stream=0):
        self.log, self.stream = log, stream

    def close(self):
        pass

    def __getattr__(self, name):
        return lambda *a, **kw: self.log.append(("op", name))


def test_training_example_waits_for_its_tensors(monkeypatch, log, caller):
    """Everything that a step reads is filled on the caller's stream before the step's stream waits for that one."""
    own = Stream(8, log)
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    offsets, order = torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    monkeypatch.setattr(torch.cuda, "Stream", lambda: own)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda: None)
    monkeypatch.setattr(torch.cuda, "CUDAGraph", lambda: None)
    monkeypatch.setattr(torch.cuda, "graph", lambda *a, **kw: contextlib.nullcontext())
    monkeypatch.setattr(routed, "_routed", lambda n, seed: (Ops(log), 2, x, offsets, order, Ops(log)))
    monkeypatch.setattr(routed, "RoutedOps", lambda stream: Ops(log, stream))
    monkeypatch.setattr(routed, "AdamW", noting(log, lambda ops, *a, **kw: ops))       # (its states are filled too)
    for fill in ("randn", "randint", "full", "zeros"):
        monkeypatch.setattr(torch, fill, noting(log, getattr(torch, fill)))
    routed.train_tokens(steps=1, n=4, tokens=8)
    last = max(i for i, e in enumerate(log) if e == ("fill",))
    first = min(i for i, e in enumerate(log) if e[0] == "op")
    assert ("op", "adapter") == log[first] and ("wait", 8, 7) in log[last:first], log
