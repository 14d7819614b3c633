"""The objects of paper_2608_14575_amd/routed.py without a device: what is ordered against
what, on stand-ins for streams and contexts that write down the calls."""
import contextlib
import ctypes as C
import gc
import types
import weakref

import numpy as np
import pytest

from paper_2608_14575_amd import hwr, routed

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
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
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


class Plan:
    """A context without a device for AdamW objects: hwr_adamw_init and _free note what they are called for, hwr_adamw_step
    what it is called with."""
    device, stream, ctx = -1, 0, 3

    def __init__(self, monkeypatch, log):
        @C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_void_p, C.c_void_p)
        def step(ctx, handle, args):
            log.append(("step", ctx, handle, hwr.hwr_adamw_args.from_address(args).step))
            return 0

        def init(ctx, config):
            log.append(("init", ctx, config.n_tensors))
            return C.c_void_p(5)

        monkeypatch.setattr(hwr, "hwr_adamw_init", init)
        monkeypatch.setattr(hwr, "hwr_adamw_free", lambda handle: log.append(("free", handle.value)))
        self._kinds = {torch.bfloat16: hwr.HWR_BF16, torch.float32: hwr.HWR_F32}
        self._f32 = torch.float32
        self._lib = types.SimpleNamespace(hwr_adamw_step=step)


def test_dropped_adamw_is_freed_at_once(monkeypatch, log, caller):
    """Without the cycle collector, which would free device memory at any later moment, also while a stream is captured."""
    caller.cuda_stream = 0
    opt = routed.AdamW(Plan(monkeypatch, log), [torch.ones(4)], [torch.ones(4)], lr=1e-3, steps=8)
    opt.step()
    assert log[-1] == ("step", 3, 5, 9) and opt.steps == 9
    state, whole = weakref.ref(opt.state["m"][0]), weakref.ref(opt)
    gc.disable()
    try:
        del opt
        assert whole() is None and state() is None and log[-1] == ("free", 5)
    finally:
        gc.enable()


@pytest.mark.parametrize("bits,master", [(32, False), (8, False), (8, True)])
def test_made_state_is_there_before_the_first_step(monkeypatch, log, caller, bits, master):
    """States are made on torch's current stream, steps run on the context's: where they are two, the object waits for the first.
    A program's own state is the program's to order."""
    monkeypatch.setattr(torch, "zeros", noting(log, torch.zeros))
    p = [torch.ones(4, dtype=torch.bfloat16)]
    opt = routed.AdamW(Plan(monkeypatch, log), p, [torch.ones_like(p[0])], lr=1e-3, bits=bits, master=master)
    last = max(i for i, e in enumerate(log) if e == ("fill",))
    assert ("synchronize", 7) in log[last:], log
    state = opt.state
    del log[:]
    routed.AdamW(Plan(monkeypatch, log), p, [torch.ones_like(p[0])], lr=1e-3, state=state)
    assert ("synchronize", 7) not in log
    caller.cuda_stream = 0                                      # the context's own
    del log[:]
    routed.AdamW(Plan(monkeypatch, log), p, [torch.ones_like(p[0])], lr=1e-3, bits=bits, master=master)
    assert ("fill",) in log and not any(e[0] == "synchronize" for e in log)


def test_adamw_is_not_made_under_capture(monkeypatch, log, caller):
    """Nothing is filled, allocated or asked of the library."""
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    monkeypatch.setattr(torch, "zeros", noting(log, torch.zeros))
    with pytest.raises(hwr.HwrError) as e:
        routed.AdamW(Plan(monkeypatch, log), [torch.ones(4)], [torch.ones(4)], lr=1e-3)
    assert e.value.status == hwr.HWR_ERR_STATE and log == []


def test_memory_stays_while_steps_write_it(monkeypatch, log, caller):
    """A tensor that is given other memory leaves the object its own: steps write what is there, until the object is dropped."""
    caller.cuda_stream = 0
    values = [np.ones(4, np.float32) for _ in range(5)]
    p, g, m, v = (torch.from_numpy(x) for x in values[:4])
    opt = routed.AdamW(Plan(monkeypatch, log), [p], [g], lr=1e-3, state={"m": [m], "v": [v]})
    gone = [weakref.ref(x) for x in values[:4]]
    for t in (p, g, m, v):
        t.data = torch.from_numpy(values[4])
    del values[:4], t
    gc.collect()
    assert all(r() is not None for r in gone)
    del opt
    gc.collect()
    assert all(r() is None for r in gone)
