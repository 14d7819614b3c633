"""The training example and AdamW objects on streams of which none is torch's default one."""
import pytest

from paper_2608_14575_amd import routed

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

LATE = 20_000_000       # cycles, about 10 ms: longer than the host takes from a fill to the first step


def late(fill):
    """The fill, with its values there only after a while (NaNs until then)."""
    def call(*a, **kw):
        t = fill(*a, **kw)
        if t.is_cuda:
            value = t.clone()
            t.fill_(float("nan"))
            torch.cuda.synchronize()
            torch.cuda._sleep(LATE)
            t.copy_(value)
        return t
    return call


def test_training_example_on_a_stream(monkeypatch):
    """The losses, weights and gradients of a run on the default stream, bit for bit, also where what a step reads is filled late."""
    want, p, grad = routed.train_tokens(steps=3, n=512, tokens=512)
    for fill in (torch.full, late(torch.full)):
        monkeypatch.setattr(torch, "full", fill)
        with torch.cuda.stream(torch.cuda.Stream()):
            got, q, d = routed.train_tokens(steps=3, n=512, tokens=512)
        torch.cuda.synchronize()
        assert got == want
        for name in p:
            assert torch.equal(p[name], q[name]) and torch.equal(grad[name], d[name]), name


def test_made_state_on_another_stream(monkeypatch):
    """States that are made on a stream which the context does not run on are there before the first step."""
    def run(ops):
        g = torch.Generator("cuda").manual_seed(2)
        p, d = ([torch.randn(n, generator=g, device="cuda") for n in (5000, 3, 256)] for _ in range(2))
        torch.cuda.synchronize()
        opt = routed.AdamW(ops, p, d, lr=1e-2)
        opt.step()
        torch.cuda.synchronize()
        return p + opt.state["m"] + opt.state["v"]

    want = run(routed.RoutedOps(stream=torch.cuda.current_stream().cuda_stream))
    own = torch.cuda.Stream()
    monkeypatch.setattr(torch, "zeros", late(torch.zeros))
    with torch.cuda.stream(torch.cuda.Stream()):
        got = run(routed.RoutedOps(stream=own.cuda_stream))
    assert all(torch.equal(a, b) for a, b in zip(want, got))
