"""The most likely tokens of rows whose masks are infinities and lowest values, one beside the other."""
import math

import pytest

from paper_2608_14575_amd import routed

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# 16 threads' worth, a wave, 256 threads, 1,024, shared rows; more and fewer tokens than candidates
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,m,top", [(3, 2, 2), (5, 40, 32), (9, 300, 32), (4, 511, 20), (7, 1500, 20), (600, 3000, 9), (5000, 2500, 4),
                                     (3, 9000, 32), (2, 40000, 32)])
def test_masks_of_both_kinds_are_equal(n, m, top, dtype):
    """Below -3.3e38 a logit counts as -inf: such tokens come last, the lower first, whatever their logits."""
    ops = routed.RoutedOps(stream=torch.cuda.current_stream().cuda_stream)
    g = torch.Generator("cuda").manual_seed(m)
    t = TYPES[dtype]
    x = torch.randn((n, m), generator=g, device="cuda").to(t)
    kind = torch.rand((n, m), generator=g, device="cuda")
    allowed = torch.randint(0, top + 1, (n, 1), generator=g, device="cuda") / m        # (in some rows none)
    x[kind >= allowed] = -math.inf
    x[kind > (1 + allowed) / 2] = torch.finfo(t).min
    token, logp = torch.empty((n, top), dtype=torch.int32, device="cuda"), torch.empty((n, top), device="cuda")
    lse = torch.empty(n, device="cuda")
    ops.log_probs(x, lse=lse, top_token=token, top_logp=logp)
    z = torch.where(x.double() < -3.3e38, -math.inf, x.double())
    want = torch.sort(z, dim=1, descending=True, stable=True)[1][:, :top]
    assert torch.equal(token.long(), want)
    masked = z.gather(1, want) == -math.inf
    assert (logp[masked] == -math.inf).all() and logp[~masked].isfinite().all()
    assert ((lse == -math.inf) == (z == -math.inf).all(1)).all()
    ops.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kept", [5, 20, 21, 70, 600])
@pytest.mark.parametrize("n,m", [(48, 32003), (3, 128000), (300, 5000), (4100, 2600)])
def test_allowed_tokens_side_by_side(n, m, kept, dtype):
    """A run of allowed tokens, as few and a few more than are asked for: few threads hold them all."""
    top, t = 20, TYPES[dtype]
    ops = routed.RoutedOps(stream=torch.cuda.current_stream().cuda_stream)
    g = torch.Generator("cuda").manual_seed(kept)
    first = torch.randint(0, m - kept + 1, (n, 1), generator=g, device="cuda")
    at = torch.arange(m, device="cuda")[None]
    x = torch.randn((n, m), generator=g, device="cuda").masked_fill_((at < first) | (at >= first + kept), -math.inf).to(t)
    token, logp = torch.empty((n, top), dtype=torch.int32, device="cuda"), torch.empty((n, top), device="cuda")
    ops.log_probs(x, top_token=token, top_logp=logp)
    z, want = torch.sort(x.float(), dim=1, descending=True, stable=True)
    assert torch.equal(token.long(), want[:, :top])
    assert torch.equal(logp == -math.inf, z[:, :top] == -math.inf)
    ops.close()
