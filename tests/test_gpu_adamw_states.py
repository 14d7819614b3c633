"""The second moment in 8 bits over many steps against the recurrence in 64 bits."""
import pytest

from paper_2608_14575_amd import routed

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("beta2,steps", [(0.999, 6000), (0.98, 800), (0.95, 400)])
@pytest.mark.parametrize("decades", [0, 3])
def test_second_moment_settles_a_little_above(beta2, steps, decades):
    """The root r of v is rounded up or down without a bias, which leaves r^2 with one: the rounding's variance.

    To first order, gradients normal, codes not below 2^-6 (true here: roots of a block lie within three decades, and codes
    reach 448).  Between two steps r / scale moves by d off a code, of which the root's own part is at most (1 - beta2) / 2
    |g^2 / v - 1| of r, and the scale's, which goes by the block's largest, as much again; E |g^2 / v - 1| = 0.968.  The variance is
    d (s - d) < d s with the codes' distance s at most r / 8: a step adds at most (1 - beta2) 0.968 / 8 of v, the steps that v
    remembers, 1 / (1 - beta2), 0.121 of the v that is stored: v is at most 1 / (1 - 0.121) = 1.138 of what it should be, and not less
    than that.  The noise of v in a step is 2 r times the root's: a variance of 4 v times the above, and over 1 / (1 - beta2^2) steps
    at most 4 0.121 / (1 + beta2) < 0.25 v^2 (1.138^2 for the v that is stored): a standard deviation below 0.57.  Means over 2^16 values: 6 standard
    errors are 6 0.57 / 256 = 0.0134.  The root itself has no bias beside what the square's root makes of that noise: its mean is between
    1 - 0.57^2 / 8 - 0.0134 / 2 (noise alone) and sqrt(1.138) + 0.0134 / 2."""
    n = 1 << 16
    ops = routed.RoutedOps(stream=torch.cuda.current_stream().cuda_stream)
    g = torch.Generator("cuda").manual_seed(steps)
    size = 10.0 ** (-decades * torch.rand(n, generator=g, device="cuda"))
    p, d = torch.zeros(n, device="cuda"), torch.empty(n, device="cuda")
    opt = routed.AdamW(ops, [p], [d], lr=1e-6, betas=(0.9, beta2), weight_decay=0.0, bits=8, seed=1)
    v = torch.zeros(n, dtype=torch.float64, device="cuda")
    for _ in range(steps):
        torch.mul(torch.randn(n, generator=g, device="cuda"), size, out=d)
        opt.step()
        v.mul_(beta2).add_(d.double().square(), alpha=1 - beta2)
    ratio = opt.state["v"][0].double() * opt.state["v_scale"][0].double().repeat_interleave(256) / v.sqrt()
    assert 1 - 0.0134 < float(ratio.square().mean()) < 1.138 + 0.0134
    assert float(ratio.square().std()) < 0.57
    assert 1 - 0.57 ** 2 / 8 - 0.0067 < float(ratio.mean()) < 1.138 ** 0.5 + 0.0067
    ops.close()
