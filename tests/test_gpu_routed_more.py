"""More of the operators on a routed batch (include/hwr_ops.h): batches of up to 2^31
rows, intermediates near the largest values, few rows of many groups.

Tolerances: inputs whose products and sums are whole numbers below 2^24 give exact
sums in fp32, in any order, so that a bf16 result is off by its rounding alone (2^-8
of its value).  Otherwise: a sum of K products in fp32 is off by at most (K + 16) 2^-24 times the
sum of the terms' magnitudes, and its rounding by 2^-8 (bf16) or 2^-24 (fp32) of the value."""
import numpy as np
import pytest

from paper_2608_14575_amd import hwr, routed
from test_gpu_routed_ops import EPS, TYPES, close, grouped, outer, product, rand, sizes_of

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture()
def ops():
    assert torch.cuda.is_available(), "GPU tests need a device"
    o = routed.RoutedOps(stream=torch.cuda.current_stream().cuda_stream)
    yield o
    o.close()
    torch.cuda.empty_cache()


# ---------------------------------------------------------------- the largest batches
CHUNK = 1 << 28


def every(n, step, dtype):
    """[n][1]: one in every `step`-th row, zeros elsewhere."""
    v = torch.zeros(n, 1, dtype=dtype, device="cuda")
    v[::step] = 1
    return v


def test_group_of_2_31_rows(ops):
    n, G = 2 ** 31 - 1, 3
    choice = torch.ones(n, dtype=torch.int32, device="cuda")
    choice[n - 2], choice[5] = 0, 7                     # one row of group 0, one in no group
    offsets = torch.empty(G + 1, dtype=torch.int32, device="cuda")
    order = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    ops.group(choice, G, offsets=offsets, order=order)
    assert offsets.tolist() == [0, 1, n - 1, n - 1]
    assert order[0].item() == n - 2 and order[n - 1].item() == 5
    assert order[n - 2].item() == n - 1                 # the last of group 1
    for a in range(0, n, CHUNK):                        # group 1: the rows in order, without those two
        want = torch.arange(a, min(a + CHUNK, n), dtype=torch.int64, device="cuda")
        want += (want >= 5).long()
        got = order[a + 1:a + 1 + len(want)].long()
        got, want = got[:n - 2 - a], want[:n - 2 - a]
        want = want + (want >= n - 2).long()
        assert torch.equal(got, want)


def test_products_of_2_31_rows(ops):
    n, t = 2 ** 31 - 512, torch.bfloat16
    off = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    x = every(n, 1 << 10, t)
    x[n - 1] = 1
    w = torch.full((1, 1, 1), 3.0, dtype=t, device="cuda")
    y = torch.full((n, 1), 7.0, dtype=t, device="cuda")
    ops.matmul(x, w, off, y=y)
    for a in range(0, n, CHUNK):
        assert torch.equal(y[a:a + CHUNK], x[a:a + CHUNK] * 3)
    y.fill_(7)
    dw = torch.empty_like(w)
    ops.matmul_grad(x, x, w, off, dx=y, dw=dw)
    count = sum(int(x[a:a + CHUNK].sum(dtype=torch.float64)) for a in range(0, n, CHUNK))
    assert count == 2 ** 21 + 1
    assert abs(float(dw) - count) <= 2.0 ** -8 * count
    for a in range(0, n, CHUNK):
        assert torch.equal(y[a:a + CHUNK], x[a:a + CHUNK] * 3)


def test_adapters_of_2_27_rows(ops):
    """More rows than one row of the grid of the low-rank intermediates' pair holds."""
    n, t, G = 2 ** 27 + 1000, torch.bfloat16, 2
    half = n // 2 + 11
    off = torch.tensor([0, half, n], dtype=torch.int32, device="cuda")
    x, dy = every(n, 64, t), every(n, 128, t)
    x[n - 1], dy[n - 1] = 1, 1
    w = torch.full((1, 1), 2.0, dtype=t, device="cuda")
    a = torch.tensor([1.0, 2.0], dtype=t, device="cuda").view(G, 1, 1)
    b = torch.tensor([3.0, 5.0], dtype=t, device="cuda").view(G, 1, 1)
    dx, da, db = torch.full_like(x, 7.0), torch.empty_like(a), torch.empty_like(b)
    ops.adapter_grad(dy, x, w, a, b, None, off, dx=dx, da=da, db=db)
    y = torch.full_like(dy, 7.0)
    ops.adapter(x, w, a, b, None, off, y=y)
    for g, (p0, p1) in enumerate(((0, half), (half, n))):
        ab = float(a[g] * b[g])
        assert torch.equal(y[p0:p1], x[p0:p1] * (2 + ab))
        assert torch.equal(dx[p0:p1], dy[p0:p1] * (2 + ab))
        both = int((x[p0:p1] * dy[p0:p1]).sum(dtype=torch.float64))
        assert both > 2 ** 18
        for got, want in ((da[g], float(b[g]) * both), (db[g], float(a[g]) * both)):
            assert abs(float(got) - want) <= 2.0 ** -8 * want


# ---------------------------------------------------------------- the largest values
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("n", [8, 300])
def test_intermediates_past_the_largest_bf16(ops, n, sign):
    """A low-rank intermediate that fp32 holds and bf16 rounds to an infinity: what is
    made of it is finite, of few rows and of many.  In bf16 calls the intermediate is a sum of
    two bf16 values, exact here (2^-8: the rounding of the result)."""
    t, k, m, R, top = torch.bfloat16, 16, 24, 4, (2 - 2 ** -7) * 2.0 ** 127
    v = sign * (top + 1.75 * 2.0 ** 119)
    assert torch.tensor(v).isfinite() and torch.tensor(v).to(t).isinf()
    zeros = lambda *s: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    off = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    big = torch.tensor([top, 1.75 * 2.0 ** 119], dtype=t, device="cuda") * sign

    def near(got, want):
        assert (got.double() - want).abs().max() <= 2.0 ** -8 * abs(want), (got, want)

    # s x A of row 1, column 2 is v
    x, w, a, b = zeros(n, k), zeros(k, m), zeros(1, k, R), zeros(1, R, m)
    x[1, :2] = 1
    a[0, :2, 2] = big
    b[0, 2] = 2.0 ** -10
    y = torch.full((n, m), 7.0, dtype=t, device="cuda")
    ops.adapter(x, w, a, b, None, off, y=y)
    near(y[1], v * 2.0 ** -10)
    assert not y[0].any() and not y[2:].any()
    dy, db = zeros(n, m), torch.empty_like(b)
    dy[1] = 2.0 ** -9
    ops.adapter_grad(dy, x, w, a, b, None, off, db=db)
    near(db[0, 2], v * 2.0 ** -9)
    # u of row 1, column 2 is v
    x, dy, a, b = zeros(n, k), zeros(n, m), zeros(1, k, R), zeros(1, R, m)
    dy[1, :2] = 1
    b[0, 2, :2] = big
    a[0, :, 2] = 2.0 ** -10
    x[1] = 2.0 ** -9
    dx, da = torch.empty_like(x), torch.empty_like(a)
    ops.adapter_grad(dy, x, w, a, b, None, off, dx=dx, da=da)
    near(dx[1], v * 2.0 ** -10)
    near(da[0, :, 2], v * 2.0 ** -9)


# ---------------------------------------------------------------- few rows of many groups
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,G,k,m,kind", [(1, 32, 2048, 1032, "one"), (4, 300, 1024, 1024, "even"), (7, 9, 1032, 2056, "skew"),
                                          (20, 70, 1027, 1029, "skew"), (5, 40, 1024, 1536, "one")])
def test_gradients_of_fewer_rows_than_groups(ops, n, G, k, m, kind, dtype):
    t, u, _ = TYPES[dtype]
    gen = torch.Generator("cuda").manual_seed(n + k)
    gid, off, order = grouped(sizes_of(kind, n, G, np.random.default_rng(n)), G)
    x, dy, w = rand(gen, n, k, dtype=t), rand(gen, n, m, dtype=t), rand(gen, G, k, m, dtype=t)
    dx, dw = torch.full_like(x, 7.0), torch.full_like(w, 7.0)
    ops.matmul_grad(dy, x, w, off, order, dx=dx, dw=dw)
    ref, s = product(dy, w.transpose(1, 2).contiguous(), gid)
    close(dx, ref, u * ref.abs() + (m + 16) * EPS * s)
    ref, s, cnt = outer(x, dy, gid, G)
    close(dw, ref, u * ref.abs() + (cnt + 16) * EPS * s)
    again = torch.full_like(x, 7.0)
    ops.matmul_grad(dy, x, w, off, order, dx=again)
    assert torch.equal(again, dx)
