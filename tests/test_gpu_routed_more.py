"""More of the operators on a routed batch (include/hwr_ops.h): batches of up to 2^31
rows, intermediates near the largest values, few rows of many groups, infinities and NaN in
whole chunks, forms that the other tests do not reach, and graphs among other calls.

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


# ---------------------------------------------------------------- the binding's functions
def test_functions_of_the_binding(ops):
    """hwr.hwr_group_rows and its fellows (the C functions, with their errors raised) give
    the bits that RoutedOps gives, with dense rows (stride 0) and without a table."""
    gen = torch.Generator("cuda").manual_seed(12)
    n, G, k, m, R, t = 300, 5, 264, 136, 12, torch.bfloat16
    choice = torch.randint(-1, G + 1, (n,), generator=gen, device="cuda", dtype=torch.int32)
    x, dy = rand(gen, n, k, dtype=t), rand(gen, n, m, dtype=t)
    w, ws, a, b = rand(gen, G, k, m, dtype=t), rand(gen, k, m, dtype=t), rand(gen, G, k, R, dtype=t), rand(gen, G, R, m, dtype=t)
    scale = 0.5 + torch.rand(G, generator=gen, device="cuda")

    def outputs():
        return {"offsets": torch.full((G + 1,), -7, dtype=torch.int32, device="cuda"),
                "order": torch.full((n,), -7, dtype=torch.int32, device="cuda"), "y": torch.full_like(dy, 7.0),
                "z": torch.full_like(dy, 7.0), "dx": torch.full_like(x, 7.0), "dw": torch.full_like(w, 7.0),
                "dz": torch.full_like(x, 7.0), "da": torch.full_like(a, 7.0), "db": torch.full_like(b, 7.0)}

    want = outputs()
    off, order = want["offsets"], want["order"]
    ops.group(choice, G, offsets=off, order=order)
    ops.matmul(x, w, off, order, y=want["y"])
    ops.matmul_grad(dy, x, w, off, order, dx=want["dx"], dw=want["dw"])
    ops.adapter(x, ws, a, b, scale, off, order, y=want["z"])
    ops.adapter_grad(dy, x, ws, a, b, scale, off, order, dx=want["dz"], da=want["da"], db=want["db"])

    got = outputs()
    p = {name: v.data_ptr() for name, v in got.items()}
    groups = hwr.hwr_groups(n, G, p["offsets"], p["order"])
    xp, dyp, wp, wsp, ap, bp, sp = (v.data_ptr() for v in (x, dy, w, ws, a, b, scale))
    hwr.hwr_group_rows(ops.ctx, n, choice.data_ptr(), None, 0, G, p["offsets"], p["order"])
    hwr.hwr_grouped_matmul(ops.ctx, groups, hwr.hwr_matmul_args(hwr.HWR_BF16, k, m, xp, 0, wp, p["y"], 0))
    hwr.hwr_grouped_matmul_grad(ops.ctx, groups,
                                hwr.hwr_matmul_grad_args(hwr.HWR_BF16, k, m, dyp, 0, xp, 0, wp, p["dx"], 0, p["dw"]))
    hwr.hwr_adapter_matmul(ops.ctx, groups, hwr.hwr_adapter_args(hwr.HWR_BF16, k, m, R, xp, 0, wsp, ap, bp, sp, p["z"], 0))
    hwr.hwr_adapter_matmul_grad(ops.ctx, groups,
                                hwr.hwr_adapter_grad_args(hwr.HWR_BF16, k, m, R, dyp, 0, xp, 0, wsp, ap, bp, sp, p["dz"], 0,
                                                          p["da"], p["db"]))
    for name in want:
        assert torch.equal(got[name], want[name]), name
    for call in (lambda: hwr.hwr_grouped_matmul(ops.ctx, groups, hwr.hwr_matmul_args(hwr.HWR_BF16, 0, m, xp, 0, wp, p["y"], 0)),
                 lambda: hwr.hwr_group_rows(ops.ctx, n, choice.data_ptr(), None, 1, G, p["offsets"], p["order"])):
        with pytest.raises(hwr.HwrError) as e:
            call()
        assert e.value.status == hwr.HWR_ERR_INVALID_ARG and hwr.hwr_ops_last_error(ops.ctx) in str(e.value)


# ---------------------------------------------------------------- infinities and NaN
WHOLE = [
    # n, G, k, m, R: whole chunks, so that operands go straight into LDS, in tiles of 32 or 64 (with
    # and without parts), 128 and 256 rows and columns, and gradients in tiles of 64, 128 and 256
    (300, 4, 256, 320, 16),
    (700, 4, 1024, 136, 40),
    (3000, 4, 128, 2048, 8),
    (4000, 16, 512, 512, 24),
    (9000, 4, 512, 2048, 32),
    (33000, 3, 1024, 512, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,G,k,m,R", WHOLE)
def test_values_stay_in_their_rows_and_groups_in_whole_chunks(ops, n, G, k, m, R, dtype):
    """A NaN or infinity in a row, or in a group's weights, changes the bits of no other
    row and of no other group's gradients."""
    t = TYPES[dtype][0]
    gen = torch.Generator("cuda").manual_seed(n)
    gid, off, order = grouped(np.random.default_rng(n).permutation(np.arange(n) % (G + 1) - 1), G)
    x, dy = rand(gen, n, k, dtype=t), rand(gen, n, m, dtype=t)
    ws, w = rand(gen, k, m, dtype=t), rand(gen, G, k, m, dtype=t)
    a, b = rand(gen, G, k, R, dtype=t), rand(gen, G, R, m, dtype=t)
    scale = 0.5 + torch.rand(G, generator=gen, device="cuda")

    def run(x, dy, w, a, b):
        o = {"y": torch.empty_like(dy), "z": torch.empty_like(dy), "dx": torch.empty_like(x), "dz": torch.empty_like(x),
             "dw": torch.empty_like(w), "da": torch.empty_like(a), "db": torch.empty_like(b)}
        ops.matmul(x, w, off, order, y=o["y"])
        ops.matmul_grad(dy, x, w, off, order, dx=o["dx"], dw=o["dw"])
        ops.adapter(x, ws, a, b, scale, off, order, y=o["z"])
        ops.adapter_grad(dy, x, ws, a, b, scale, off, order, dx=o["dz"], da=o["da"], db=o["db"])
        return o

    clean = run(x, dy, w, a, b)
    group = torch.from_numpy(gid).cuda()
    for bad in (float("nan"), float("inf"), -float("inf")):
        # the first row of group 1, the last of group 2, one in no group: all three at once
        rows = [int(np.nonzero(gid == 1)[0][0]), int(np.nonzero(gid == 2)[0][-1]), int(np.nonzero(gid == -1)[0][0])]
        xb, yb = x.clone(), dy.clone()
        xb[rows, k - 1], yb[rows, m - 1] = bad, bad
        got = run(xb, yb, w, a, b)
        rest = torch.ones(n, dtype=torch.bool, device="cuda")
        rest[rows] = False
        for q in ("y", "z", "dx", "dz"):
            assert torch.equal(got[q][rest], clean[q][rest]), (q, bad)
        others = [g for g in range(G) if g not in (1, 2)]
        for q in ("dw", "da", "db"):
            assert torch.equal(got[q][others], clean[q][others]), (q, bad)
        assert not got["y"][rows[2]].any() and not got["dx"][rows[2]].any()
        for r in rows[:2]:
            assert not torch.isfinite(got["y"][r]).any() and not torch.isfinite(got["z"][r]).any()
            assert not torch.isfinite(got["dx"][r]).any() and not torch.isfinite(got["dz"][r]).any()
        for g in (1, 2):
            # dW[e][c] = sum of x[r][e] dy[r][c]: the bad input column's row, the bad output column's column
            assert not torch.isfinite(got["dw"][g][k - 1]).any() and not torch.isfinite(got["dw"][g][:, m - 1]).any()
            assert torch.isfinite(got["dw"][g][:k - 1, :m - 1]).all()
            assert not torch.isfinite(got["da"][g]).any() and not torch.isfinite(got["db"][g]).any()
        # group 2's weights
        wb, ab, bb = w.clone(), a.clone(), b.clone()
        wb[2, 0, 0], ab[2, 1, 1], bb[2, 2, 2] = bad, bad, bad
        got = run(x, dy, wb, ab, bb)
        for q in ("y", "z", "dx", "dz"):
            assert torch.equal(got[q][group != 2], clean[q][group != 2]), (q, bad)
        for q in ("dw", "da", "db"):
            assert torch.equal(got[q][[g for g in range(G) if g != 2]], clean[q][[g for g in range(G) if g != 2]]), (q, bad)
        mine = group == 2
        assert torch.isfinite(got["y"][mine][:, 1:]).all() and not torch.isfinite(got["y"][mine][:, 0]).any()
        assert torch.equal(got["dw"][2], clean["dw"][2])
    again = run(x, dy, w, a, b)
    assert all(torch.equal(again[q], clean[q]) for q in clean)


# ---------------------------------------------------------------- forms of the low-rank intermediates
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,G,k,m,R", [(9000, 4, 264, 392, 64), (9000, 4, 261, 390, 50), (8191, 3, 136, 136, 33),
                                       (8192, 3, 136, 136, 33), (500, 3, 200, 264, 127), (9000, 2, 72, 80, 126)])
def test_ranks_of_many_rows(ops, n, G, k, m, R, dtype):
    """Ranks of 33 to 64 with two blocks of 16 rows to a workgroup (from 8,192 rows on), and above 64
    where they are no multiple of 4.  An intermediate of a bf16 call is off by 2^-16 of its value more."""
    t, u, lo = TYPES[dtype]
    gen = torch.Generator("cuda").manual_seed(n + R)
    gid, off, order = grouped(sizes_of("skew", n, G, np.random.default_rng(n)), G)
    x, dy = rand(gen, n, k, dtype=t), rand(gen, n, m, dtype=t)
    w, a, b = rand(gen, k, m, dtype=t), rand(gen, G, k, R, dtype=t), rand(gen, G, R, m, dtype=t)
    y, dx, da, db = (torch.full_like(v, 7.0) for v in (dy, x, a, b))
    ops.adapter(x, w, a, b, None, off, order, y=y)
    ops.adapter_grad(dy, x, w, a, b, None, off, order, dx=dx, da=da, db=db)
    turn = lambda v: v.transpose(-1, -2).contiguous()  # noqa: E731
    shared = np.zeros(n, np.int64)
    low, slow = product(x, a, gid)
    up, sup = product(dy, turn(b), gid)
    for got, p, wide, mid, smid, thin, width in ((y, x, w[None], low, slow, b, k), (dx, dy, turn(w)[None], up, sup, turn(a), m)):
        main, smain = product(p, wide, shared)
        add, _ = product(mid, thin, gid)
        mags, _ = product(mid.abs(), thin.abs(), gid)
        sadd, _ = product(smid, thin.abs(), gid)
        close(got, main + add, u * (main + add).abs() + (width + R + 32) * EPS * (smain + sadd) + 2 * lo * mags)
    for got, p, q, sp, sq, width in ((da, x, up, x.abs(), sup, m), (db, low, dy, slow, dy.abs(), k)):
        ref, mags, cnt = outer(p, q, gid, G)
        close(got, ref, u * ref.abs() + (width + cnt + 32) * EPS * outer(sp, sq, gid, G)[0] + 2 * lo * mags)


# ---------------------------------------------------------------- rows by group
@pytest.mark.parametrize("n,G", [(2097152, 64), (2097153, 100), (3000000, 1024), (4194305, 5)])
def test_group_of_more_than_512_blocks(ops, n, G):
    """Past 512 blocks of rows the scan over a key's blocks goes on where it left off."""
    gen = torch.Generator("cuda").manual_seed(n + G)
    choice = torch.randint(-1, G + 1, (n,), generator=gen, device="cuda", dtype=torch.int32)
    order = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    offsets = torch.full((G + 1,), -7, dtype=torch.int32, device="cuda")
    ops.group(choice, G, offsets=offsets, order=order)
    key = torch.where((choice >= 0) & (choice < G), choice, G).long()
    keys, want = torch.sort(key, stable=True)
    assert torch.equal(order.long(), want)
    assert torch.equal(offsets.long(), torch.searchsorted(keys, torch.arange(G + 1, device="cuda")))


# ---------------------------------------------------------------- graphs
def test_replays_in_order_with_other_calls(ops):
    """A graph, a second one and eager calls of one context share its work space: replays
    on another stream, ordered by events alone, leave each other's results as they should be."""
    gen = torch.Generator("cuda").manual_seed(21)
    t, n, G, k, m, R = torch.bfloat16, 1500, 4, 1001, 523, 24        # copies, intermediates, partial sums
    side, current = torch.cuda.Stream(), torch.cuda.current_stream()
    o = routed.RoutedOps(stream=side.cuda_stream)
    gid, off, order = grouped(sizes_of("skew", n, G, np.random.default_rng(2)), G)
    w, a, b = rand(gen, k, m, dtype=t), rand(gen, G, k, R, dtype=t), rand(gen, G, R, m, dtype=t)

    def inputs():
        return rand(gen, n, k, dtype=t), rand(gen, n, m, dtype=t)

    def outputs():
        return {"y": torch.full((n, m), 7.0, dtype=t, device="cuda"), "dx": torch.full((n, k), 7.0, dtype=t, device="cuda"),
                "da": torch.full_like(a, 7.0), "db": torch.full_like(b, 7.0)}

    def step(q, x, dy, out):
        q.adapter(x, w, a, b, None, off, order, y=out["y"])
        q.adapter_grad(dy, x, w, a, b, None, off, order, dx=out["dx"], da=out["da"], db=out["db"])

    held = [inputs() for _ in range(2)]
    out = [outputs() for _ in range(3)]
    side.wait_stream(current)
    step(o, *held[0], out[0])                                # work space
    graphs = []
    torch.cuda.synchronize()
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(o, *held[i], out[i])
        graphs.append(g)
    for i in range(4):
        x, dy = inputs()
        for h in held:
            for v, new in zip(h, inputs()):
                v.copy_(new)
        want = [outputs() for _ in range(3)]
        for j, (xj, dyj) in enumerate([*held, (x, dy)]):
            step(ops, xj, dyj, want[j])
        graphs[0].replay()                                   # on the current stream
        side.wait_stream(current)
        step(o, x, dy, out[2])                               # eager, on the context's
        current.wait_stream(side)
        graphs[1].replay()
        for j in range(3):
            for q in out[j]:
                assert torch.equal(out[j][q], want[j][q]), (i, j, q)
    torch.cuda.synchronize()
    del graphs
    o.close()


# ---------------------------------------------------------------- autograd
def test_in_an_autograd_function(ops):
    """The calls themselves record nothing; a Function around a product and its gradient does."""
    gen = torch.Generator("cuda").manual_seed(31)
    n, G, k, m, t = 500, 3, 72, 40, torch.float32
    gid, off, order = grouped(sizes_of("skew", n, G, np.random.default_rng(5)), G)
    x, w, c = rand(gen, n, k, dtype=t).requires_grad_(), rand(gen, G, k, m, dtype=t).requires_grad_(), rand(gen, n, m, dtype=t)
    y = torch.empty_like(c)
    ops.matmul(x, w, off, order, y=y)
    assert not y.requires_grad

    class Grouped(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w):
            ctx.save_for_backward(x, w)
            y = torch.empty_like(c)
            ops.matmul(x, w, off, order, y=y)
            return y

        @staticmethod
        def backward(ctx, dy):
            x, w = ctx.saved_tensors
            dx, dw = torch.empty_like(x), torch.empty_like(w)
            ops.matmul_grad(dy.contiguous(), x, w, off, order, dx=dx, dw=dw)
            return dx, dw

    (Grouped.apply(x, w) * c).sum().backward()
    ref, s = product(c, w.detach().transpose(1, 2).contiguous(), gid)
    close(x.grad, ref, EPS * ref.abs() + (m + 16) * EPS * s)
    ref, s, cnt = outer(x.detach(), c, gid, G)
    close(w.grad, ref, EPS * ref.abs() + (cnt + 16) * EPS * s)
