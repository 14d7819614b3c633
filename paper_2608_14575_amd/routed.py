"""Operators on a routed batch (include/hwr_ops.h) for torch tensors.

``RoutedOps`` groups the rows of a batch by the model the router chose and runs
them with that model's weights: grouped products and low-rank adapters beside a
shared projection, with their gradients.  It checks every tensor (kind, device,
shape, layout) and calls the library; every step runs in HIP kernels.

    python -m paper_2608_14575_amd.routed

routes a batch, groups it, and takes a few training steps on the adapters and
heads of the chosen models, all on the device and one stream.
"""
from __future__ import annotations

import ctypes as C
import struct

from . import hwr
from .hwr import HWR_BF16, HWR_ERR_INVALID_ARG, HWR_F32, HwrError


_MAX_INT = 2 ** 31 - 1


def _bad(name, msg):
    raise HwrError(HWR_ERR_INVALID_ARG, f"{name}: {msg}")


class _Call:
    """An entry point that takes hwr_groups and a structure of arguments: both are
    packed into one block that stays (a structure made anew for every call took
    about 1 us of a call's 10; a context is not used by two threads at once)."""
    _CODES = {C.c_int32: "i", C.c_int64: "q", C.c_void_p: "P"}

    def __init__(self, fn, args):
        codes = ["".join(self._CODES[t] for _, t in s._fields_) for s in (hwr.hwr_groups, args)]
        at = C.sizeof(hwr.hwr_groups)                  # a multiple of every alignment
        self._block = C.create_string_buffer(at + C.sizeof(args))
        self._pack = struct.Struct("@" + "".join(codes)).pack_into
        self._fn = C.cast(fn, C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_void_p, C.c_void_p))
        self._at = C.addressof(self._block), C.addressof(self._block) + at

    def __call__(self, ctx, n, G, offsets, order, args) -> int:
        try:
            self._pack(self._block, 0, n, G, offsets, order, *args)
        except struct.error as e:
            _bad("sizes", f"outside their types ({e})")
        return self._fn(ctx, *self._at)


class RoutedOps:
    """Owns one hwr_ops context on a device and stream.  Outputs are the
    caller's; calls return without waiting, ordered on the stream.  Tensors
    used on other streams have to be ordered against it by the caller.

    Matrices are bfloat16 or float32, one type in a call.  Rows of x, y, dy and
    dx may be strided (unit stride within a row); weights and their gradients are
    dense.  ``offsets`` and ``order`` are what ``group`` writes; ``order`` None means
    that row i is at place i.

    Gradients are calls of their own: nothing is recorded for torch's autograd, also where
    an input requires a gradient, and outputs are written without a new version of the tensor.
    A ``torch.autograd.Function`` around a product and its gradient records them."""

    def __init__(self, device: int = 0, stream: int = 0):
        import torch
        self._kinds = {torch.bfloat16: HWR_BF16, torch.float32: HWR_F32}
        self._i32, self._f32 = torch.int32, torch.float32
        self.device, self.stream = int(device), int(stream)
        self.ctx = hwr.hwr_ops_init(self.device, self.stream)
        self._lib = hwr.load()
        self._matmul = _Call(self._lib.hwr_grouped_matmul, hwr.hwr_matmul_args)
        self._matmul_grad = _Call(self._lib.hwr_grouped_matmul_grad, hwr.hwr_matmul_grad_args)
        self._adapter = _Call(self._lib.hwr_adapter_matmul, hwr.hwr_adapter_args)
        self._adapter_grad = _Call(self._lib.hwr_adapter_matmul_grad, hwr.hwr_adapter_grad_args)

    def close(self) -> None:
        if getattr(self, "ctx", None):
            hwr.hwr_ops_free(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def reserve(self, nbytes: int) -> None:
        """Work space for later calls (needed before calls under graph capture).  A context's
        calls and the replays of all graphs captured from it share that space: order replays
        on other streams against them, or capture each graph from a context of its own."""
        hwr.hwr_ops_reserve(self.ctx, int(nbytes))

    # ------------------------------------------------------------ checks
    # (the reason for a refusal is looked for once a tensor does not fit)
    def _refuse(self, name, t, dtype, shape):
        if t.get_device() != self.device:
            _bad(name, f"on {t.device}, expected cuda:{self.device}")
        if t.dtype is not dtype:
            _bad(name, f"dtype {t.dtype} (expected {dtype})")
        if t.shape != shape:
            _bad(name, f"shape {tuple(t.shape)}, expected {shape}")
        _bad(name, "not contiguous")

    def _dense(self, name, t, dtype, shape) -> int:
        if t.dtype is not dtype or t.shape != shape or t.get_device() != self.device or not t.is_contiguous():
            self._refuse(name, t, dtype, shape)
        return t.data_ptr()

    def _rows(self, name, t, dtype, shape):
        """Pointer and row stride of an [n][width] matrix."""
        if t.dtype is not dtype or t.shape != shape or t.get_device() != self.device:
            self._refuse(name, t, dtype, shape)
        n, width = shape
        if t.is_contiguous():
            return t.data_ptr(), width
        ld, unit = t.stride()
        if (unit != 1 and width > 1) or (ld < width and n > 1):
            _bad(name, f"strides {t.stride()}: rows must be contiguous and must not overlap")
        return t.data_ptr(), max(ld, width)

    def _x(self, x):
        """Type and shape of the rows."""
        dt, shape = x.dtype, x.shape
        if dt not in self._kinds:
            _bad("x", f"dtype {dt} (expected bfloat16 or float32)")
        if len(shape) != 2:
            _bad("x", f"{len(shape)} dimensions, expected 2")
        return dt, shape

    def _run(self, call, n, G, offsets, order, *args):
        st = call(self.ctx, n, G, self._dense("offsets", offsets, self._i32, (G + 1,)),
                  0 if order is None else self._dense("order", order, self._i32, (n,)), args)
        if st:
            raise HwrError(st, hwr.hwr_ops_last_error(self.ctx))

    # ------------------------------------------------------------ operators
    def group(self, choice, n_groups: int, *, offsets, order, table=None) -> None:
        """Rows by group: ``choice`` [n] int32, the group of each row or (with
        ``table`` [pairs] int32) the pair whose group the table holds; anything out
        of range is a row in no group.  Writes ``offsets`` [n_groups + 1] and ``order`` [n]."""
        i32, n, nt = self._i32, choice.numel(), 0 if table is None else table.numel()
        if max(n, nt, n_groups) > _MAX_INT or n_groups < 0:
            _bad("choice, table, n_groups", f"{n}, {nt}, {n_groups}: outside 32 bits")
        if table is not None and nt == 0:              # (without an address it would be no table)
            _bad("table", "empty")
        st = self._lib.hwr_group_rows(self.ctx, n, self._dense("choice", choice, i32, (n,)),
                                      None if table is None else self._dense("table", table, i32, (nt,)), nt, n_groups,
                                      self._dense("offsets", offsets, i32, (n_groups + 1,)),
                                      self._dense("order", order, i32, (n,)))
        if st:
            raise HwrError(st, hwr.hwr_ops_last_error(self.ctx))

    def _weights(self, w):
        if w.dim() != 3:
            _bad("w", f"{w.dim()} dimensions, expected 3")
        return w.shape

    def matmul(self, x, w, offsets, order=None, *, y) -> None:
        """y[r] = x[r] w[g(r)]; w [G][k][m].  A row in no group gets zeros."""
        dt, (n, k) = self._x(x)
        G, _, m = self._weights(w)
        xp, ldx = self._rows("x", x, dt, (n, k))
        yp, ldy = self._rows("y", y, dt, (n, m))
        self._run(self._matmul, n, G, offsets, order,
                  self._kinds[dt], k, m, xp, ldx, self._dense("w", w, dt, (G, k, m)), yp, ldy)

    def matmul_grad(self, dy, x, w, offsets, order=None, *, dx=None, dw=None) -> None:
        """Gradients of ``matmul``: dx [n][k] and dw [G][k][m], either may be left out."""
        dt, (n, k) = self._x(x)
        G, _, m = self._weights(w)
        dyp, lddy = self._rows("dy", dy, dt, (n, m))
        xp, ldx = self._rows("x", x, dt, (n, k))
        dxp, lddx = (0, 0) if dx is None else self._rows("dx", dx, dt, (n, k))
        self._run(self._matmul_grad, n, G, offsets, order,
                  self._kinds[dt], k, m, dyp, lddy, xp, ldx, self._dense("w", w, dt, (G, k, m)), dxp, lddx,
                  0 if dw is None else self._dense("dw", dw, dt, (G, k, m)))

    def _adapters(self, dt, k, w, a, b, scale):
        """Sizes m, G and rank, and the pointers."""
        if w.dim() != 2 or a.dim() != 3:
            _bad("w, a", f"{w.dim()} and {a.dim()} dimensions, expected 2 and 3")
        m, (G, _, R) = w.shape[1], a.shape
        return (m, G, R, self._dense("w", w, dt, (k, m)), self._dense("a", a, dt, (G, k, R)),
                self._dense("b", b, dt, (G, R, m)), 0 if scale is None else self._dense("scale", scale, self._f32, (G,)))

    def adapter(self, x, w, a, b, scale, offsets, order=None, *, y) -> None:
        """y[r] = x[r] w + scale[g] (x[r] a[g]) b[g]; w [k][m], a [G][k][rank],
        b [G][rank][m], scale [G] float32 or None (1).  A row in no group gets x[r] w."""
        dt, (n, k) = self._x(x)
        m, G, R, wp, ap, bp, sp = self._adapters(dt, k, w, a, b, scale)
        xp, ldx = self._rows("x", x, dt, (n, k))
        yp, ldy = self._rows("y", y, dt, (n, m))
        self._run(self._adapter, n, G, offsets, order, self._kinds[dt], k, m, R, xp, ldx, wp, ap, bp, sp, yp, ldy)

    def adapter_grad(self, dy, x, w, a, b, scale, offsets, order=None, *, dx=None, da=None, db=None) -> None:
        """Gradients of ``adapter``: dx [n][k], da [G][k][rank] and db [G][rank][m],
        any may be left out; w is frozen."""
        dt, (n, k) = self._x(x)
        m, G, R, wp, ap, bp, sp = self._adapters(dt, k, w, a, b, scale)
        dyp, lddy = self._rows("dy", dy, dt, (n, m))
        xp, ldx = self._rows("x", x, dt, (n, k))
        dxp, lddx = (0, 0) if dx is None else self._rows("dx", dx, dt, (n, k))
        self._run(self._adapter_grad, n, G, offsets, order,
                  self._kinds[dt], k, m, R, dyp, lddy, xp, ldx, wp, ap, bp, sp, dxp, lddx,
                  0 if da is None else self._dense("da", da, dt, (G, k, R)),
                  0 if db is None else self._dense("db", db, dt, (G, R, m)))


def example(steps: int = 5, n: int = 4096, seed: int = 7) -> list:
    """Routes n queries, groups them by the chosen pair's model, and trains, on
    the grouped rows, one low-rank adapter per model beside a shared projection
    and one output head per model towards random targets; returns the losses."""
    import numpy as np
    import torch
    from . import synth

    dev, s = torch.device("cuda:0"), torch.cuda.current_stream()
    sp = synth.spec("C3", n_queries=n)
    pb, st, qs = synth.make_problem(sp, seed), synth.make_state(sp, seed), synth.make_queries(sp, seed)
    router = hwr.Router.from_problem(pb, stream=s.cuda_stream)
    ops = RoutedOps(stream=s.cuda_stream)
    router.update(st)

    # where each query goes
    emb = torch.from_numpy(qs.emb_bits.view(np.int16)).to(dev)
    choice = torch.empty(n, dtype=torch.int32, device=dev)
    router.route(emb, *(torch.from_numpy(v).to(dev) for v in (qs.input_len, qs.expected_out_len, qs.slo_s)),
                 mem=hwr.HWR_MEM_DEVICE, choice=choice)

    # the rows of each model
    G = sp.n_models
    offsets = torch.empty(G + 1, dtype=torch.int32, device=dev)
    order = torch.empty(n, dtype=torch.int32, device=dev)
    ops.group(choice, G, table=torch.from_numpy(pb.dep_model).to(dev, torch.int32), offsets=offsets, order=order)

    # h = x W + s (x A_g) B_g, out = h H_g; loss = |out - target|^2 / 2 per row
    g = torch.Generator(dev).manual_seed(seed)
    bf = torch.bfloat16
    k, m, R, o = sp.embed_dim, 1024, 16, 128

    def weights(*shape, std):
        return (torch.randn(shape, generator=g, device=dev) * std).to(bf)

    x = emb.view(bf).mul(k ** 0.5)
    w = weights(k, m, std=k ** -0.5)
    p = {"a": weights(G, k, R, std=k ** -0.5), "b": torch.zeros(G, R, m, dtype=bf, device=dev),
         "head": weights(G, m, o, std=m ** -0.5)}
    master = {name: v.float() for name, v in p.items()}
    scale = torch.full((G,), 2.0, device=dev)
    target = torch.randn((n, o), generator=g, device=dev)
    h, out = torch.empty(n, m, dtype=bf, device=dev), torch.empty(n, o, dtype=bf, device=dev)
    dh = torch.empty_like(h)
    grad = {name: torch.empty_like(v) for name, v in p.items()}
    # a step that a model of few rows and one of many both bear
    rate = 0.25 / (m + offsets[1:] - offsets[:-1]).float()[:, None, None]
    losses = []
    for _ in range(steps):
        ops.adapter(x, w, p["a"], p["b"], scale, offsets, order, y=h)
        ops.matmul(h, p["head"], offsets, order, y=out)
        d = out.float() - target
        losses.append(float(d.square().mean()) / 2)
        ops.matmul_grad(d.to(bf), h, p["head"], offsets, order, dx=dh, dw=grad["head"])
        ops.adapter_grad(dh, x, w, p["a"], p["b"], scale, offsets, order, da=grad["a"], db=grad["b"])
        for name in p:
            master[name] -= rate * grad[name].float()
            p[name].copy_(master[name])
    ops.close()
    router.close()
    return losses


if __name__ == "__main__":
    for i, loss in enumerate(example()):
        print(f"step {i}: loss {loss:.4f}", flush=True)
