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
_ACTS = {"none": hwr.HWR_ACT_NONE, "relu": hwr.HWR_ACT_RELU, "silu": hwr.HWR_ACT_SILU, "gelu": hwr.HWR_ACT_GELU}


def _bad(name, msg):
    raise HwrError(HWR_ERR_INVALID_ARG, f"{name}: {msg}")


class _Call:
    """An entry point that takes hwr_groups and a structure of arguments: both are
    packed into one block that stays (a structure made anew for every call took
    about 1 us of a call's 10; a context is not used by two threads at once)."""
    _CODES = {C.c_int32: "i", C.c_int64: "q", C.c_void_p: "P", C.c_float: "f", C.c_double: "d", C.c_uint64: "Q"}

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


class _Args(_Call):
    """The same for an entry point without groups."""

    def __init__(self, fn, args):
        self._block = C.create_string_buffer(C.sizeof(args))
        self._pack = struct.Struct("@" + "".join(self._CODES[t] for _, t in args._fields_)).pack_into
        self._fn = C.cast(fn, C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_void_p))
        self._at = C.addressof(self._block)

    def __call__(self, ctx, *args) -> int:
        try:
            self._pack(self._block, 0, *args)
        except (struct.error, OverflowError) as e:
            _bad("sizes", f"outside their types ({e})")
        return self._fn(ctx, self._at)


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
        self._linear = _Call(self._lib.hwr_grouped_linear, hwr.hwr_linear_args)
        self._linear_grad = _Call(self._lib.hwr_grouped_linear_grad, hwr.hwr_linear_grad_args)
        self._adapter = _Call(self._lib.hwr_adapter_matmul, hwr.hwr_adapter_args)
        self._adapter_grad = _Call(self._lib.hwr_adapter_matmul_grad, hwr.hwr_adapter_grad_args)
        self._log_probs = _Args(self._lib.hwr_log_probs, hwr.hwr_log_probs_args)
        self._log_probs_grad = _Args(self._lib.hwr_log_probs_grad, hwr.hwr_log_probs_grad_args)

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

    def _act(self, act) -> int:
        if act not in _ACTS:
            _bad("act", f"{act!r}, expected one of {sorted(_ACTS)}")
        return _ACTS[act]

    def linear(self, x, w, offsets, order=None, *, bias=None, act="none", residual=None, y, z=None) -> None:
        """A layer: z[r] = x[r] w[g(r)] + bias[g(r)], y[r] = act(z[r]) + residual[r]; w [G][k][m],
        bias [G][m], act "none", "relu", "silu" or "gelu" (of the normal distribution).  ``z``, which
        ``linear_grad`` reads, is written where it is given.  A row in no group gets the residual, or zeros."""
        dt, (n, k) = self._x(x)
        G, _, m = self._weights(w)
        xp, ldx = self._rows("x", x, dt, (n, k))
        rp, ldr = (0, 0) if residual is None else self._rows("residual", residual, dt, (n, m))
        yp, ldy = self._rows("y", y, dt, (n, m))
        zp, ldz = (0, 0) if z is None else self._rows("z", z, dt, (n, m))
        self._run(self._linear, n, G, offsets, order,
                  self._kinds[dt], k, m, self._act(act), xp, ldx, self._dense("w", w, dt, (G, k, m)),
                  0 if bias is None else self._dense("bias", bias, dt, (G, m)), rp, ldr, yp, ldy, zp, ldz)

    def linear_grad(self, dy, x, w, offsets, order=None, *, act="none", z=None, dx=None, dw=None, dbias=None) -> None:
        """Gradients of ``linear``: dx [n][k], dw [G][k][m] and dbias [G][m], any may be left out (the
        residual's is dy); ``z`` is needed with an activation."""
        dt, (n, k) = self._x(x)
        G, _, m = self._weights(w)
        dyp, lddy = self._rows("dy", dy, dt, (n, m))
        zp, ldz = (0, 0) if z is None else self._rows("z", z, dt, (n, m))
        xp, ldx = self._rows("x", x, dt, (n, k))
        dxp, lddx = (0, 0) if dx is None else self._rows("dx", dx, dt, (n, k))
        self._run(self._linear_grad, n, G, offsets, order,
                  self._kinds[dt], k, m, self._act(act), dyp, lddy, zp, ldz, xp, ldx, self._dense("w", w, dt, (G, k, m)),
                  dxp, lddx, 0 if dw is None else self._dense("dw", dw, dt, (G, k, m)),
                  0 if dbias is None else self._dense("dbias", dbias, dt, (G, m)))

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

    # ------------------------------------------------------------ from logits
    def _optional(self, name, t, dtype, shape) -> int:
        return 0 if t is None else self._dense(name, t, dtype, shape)

    def log_probs(self, x, token=None, *, scale=1.0, logp=None, lse=None, entropy=None, top_logp=None, top_token=None) -> None:
        """Of rows of logits x [n][m], scaled: ``lse`` [n], the log probability ``logp`` [n] of
        ``token`` [n] int32 (0 where it is outside [0, m)), ``entropy`` [n], and the most likely
        tokens, ``top_token`` [n][top] int32 and ``top_logp`` [n][top], top at most 32.  Outputs are
        float32, any may be left out.  Tokens at -inf are not allowed ones."""
        dt, (n, m) = self._x(x)
        f32, i32 = self._f32, self._i32
        xp, ldx = self._rows("x", x, dt, (n, m))
        some = top_token if top_token is not None else top_logp
        if some is not None and some.dim() != 2:
            _bad("top_token, top_logp", f"{some.dim()} dimensions, expected 2")
        top = 0 if some is None else some.shape[1]
        if some is not None and top == 0:
            _bad("top_token, top_logp", "no columns")
        st = self._log_probs(self.ctx, self._kinds[dt], n, m, top, scale, xp, ldx, self._optional("token", token, i32, (n,)),
                             self._optional("logp", logp, f32, (n,)), self._optional("lse", lse, f32, (n,)),
                             self._optional("entropy", entropy, f32, (n,)),
                             self._optional("top_logp", top_logp, f32, (n, top)),
                             self._optional("top_token", top_token, i32, (n, top)))
        if st:
            raise HwrError(st, hwr.hwr_ops_last_error(self.ctx))

    def log_probs_grad(self, x, token, lse, dlogp, *, entropy=None, dentropy=None, scale=1.0, dlogits) -> None:
        """Gradient of the logits x [n][m] from those of ``log_probs``' logp (``dlogp`` [n]; None,
        with token: none) and entropy (``dentropy`` [n], with ``entropy``).  ``dlogits`` may be x."""
        dt, (n, m) = self._x(x)
        f32 = self._f32
        xp, ldx = self._rows("x", x, dt, (n, m))
        dxp, lddx = self._rows("dlogits", dlogits, dt, (n, m))
        st = self._log_probs_grad(self.ctx, self._kinds[dt], n, m, scale, xp, ldx,
                                  self._optional("token", token, self._i32, (n,)), self._dense("lse", lse, f32, (n,)),
                                  self._optional("dlogp", dlogp, f32, (n,)), self._optional("entropy", entropy, f32, (n,)),
                                  self._optional("dentropy", dentropy, f32, (n,)), dxp, lddx)
        if st:
            raise HwrError(st, hwr.hwr_ops_last_error(self.ctx))


class AdamW:
    """AdamW over many tensors at once, in one launch a step, on the stream of a ``RoutedOps``.

    ``params`` and ``grads`` are lists of dense tensors, of one type (bfloat16 or float32), pair by pair of
    one size; the same tensors are read and written at every step, in the memory that they have here (one that is given
    other memory later, as by ``p.data = ...``, needs a new object).  bfloat16 weights are stepped through
    float32 masters (``master=True``) or alone, rounded up or down at random.  States have 32
    bits or 8 (``bits``): float8_e4m3fn with a float32 scale for every 256 values, the root of the second
    moment in place of it, rounded at random, from ``seed``, the step and the value's place (the second moment's
    noise: a third of it, 5% above on the mean; include/hwr_ops.h has the figures).

    ``state`` is a dict of lists, as the attribute of the same name: "m" and "v", with 8 bits "m_scale" and
    "v_scale", with masters "master"; left out, it is made here (zeros, and copies of the weights as they are on torch's
    current stream) and there before any step.

    ``steps``, the number of steps done, is counted up by ``step``: an int, or a device tensor of one int64, which
    a captured ``step`` needs.  ``lr`` may be a device tensor of one float32 then.  Both,
    ``betas``, ``eps`` and ``weight_decay`` may be changed between steps (a captured step keeps what
    it was captured with, but for the contents of the tensors).

    As with the operators, torch does not see the writes (no new version of a tensor).  Steps of one object are
    ordered among each other by the caller, on whatever streams they run.  An object is made, closed and dropped (which
    waits for the device) while no stream is captured."""

    def __init__(self, ops, params, grads, *, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, bits=32, master=False,
                 state=None, steps=0, seed=0):
        import torch
        self._handle = None
        if torch.cuda.is_current_stream_capturing():
            raise HwrError(hwr.HWR_ERR_STATE, "AdamW: torch's current stream is being captured: make it before")
        params, grads = list(params), list(grads)
        if len(params) != len(grads):
            _bad("grads", f"{len(grads)} tensors for {len(params)} weights")
        dt = params[0].dtype if params else torch.float32
        if dt not in ops._kinds:
            _bad("params", f"dtype {dt} (expected bfloat16 or float32)")
        if state is None:
            if bits not in (8, 32):
                _bad("bits", f"{bits} (expected 8 or 32)")
            if master and dt is torch.float32:
                _bad("master", "for bfloat16 weights")
            state = self._make_state(torch, params, bits, master)
            made = torch.cuda.current_stream(ops.device)
            if made.cuda_stream != ops.stream:         # (steps run on the other)
                made.synchronize()
        state = {k: list(v) for k, v in state.items()}
        bits = 8 if "m_scale" in state else 32
        kind = torch.float8_e4m3fn if bits == 8 else torch.float32
        kinds = {"m": kind, "v": kind}
        if bits == 8:
            kinds.update(m_scale=torch.float32, v_scale=torch.float32)
        if "master" in state:
            kinds["master"] = torch.float32
        if set(state) != set(kinds):
            _bad("state", f"{sorted(state)}, expected {sorted(kinds)}")
        for k, v in state.items():
            if len(v) != len(params):
                _bad(k, f"{len(v)} tensors for {len(params)} weights")
        values, address = [], self._address
        lists = [(k, state[k], kinds[k], k.endswith("scale")) if k in kinds else None
                 for k in ("master", "m", "v", "m_scale", "v_scale")]
        for i, (p, g) in enumerate(zip(params, grads)):
            n = p.numel()
            values += (n, address(ops, "params", i, p, dt, n), address(ops, "grads", i, g, dt, n))
            for q in lists:
                values.append(0 if q is None else address(ops, q[0], i, q[1][i], q[2], (n + 255) // 256 if q[3] else n))
        table = (hwr.hwr_adamw_tensor * len(params))()
        struct.pack_into(f"@{len(values)}Q", table, 0, *values)        # (the structure: eight numbers of 64 bits)
        config = hwr.hwr_adamw_config(ops._kinds[dt], bits, len(params), table)
        self._handle = hwr.hwr_adamw_init(ops.ctx, config)
        self.ops, self.params, self.grads, self.state = ops, params, grads, state
        # (steps go by addresses: the memory stays, also where a tensor is given other)
        self._memory = [t.untyped_storage() for q in (params, grads, *state.values()) for t in q]
        self.lr, self.betas, self.eps, self.weight_decay, self.steps, self.seed = lr, betas, eps, weight_decay, steps, seed
        self._i64 = torch.int64
        self._args = _Args(ops._lib.hwr_adamw_step, hwr.hwr_adamw_args)
        fn, handle = C.cast(ops._lib.hwr_adamw_step, C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_void_p, C.c_void_p)), self._handle
        self._args._fn = lambda ctx, at: fn(ctx, handle, at)       # (not of self, which would stay until its cycle is collected)

    @staticmethod
    def _address(ops, name, i, t, dtype, n):
        if t.get_device() != ops.device:
            _bad(f"{name}[{i}]", f"on {t.device}, expected cuda:{ops.device}")
        if t.dtype is not dtype or t.numel() != n:
            _bad(f"{name}[{i}]", f"{t.numel()} of {t.dtype}, expected {n} of {dtype}")
        if not t.is_contiguous():
            _bad(f"{name}[{i}]", "not contiguous")
        return t.data_ptr()

    @staticmethod
    def _make_state(torch, params, bits, master):
        def zeros(p, n, dtype):
            return torch.zeros(n, dtype=dtype, device=p.device)

        kind = torch.float8_e4m3fn if bits == 8 else torch.float32
        state = {k: [zeros(p, p.shape, kind) for p in params] for k in ("m", "v")}
        if bits == 8:
            state.update({k: [zeros(p, (p.numel() + 255) // 256, torch.float32) for p in params] for k in ("m_scale", "v_scale")})
        if master:
            state["master"] = [p.detach().float() for p in params]
        return state

    def close(self) -> None:
        if getattr(self, "_handle", None):
            hwr.hwr_adamw_free(self._handle)           # (waits for the device)
            self._handle, self._memory = None, []

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def step(self) -> None:
        """One step of all tensors, queued on the stream of the ``RoutedOps``."""
        if not self._handle:
            _bad("AdamW", "closed")
        ops, steps, lr, (b1, b2) = self.ops, self.steps, self.lr, self.betas
        number, counter, rate = 0, 0, 0
        if not hasattr(steps, "data_ptr"):
            number = int(steps) + 1
        else:
            counter = ops._dense("steps", steps.view(1) if steps.dim() == 0 else steps, self._i64, (1,))
        if hasattr(lr, "data_ptr"):
            rate, lr = ops._dense("lr", lr.view(1) if lr.dim() == 0 else lr, ops._f32, (1,)), 0.0
        st = self._args(ops.ctx, lr, b1, b2, self.eps, self.weight_decay, self.seed & 0xFFFFFFFFFFFFFFFF, number, counter, rate)
        if st:
            raise HwrError(st, hwr.hwr_ops_last_error(ops.ctx))
        if not counter:
            self.steps = number


def _routed(n, seed):
    """Routes n queries and groups them by the chosen pair's model: the operators, the number of models, the
    queries' embeddings as rows, their groups, and what to close at the end."""
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
    return ops, G, emb.view(torch.bfloat16).mul(sp.embed_dim ** 0.5), offsets, order, router


def example(steps: int = 5, n: int = 4096, seed: int = 7) -> list:
    """Routes n queries, groups them by the chosen pair's model, and trains, on
    the grouped rows, one low-rank adapter per model beside a shared projection
    and one output head per model towards random targets; returns the losses."""
    import torch

    ops, G, x, offsets, order, router = _routed(n, seed)
    dev = x.device

    # h = x W + s (x A_g) B_g, out = h H_g; loss = |out - target|^2 / 2 per row
    g = torch.Generator(dev).manual_seed(seed)
    bf = torch.bfloat16
    k, m, R, o = x.shape[1], 1024, 16, 128

    def weights(*shape, std):
        return (torch.randn(shape, generator=g, device=dev) * std).to(bf)

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


def train_tokens(steps: int = 5, n: int = 4096, tokens: int = 4096, seed: int = 7):
    """Routes n queries and trains the models that they went to, on one token each: an adapter beside a shared projection,
    a layer with bias and SiLU, and a head with the log probabilities of given tokens; bf16 weights alone, AdamW
    with states in 8 bits.  The step is captured into a graph and replayed.  Returns the loss before every step, the
    weights and their last gradients."""
    import torch

    ops, G, x, offsets, order, router = _routed(n, seed)
    ops.close()
    dev, bf, stream = x.device, torch.bfloat16, torch.cuda.Stream()
    ops = RoutedOps(stream=stream.cuda_stream)
    g = torch.Generator(dev).manual_seed(seed)
    k, m, h, R = x.shape[1], 1024, 512, 16

    def weights(*shape, std):
        return (torch.randn(shape, generator=g, device=dev) * std).to(bf)

    w, scale = weights(k, m, std=k ** -0.5), torch.full((G,), 2.0, device=dev)
    p = {"a": weights(G, k, R, std=k ** -0.5), "b": weights(G, R, m, std=1e-2), "layer": weights(G, m, h, std=m ** -0.5),
         "layer_bias": weights(G, h, std=0.1), "head": weights(G, h, tokens, std=h ** -0.5), "head_bias": weights(G, tokens, std=0.1)}
    grad = {name: torch.empty_like(v) for name, v in p.items()}
    token = torch.randint(0, tokens, (n,), generator=g, device=dev, dtype=torch.int32)

    def rows(width, dtype=bf):
        return torch.empty((n, width), dtype=dtype, device=dev)

    y, z, hidden, logits = rows(m), rows(h), rows(h), rows(tokens)
    dy, dhidden = rows(m), rows(h)
    logp, lse = torch.empty(n, device=dev), torch.empty(n, device=dev)
    dlogp = torch.full((n,), -1.0 / n, device=dev)               # loss: minus the mean log probability
    opt = AdamW(ops, list(p.values()), list(grad.values()), lr=1e-2, weight_decay=0.0, bits=8, seed=seed,
                steps=torch.zeros(1, dtype=torch.int64, device=dev))
    stream.wait_stream(torch.cuda.current_stream())              # (all of these were filled there)

    def step():
        ops.adapter(x, w, p["a"], p["b"], scale, offsets, order, y=y)
        ops.linear(y, p["layer"], offsets, order, bias=p["layer_bias"], act="silu", y=hidden, z=z)
        ops.linear(hidden, p["head"], offsets, order, bias=p["head_bias"], y=logits)
        ops.log_probs(logits, token, logp=logp, lse=lse)
        ops.log_probs_grad(logits, token, lse, dlogp, dlogits=logits)
        ops.linear_grad(logits, hidden, p["head"], offsets, order, dx=dhidden, dw=grad["head"], dbias=grad["head_bias"])
        ops.linear_grad(dhidden, y, p["layer"], offsets, order, act="silu", z=z, dx=dy, dw=grad["layer"], dbias=grad["layer_bias"])
        ops.adapter_grad(dy, x, w, p["a"], p["b"], scale, offsets, order, da=grad["a"], db=grad["b"])
        opt.step()

    losses, graph = [], None
    for _ in range(steps):
        if graph:
            graph.replay()
        else:
            step()                                               # (the first makes the work space)
        torch.cuda.synchronize()
        losses.append(-float(logp.mean()))
        if graph is None:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                step()
    del graph
    opt.close()
    ops.close()
    router.close()
    return losses, p, grad


if __name__ == "__main__":
    for i, loss in enumerate(example()):
        print(f"step {i}: loss {loss:.4f}", flush=True)
    for i, loss in enumerate(train_tokens()[0]):
        print(f"tokens, step {i}: loss {loss:.4f}", flush=True)
