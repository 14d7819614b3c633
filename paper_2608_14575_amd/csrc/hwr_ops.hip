// Host side of the operators on a routed batch (hwr_ops.h): validation, work
// space and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <string>
#include <vector>

#include "c_boundary.hpp"
#include "hwr_ops.h"
#include "ops_internal.hpp"

using namespace hwr;

struct hwr_ops {
    int dev = 0, cus = 0;
    hipStream_t stream = nullptr;
    void *zeros = nullptr;
    // Work space: the last block is in use.  Blocks grow by powers of two and stay
    // until hwr_ops_free: captured graphs hold their addresses.
    std::vector<void *> blocks;
    uint64_t size = 0;
    std::string err;
};

namespace {

thread_local std::string g_ops_error;

constexpr int kMaxWidth = 65536;
constexpr int kMaxRank = 128;
constexpr int kMaxRows = INT32_MAX - 511;    // places are counted in 32 bits, up to a few tiles past the last
constexpr uint64_t kZeroBytes = 256;

hwr_status fail(hwr_ops *c, hwr_status s, const std::string &msg) {
    (c ? c->err : g_ops_error) = msg;
    return s;
}
hwr_status invalid(hwr_ops *c, const char *msg) { return fail(c, HWR_ERR_INVALID_ARG, msg); }

// (The runtime keeps the error until it is asked for: the next launch would report it again.)
hwr_status hip_fail(hwr_ops *c, hipError_t e, const char *what) {
    (void)hipGetLastError();
    std::string m = std::string(what) + ": " + hipGetErrorName(e) + " (" + hipGetErrorString(e) + ")";
    return fail(c, e == hipErrorOutOfMemory ? HWR_ERR_OOM : HWR_ERR_HIP, m);
}

#define OPS_HIP(ctx, call)                                           \
    do {                                                             \
        hipError_t e_ = (call);                                      \
        if (e_ != hipSuccess) return hip_fail((ctx), e_, #call);     \
    } while (0)

void release(hwr_ops *c) {
    for (void *p : c->blocks) (void)hipFree(p);
    if (c->zeros) (void)hipFree(c->zeros);
    delete c;
}

// Makes a device current for a scope; the caller's is current again after it.
class OnDevice {
  public:
    explicit OnDevice(int dev) {
        error = hipGetDevice(&before_);
        if (error == hipSuccess && before_ != dev) {
            error = hipSetDevice(dev);
            changed_ = error == hipSuccess;
        }
    }
    ~OnDevice() {
        if (changed_) (void)hipSetDevice(before_);
    }
    OnDevice(const OnDevice &) = delete;
    OnDevice &operator=(const OnDevice &) = delete;
    hipError_t error;

  private:
    int before_ = 0;
    bool changed_ = false;
};

#define OPS_ON_DEVICE(ctx, dev)    \
    const OnDevice on_device(dev); \
    if (on_device.error != hipSuccess) return hip_fail((ctx), on_device.error, "hipSetDevice")

// At least `bytes` of work space at *out.
hwr_status workspace(hwr_ops *c, uint64_t bytes, char **out) {
    if (bytes > c->size) {
        hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
        if (c->stream) OPS_HIP(c, hipStreamIsCapturing(c->stream, &cap));
        if (cap != hipStreamCaptureStatusNone)
            return fail(c, HWR_ERR_STATE, "this call needs more work space than the context has, and its stream is being "
                        "captured: hwr_ops_reserve " + std::to_string(bytes) + " bytes before");
        uint64_t size = c->size ? c->size : uint64_t(1) << 20;
        while (size < bytes) size *= 2;
        c->blocks.reserve(c->blocks.size() + 1);
        void *p = nullptr;
        hipError_t e = hipMalloc(&p, size);
        if (e == hipErrorOutOfMemory && size > bytes) {
            (void)hipGetLastError();
            size = bytes;
            e = hipMalloc(&p, size);
        }
        if (e != hipSuccess) return hip_fail(c, e, "work space");
        c->blocks.push_back(p);
        c->size = size;
    }
    *out = c->blocks.empty() ? nullptr : static_cast<char *>(c->blocks.back());
    return HWR_OK;
}

hwr_status init_impl(int32_t device, void *stream, hwr_ops **out) {
    if (!out) return invalid(nullptr, "out is NULL");
    *out = nullptr;
    int ndev = 0;
    hipError_t e = hipGetDeviceCount(&ndev);
    if (e != hipSuccess || ndev < 1) {
        (void)hipGetLastError();
        return fail(nullptr, HWR_ERR_HIP, "no HIP device available");
    }
    if (device < 0 || device >= ndev) return invalid(nullptr, "device ordinal out of range");
    hipDeviceProp_t prop;
    e = hipGetDeviceProperties(&prop, device);
    if (e != hipSuccess) return hip_fail(nullptr, e, "hipGetDeviceProperties");
    if (std::strncmp(prop.gcnArchName, "gfx950", 6) != 0)
        return fail(nullptr, HWR_ERR_UNSUPPORTED, std::string("library is built for gfx950, device is ") + prop.gcnArchName);
    OPS_ON_DEVICE(nullptr, device);
    hwr_ops *c = new hwr_ops();
    c->dev = device;
    c->cus = prop.multiProcessorCount;
    c->stream = static_cast<hipStream_t>(stream);
    e = hipMalloc(&c->zeros, kZeroBytes);
    if (e == hipSuccess) e = hipMemset(c->zeros, 0, kZeroBytes);
    if (e == hipSuccess) e = hipDeviceSynchronize();
    if (e != hipSuccess) {
        release(c);
        return hip_fail(nullptr, e, "context memory");
    }
    *out = c;
    return HWR_OK;
}

// ---------------------------------------------------------------- checks
bool misaligned(int32_t dtype, std::initializer_list<const void *> ptrs) {
    for (const void *p : ptrs)
        if (reinterpret_cast<uintptr_t>(p) & (dtype == HWR_BF16 ? 1 : 3)) return true;
    return false;
}
// Null when sound, else what is wrong.
const char *check_groups(const hwr_groups *g) {
    if (!g) return "groups is NULL";
    if (g->n < 0 || g->n > kMaxRows) return "rows outside 0..2147483136";
    if (g->n_groups < 1 || g->n_groups > kMaxPairs) return "n_groups outside 1..1024";
    if (!g->offsets) return "offsets is NULL";
    if (misaligned(HWR_F32, {g->offsets, g->order})) return "offsets or order is not aligned to its elements";
    return nullptr;
}
const char *check_shape(int32_t dtype, int32_t k, int32_t m) {
    if (dtype != HWR_F32 && dtype != HWR_BF16) return "unknown dtype";
    if (k < 1 || k > kMaxWidth || m < 1 || m > kMaxWidth) return "k or m outside 1..65536";
    return nullptr;
}
const char *check_rank(int32_t rank) { return rank < 1 || rank > kMaxRank ? "rank outside 1..128" : nullptr; }
bool bad_ld(int64_t ld, int32_t width) { return ld != 0 && ld < width; }
int64_t dense(int64_t ld, int32_t width) { return ld ? ld : width; }
GroupsArg groups_arg(const hwr_groups *g) { return {g->n, g->n_groups, g->offsets, g->order}; }

int rank_blocks(int rank) { return (rank + kRankBlock - 1) / kRankBlock; }
uint64_t low_bytes(int n, int rank) { return static_cast<uint64_t>(n) * rank_blocks(rank) * kLowBytes; }

// ---------------------------------------------------------------- odd widths
// Matrices of a call whose rows are not whole, aligned chunks, and their padded
// copies in the work space.
class Pads {
  public:
    explicit Pads(bool bf16) : bf16_(bf16) { args_.count = 0; }
    // The matrix at *src ([rows][width], rows *ld elements apart), if it needs a copy.  One
    // that this call does not use counts all the same: what an output is made of, and so its
    // bits, does not depend on which others are asked for.
    void add(const void **src, int64_t *ld, int64_t rows, int width, bool used = true) {
        const int64_t chunk = padded_width(bf16_, 1);
        if ((reinterpret_cast<uintptr_t>(*src) & 15) == 0 && *ld % chunk == 0 && width % chunk == 0) return;
        const PadArgs::Matrix m{*src, nullptr, rows, *ld, width};
        all_ += size(m);
        if (!used) return;
        slots_[args_.count] = {src, ld};
        args_.m[args_.count++] = m;
    }
    // Whether copies are worth their time for products of so many operations.  If so they lie
    // past the first *used bytes of the work space (and are counted in), and the matrices' row
    // strides become theirs, their addresses distances from the work space's start.  A copy is a
    // pass over the matrix (3.5 TB/s, 3 us to launch); without it operands pass through
    // registers, which takes about twice the time of the products at their ordinary rate,
    // and more where a weight gradient is among them.  (bf16, us with / without copies: adapter
    // 15,945 x 1176 x 1046 121.9 / 134.9, 8,413 x 1385 x 320 53.8 / 47.4; grouped gradients 5,198 x 427 x
    // 1058 in 20 groups 58.9 / 72.4, 116 x 1061 x 278 in 32 groups 44.8 / 31.8.)
    bool plan(double flops, bool gradients, uint64_t *used) {
        const double rate = (bf16_ ? 6e14 : 8e13) / (gradients ? 2 : 1);
        if (all_ == 0 || all_ / 1.75e12 + 3e-6 >= flops / rate) {
            args_.count = 0;
            return false;
        }
        for (int i = 0; i < args_.count; ++i) {
            at_[i] = *used;
            *used += size(args_.m[i]);
            *slots_[i].src = reinterpret_cast<const void *>(at_[i]);
            *slots_[i].ld = padded_width(bf16_, args_.m[i].width);
        }
        return true;
    }
    // Makes the copies that were planned; the matrices' addresses become theirs.
    hwr_status copy(hwr_ops *c, char *ws) {
        if (args_.count == 0) return HWR_OK;
        for (int i = 0; i < args_.count; ++i) *slots_[i].src = args_.m[i].dst = ws + at_[i];
        OPS_HIP(c, launch_pad(bf16_, args_, c->stream));
        return HWR_OK;
    }

  private:
    struct Slot {
        const void **src;
        int64_t *ld;
    };
    uint64_t size(const PadArgs::Matrix &m) const {
        return (static_cast<uint64_t>(m.rows) * padded_width(bf16_, m.width) * (bf16_ ? 2 : 4) + 255) / 256 * 256;
    }
    bool bf16_;
    uint64_t all_ = 0;
    PadArgs args_;
    Slot slots_[kMaxPads];
    uint64_t at_[kMaxPads];
};

// A product by row: w has `lines` rows of `ldw` elements a group, or one group for all rows (shared).
RowsArgs rows_args(hwr_ops *c, const hwr_groups *g, bool ks, bool padded, const void *x, int64_t ldx, int k, const void *w,
                   int64_t ldw, int lines, bool shared, int m, void *y, int64_t ldy) {
    RowsArgs r{};
    r.g = groups_arg(g);
    r.k = k;
    r.m = m;
    r.x = x;
    r.ldx = ldx;
    r.w = w;
    r.w_stride = shared ? 0 : lines * ldw;
    r.ldw = static_cast<int>(ldw);
    r.mw = ks ? r.ldw : m;
    r.padded = padded;
    r.y = y;
    r.ldy = ldy;
    r.zeros = c->zeros;
    r.m_pad = (m + 3) / 4 * 4;
    return r;
}
uint64_t rows_bytes(hwr_ops *c, bool bf16, RowsKind kind, bool ks, const RowsArgs &r) {
    const int parts = rows_plan(bf16, kind, ks, r, c->cus).parts;
    return parts > 1 ? static_cast<uint64_t>(parts) * r.g.n * r.m_pad * sizeof(float) : 0;
}
// With its partial sums (rows_bytes) at `partial`.
hwr_status rows(hwr_ops *c, bool bf16, RowsKind kind, bool ks, RowsArgs r, char *partial) {
    r.parts = rows_plan(bf16, kind, ks, r, c->cus).parts;
    r.partial = reinterpret_cast<float *>(partial);
    OPS_HIP(c, launch_rows(bf16, kind, ks, r, c->cus, c->stream));
    if (r.parts == 1) return HWR_OK;
    FewArgs f{};
    f.g = r.g;
    f.m = r.m;
    f.m_pad = r.m_pad;
    f.y = r.y;
    f.ldy = r.ldy;
    f.parts = r.parts;
    f.partial = r.partial;
    OPS_HIP(c, launch_join(bf16, f, c->stream));
    return HWR_OK;
}

// out[g] = P^T Q, with its partial sums (weight_grad_bytes) at `partial`.
uint64_t weight_grad_bytes(hwr_ops *c, bool bf16, ColsKind kind, const ColsArgs &w) {
    const int parts = cols_plan(bf16, kind, w, c->cus).parts;
    return parts > 1 ? static_cast<uint64_t>(parts) * w.g.G * w.np * w.nq * sizeof(float) : 0;
}
hwr_status weight_grad(hwr_ops *c, bool bf16, ColsKind kind, ColsArgs w, char *partial) {
    w.parts = cols_plan(bf16, kind, w, c->cus).parts;
    w.partial = reinterpret_cast<float *>(partial);
    w.zeros = c->zeros;
    OPS_HIP(c, launch_cols(bf16, kind, w, c->cus, c->stream));
    return HWR_OK;
}

constexpr int kLowParts = 4;      // parts of the shrink's contraction, few rows

// Few rows: the weights are streamed (launch_few), with its partial sums in the work space.
hwr_status few(hwr_ops *c, FewArgs f, bool bf16, bool adapter) {
    f.m_pad = (f.m + 3) / 4 * 4;
    f.parts = few_parts(f.g.n, f.g.G, f.k, f.m, bf16, adapter, c->cus);
    f.low_parts = kLowParts;
    const uint64_t sums = adapter || f.parts > 1 ? static_cast<uint64_t>(f.parts) * f.g.n * f.m_pad : 0;
    const uint64_t lows = adapter ? static_cast<uint64_t>(f.low_parts) * f.g.n * f.rank : 0;
    char *ws = nullptr;
    if (hwr_status st = workspace(c, (sums + lows) * sizeof(float), &ws)) return st;
    f.partial = reinterpret_cast<float *>(ws);
    f.low = f.partial + sums;
    OPS_HIP(c, launch_few(bf16, adapter, f, c->stream));
    return HWR_OK;
}

// ---------------------------------------------------------------- operators
hwr_status group_rows(hwr_ops *c, int32_t n, const int32_t *choice, const int32_t *table, int32_t n_table, int32_t n_groups,
                      int32_t *offsets, int32_t *order) {
    if (!c) return invalid(nullptr, "ops is NULL");
    if (n < 0) return invalid(c, "n < 0");
    if (n_groups < 1 || n_groups > kMaxPairs) return invalid(c, "n_groups outside 1..1024");
    if (!offsets || (n > 0 && (!choice || !order))) return invalid(c, "choice, offsets and order are required");
    if (table ? n_table < 1 : n_table != 0) return invalid(c, "n_table must be > 0 with a table and 0 without");
    if (misaligned(HWR_F32, {choice, table, offsets, order})) return invalid(c, "a pointer is not aligned to its elements");
    OPS_ON_DEVICE(c, c->dev);
    GroupRowsArgs a{n, n_table, n_groups, choice, table, offsets, order, group_rows_blocks(n), nullptr, nullptr};
    if (a.blocks > 1) {
        const uint64_t counts = static_cast<uint64_t>(n_groups + 1) * a.blocks;
        char *ws = nullptr;
        if (hwr_status st = workspace(c, (counts + n_groups + 1) * sizeof(int32_t), &ws)) return st;
        a.hist = reinterpret_cast<int32_t *>(ws);
        a.totals = a.hist + counts;
    }
    OPS_HIP(c, launch_group_rows(a, c->stream));
    return HWR_OK;
}

hwr_status grouped_matmul(hwr_ops *c, const hwr_groups *g, const hwr_matmul_args *a) {
    if (!c) return invalid(nullptr, "ops is NULL");
    if (const char *m = check_groups(g)) return invalid(c, m);
    if (!a) return invalid(c, "arguments are NULL");
    if (const char *m = check_shape(a->dtype, a->k, a->m)) return invalid(c, m);
    if (bad_ld(a->ldx, a->k) || bad_ld(a->ldy, a->m)) return invalid(c, "a row stride is smaller than the row");
    if (g->n == 0) return HWR_OK;
    if (!a->x || !a->w || !a->y) return invalid(c, "x, w and y are required");
    if (misaligned(a->dtype, {a->x, a->w, a->y})) return invalid(c, "a pointer is not aligned to its elements");
    OPS_ON_DEVICE(c, c->dev);
    if (few_rows(g->n, g->n_groups, a->k, a->m, false, a->dtype == HWR_BF16)) {
        FewArgs f{};
        f.g = groups_arg(g);
        f.k = a->k;
        f.m = a->m;
        f.x = a->x;
        f.ldx = dense(a->ldx, a->k);
        f.w = a->w;
        f.w_stride = static_cast<int64_t>(a->k) * a->m;
        f.y = a->y;
        f.ldy = dense(a->ldy, a->m);
        return few(c, f, a->dtype == HWR_BF16, false);
    }
    const bool bf16 = a->dtype == HWR_BF16;
    const void *x = a->x, *w = a->w;
    int64_t ldx = dense(a->ldx, a->k), ldw = a->m;
    uint64_t used = 0;
    Pads pads(bf16);
    pads.add(&x, &ldx, g->n, a->k);
    pads.add(&w, &ldw, static_cast<int64_t>(g->n_groups) * a->k, a->m);
    const bool padded = pads.plan(2.0 * g->n * a->k * a->m, false, &used);
    RowsArgs r = rows_args(c, g, true, padded, x, ldx, a->k, w, ldw, a->k, false, a->m, a->y, dense(a->ldy, a->m));
    char *ws = nullptr;
    if (hwr_status st = workspace(c, used + rows_bytes(c, bf16, RowsKind::kGrouped, true, r), &ws)) return st;
    if (hwr_status st = pads.copy(c, ws)) return st;
    r.x = x;
    r.w = w;
    return rows(c, bf16, RowsKind::kGrouped, true, r, ws + used);
}

hwr_status grouped_matmul_grad(hwr_ops *c, const hwr_groups *g, const hwr_matmul_grad_args *a) {
    if (!c) return invalid(nullptr, "ops is NULL");
    if (const char *m = check_groups(g)) return invalid(c, m);
    if (!a) return invalid(c, "arguments are NULL");
    if (const char *m = check_shape(a->dtype, a->k, a->m)) return invalid(c, m);
    if (bad_ld(a->lddy, a->m) || bad_ld(a->ldx, a->k) || bad_ld(a->lddx, a->k))
        return invalid(c, "a row stride is smaller than the row");
    if (g->n > 0 && (!a->dy || (a->dx && !a->w) || (a->dw && !a->x)))
        return invalid(c, "dy is required, w for dx, and x for dw");
    if (misaligned(a->dtype, {a->dy, a->x, a->w, a->dx, a->dw})) return invalid(c, "a pointer is not aligned to its elements");
    OPS_ON_DEVICE(c, c->dev);
    const bool bf16 = a->dtype == HWR_BF16;
    const void *dy = a->dy, *x = a->x, *w = a->w;
    int64_t lddy = dense(a->lddy, a->m), ldx = dense(a->ldx, a->k), ldw = a->m;
    uint64_t used = 0;
    Pads pads(bf16);
    pads.add(&dy, &lddy, g->n, a->m);
    pads.add(&w, &ldw, static_cast<int64_t>(g->n_groups) * a->k, a->m, a->dx != nullptr);
    pads.add(&x, &ldx, g->n, a->k, a->dw != nullptr);
    const bool padded = pads.plan(4.0 * g->n * a->k * a->m, true, &used), dx = a->dx && g->n > 0;
    RowsArgs r = rows_args(c, g, false, padded, dy, lddy, a->m, w, ldw, a->k, false, a->k, a->dx, dense(a->lddx, a->k));
    ColsArgs d{};
    d.g = groups_arg(g);
    d.np = a->k;
    d.nq = a->m;
    d.padded = padded;
    d.p = x;
    d.q = dy;
    d.ldp = ldx;
    d.ldq = lddy;
    d.out = a->dw;
    // (one after the other: they share the place of their partial sums)
    const uint64_t sums = std::max(dx ? rows_bytes(c, bf16, RowsKind::kGrouped, false, r) : 0,
                                   a->dw ? weight_grad_bytes(c, bf16, ColsKind::kDense, d) : 0);
    char *ws = nullptr;
    if (hwr_status st = workspace(c, used + sums, &ws)) return st;
    if (hwr_status st = pads.copy(c, ws)) return st;
    r.x = d.q = dy;
    r.w = w;
    d.p = x;
    if (dx)
        if (hwr_status st = rows(c, bf16, RowsKind::kGrouped, false, r, ws + used)) return st;
    if (a->dw)
        if (hwr_status st = weight_grad(c, bf16, ColsKind::kDense, d, ws + used)) return st;
    return HWR_OK;
}

hwr_status adapter_matmul(hwr_ops *c, const hwr_groups *g, const hwr_adapter_args *a) {
    if (!c) return invalid(nullptr, "ops is NULL");
    if (const char *m = check_groups(g)) return invalid(c, m);
    if (!a) return invalid(c, "arguments are NULL");
    if (const char *m = check_shape(a->dtype, a->k, a->m)) return invalid(c, m);
    if (const char *m = check_rank(a->rank)) return invalid(c, m);
    if (bad_ld(a->ldx, a->k) || bad_ld(a->ldy, a->m)) return invalid(c, "a row stride is smaller than the row");
    if (g->n == 0) return HWR_OK;
    if (!a->x || !a->w || !a->a || !a->b || !a->y) return invalid(c, "x, w, a, b and y are required");
    if (misaligned(a->dtype, {a->x, a->w, a->a, a->b, a->y}) || misaligned(HWR_F32, {a->scale}))
        return invalid(c, "a pointer is not aligned to its elements");
    OPS_ON_DEVICE(c, c->dev);
    const int64_t ldx = dense(a->ldx, a->k);
    if (few_rows(g->n, g->n_groups, a->k, a->m, true, a->dtype == HWR_BF16)) {
        FewArgs f{};
        f.g = groups_arg(g);
        f.k = a->k;
        f.m = a->m;
        f.rank = a->rank;
        f.x = a->x;
        f.ldx = ldx;
        f.w = a->w;
        f.y = a->y;
        f.ldy = dense(a->ldy, a->m);
        f.a = a->a;
        f.b = a->b;
        f.scale = a->scale;
        return few(c, f, a->dtype == HWR_BF16, true);
    }
    const bool bf16 = a->dtype == HWR_BF16;
    uint64_t used = low_bytes(g->n, a->rank);
    const void *x = a->x, *w = a->w;
    int64_t ldxp = ldx, ldw = a->m;
    Pads pads(bf16);
    pads.add(&x, &ldxp, g->n, a->k);
    pads.add(&w, &ldw, a->k, a->m);
    const bool padded = pads.plan(2.0 * g->n * a->k * a->m, false, &used);
    RowsArgs r = rows_args(c, g, true, padded, x, ldxp, a->k, w, ldw, a->k, true, a->m, a->y, dense(a->ldy, a->m));
    r.lw = a->b;
    r.rank = a->rank;
    char *ws = nullptr;
    if (hwr_status st = workspace(c, used + rows_bytes(c, bf16, RowsKind::kAdapter, true, r), &ws)) return st;
    const ShrinkArgs to_low{groups_arg(g), a->k, a->rank, a->x, ldx, a->a, a->scale, ws};
    OPS_HIP(c, launch_shrink(bf16, true, to_low, c->cus, c->stream));
    if (hwr_status st = pads.copy(c, ws)) return st;
    r.x = x;
    r.w = w;
    r.low = ws;
    return rows(c, bf16, RowsKind::kAdapter, true, r, ws + used);
}

hwr_status adapter_matmul_grad(hwr_ops *c, const hwr_groups *g, const hwr_adapter_grad_args *a) {
    if (!c) return invalid(nullptr, "ops is NULL");
    if (const char *m = check_groups(g)) return invalid(c, m);
    if (!a) return invalid(c, "arguments are NULL");
    if (const char *m = check_shape(a->dtype, a->k, a->m)) return invalid(c, m);
    if (const char *m = check_rank(a->rank)) return invalid(c, m);
    if (bad_ld(a->lddy, a->m) || bad_ld(a->ldx, a->k) || bad_ld(a->lddx, a->k))
        return invalid(c, "a row stride is smaller than the row");
    if (g->n > 0 && (!a->dy || ((a->dx || a->da) && !a->b) || (a->dx && (!a->w || !a->a)) || (a->da && !a->x) ||
                     (a->db && (!a->x || !a->a))))
        return invalid(c, "dy is required; w, a and b for dx; x and b for da; x and a for db");
    if (misaligned(a->dtype, {a->dy, a->x, a->w, a->a, a->b, a->dx, a->da, a->db}) || misaligned(HWR_F32, {a->scale}))
        return invalid(c, "a pointer is not aligned to its elements");
    OPS_ON_DEVICE(c, c->dev);
    const bool bf16 = a->dtype == HWR_BF16;
    const int64_t lddy = dense(a->lddy, a->m), ldx = dense(a->ldx, a->k);
    const uint64_t each = low_bytes(g->n, a->rank);
    uint64_t used = 2 * each;
    const void *dy = a->dy, *x = a->x, *w = a->w;
    int64_t lddyp = lddy, ldxp = ldx, ldw = a->m;
    Pads pads(bf16);
    pads.add(&dy, &lddyp, g->n, a->m, a->dx || a->db);
    pads.add(&w, &ldw, a->k, a->m, a->dx != nullptr);
    pads.add(&x, &ldxp, g->n, a->k, a->da != nullptr);
    const bool padded = pads.plan(2.0 * g->n * a->k * a->m, true, &used), dx = a->dx && g->n > 0;
    RowsArgs r = rows_args(c, g, false, padded, dy, lddyp, a->m, w, ldw, a->k, true, a->k, a->dx, dense(a->lddx, a->k));
    r.lw = a->a;
    r.rank = a->rank;
    ColsArgs da{}, db{};
    da.g = db.g = groups_arg(g);
    da.padded = db.padded = padded;
    da.blocks = db.blocks = rank_blocks(a->rank);
    da.np = a->k;
    da.nq = a->rank;
    da.p = x;
    da.ldp = ldxp;
    da.out = a->da;
    db.np = a->rank;
    db.nq = a->m;
    db.q = dy;
    db.ldq = lddyp;
    db.out = a->db;
    // dx, then dA and dB together where both are direct, else one after the other: what
    // runs after another shares the place of its partial sums
    const bool pair = a->da && a->db && cols_plan(bf16, ColsKind::kLowQ, da, c->cus).direct &&
                      cols_plan(bf16, ColsKind::kLowP, db, c->cus).direct;
    const uint64_t da_sums = a->da ? weight_grad_bytes(c, bf16, ColsKind::kLowQ, da) : 0,
                   db_sums = a->db ? weight_grad_bytes(c, bf16, ColsKind::kLowP, db) : 0;
    const uint64_t sums = std::max(dx ? rows_bytes(c, bf16, RowsKind::kAdapter, false, r) : 0,
                                   pair ? da_sums + db_sums : std::max(da_sums, db_sums));
    char *ws = nullptr;
    if (hwr_status st = workspace(c, used + sums, &ws)) return st;
    char *up = ws, *low = ws + each, *partial = ws + used;
    const ShrinkArgs to_up{groups_arg(g), a->m, a->rank, a->dy, lddy, a->b, a->scale, up};
    const ShrinkArgs to_low{groups_arg(g), a->k, a->rank, a->x, ldx, a->a, a->scale, low};
    if (g->n > 0) {
        if ((a->dx || a->da) && a->db) OPS_HIP(c, launch_shrink_pair(bf16, to_up, to_low, c->cus, c->stream));
        else if (a->dx || a->da) OPS_HIP(c, launch_shrink(bf16, false, to_up, c->cus, c->stream));
        else if (a->db) OPS_HIP(c, launch_shrink(bf16, true, to_low, c->cus, c->stream));
    }
    if (hwr_status st = pads.copy(c, ws)) return st;
    r.x = db.q = dy;
    r.w = w;
    r.low = da.q = up;
    da.p = x;
    db.p = low;
    if (dx)
        if (hwr_status st = rows(c, bf16, RowsKind::kAdapter, false, r, partial)) return st;
    if (pair) {
        da.parts = cols_plan(bf16, ColsKind::kLowQ, da, c->cus).parts;
        db.parts = cols_plan(bf16, ColsKind::kLowP, db, c->cus).parts;
        da.partial = reinterpret_cast<float *>(partial);
        db.partial = reinterpret_cast<float *>(partial + da_sums);
        da.zeros = db.zeros = c->zeros;
        OPS_HIP(c, launch_cols_low_pair(bf16, da, db, c->stream));
        return HWR_OK;
    }
    if (a->da)
        if (hwr_status st = weight_grad(c, bf16, ColsKind::kLowQ, da, partial)) return st;
    if (a->db)
        if (hwr_status st = weight_grad(c, bf16, ColsKind::kLowP, db, partial)) return st;
    return HWR_OK;
}

}  // namespace

extern "C" {

hwr_status hwr_ops_init(int32_t device, void *stream, hwr_ops **out) {
    return c_boundary([&] { return init_impl(device, stream, out); }, [](const char *m) { fail(nullptr, HWR_ERR_OOM, m); });
}

void hwr_ops_free(hwr_ops *ops) {
    if (!ops) return;
    c_boundary(
        [&] {
            const OnDevice on_device(ops->dev);
            (void)hipStreamSynchronize(ops->stream);
            release(ops);
            return HWR_OK;
        },
        [](const char *) {});
}

const char *hwr_ops_last_error(const hwr_ops *ops) { return ops ? ops->err.c_str() : g_ops_error.c_str(); }

hwr_status hwr_ops_reserve(hwr_ops *ops, uint64_t bytes) {
    return c_boundary(
        [&]() -> hwr_status {
            if (!ops) return invalid(nullptr, "ops is NULL");
            if (bytes > uint64_t(1) << 40) return invalid(ops, "bytes above 1 TiB");
            OPS_ON_DEVICE(ops, ops->dev);
            char *p;
            return workspace(ops, bytes, &p);
        },
        [&](const char *m) { fail(ops, HWR_ERR_OOM, m); });
}

hwr_status hwr_group_rows(hwr_ops *ops, int32_t n, const int32_t *choice, const int32_t *table, int32_t n_table,
                          int32_t n_groups, int32_t *offsets, int32_t *order) {
    return c_boundary([&] { return group_rows(ops, n, choice, table, n_table, n_groups, offsets, order); },
                      [&](const char *m) { fail(ops, HWR_ERR_OOM, m); });
}

hwr_status hwr_grouped_matmul(hwr_ops *ops, const hwr_groups *g, const hwr_matmul_args *a) {
    return c_boundary([&] { return grouped_matmul(ops, g, a); }, [&](const char *m) { fail(ops, HWR_ERR_OOM, m); });
}

hwr_status hwr_grouped_matmul_grad(hwr_ops *ops, const hwr_groups *g, const hwr_matmul_grad_args *a) {
    return c_boundary([&] { return grouped_matmul_grad(ops, g, a); }, [&](const char *m) { fail(ops, HWR_ERR_OOM, m); });
}

hwr_status hwr_adapter_matmul(hwr_ops *ops, const hwr_groups *g, const hwr_adapter_args *a) {
    return c_boundary([&] { return adapter_matmul(ops, g, a); }, [&](const char *m) { fail(ops, HWR_ERR_OOM, m); });
}

hwr_status hwr_adapter_matmul_grad(hwr_ops *ops, const hwr_groups *g, const hwr_adapter_grad_args *a) {
    return c_boundary([&] { return adapter_matmul_grad(ops, g, a); }, [&](const char *m) { fail(ops, HWR_ERR_OOM, m); });
}

}  // extern "C"
