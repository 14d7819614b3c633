// Weight gradients of a routed batch: out[g] = P^T Q over the places of group
// g, with P and Q rows of the batch (through the row order) or low-rank
// intermediates (by place).
//
// Both factors are staged by place, 64 (bf16) or 32 (fp32) places to a stage, and
// read by columns.  Where the output has few tiles, workgroups share a tile's
// places and write fp32 partial sums that k_cols_sum adds, in order.
#include <algorithm>

#include "ops_device.hpp"

namespace hwr {
namespace {

// The workgroup's tile of the output and places.
struct ColsTile {
    int g, ip, iq, part, p0, p1;
};

// The group whose turn it is, the largest first (up to 64 groups; more go as they
// stand): the long workgroups then start early, and short ones fill the end.
__device__ inline int largest_group(const GroupsArg &g, int turn) {
    if (g.G > 64) return turn;
    const int lane = threadIdx.x & 63;
    const int size = lane < g.G ? place_of(g, lane + 1) - place_of(g, lane) : 0;
    int before = 0;
    for (int i = 0; i < g.G; ++i) {
        const int other = __builtin_amdgcn_readlane(size, i);
        before += other > size || (other == size && i < lane);
    }
    return __builtin_ctzll(__ballot(lane < g.G && before == turn));
}

// The tiles of a group (with their parts side by side) are cut into shares of about
// 16, which go to the L2s in turn: 4 x 4 tiles that run together read 8 panels of rows.
__host__ __device__ inline int cols_shares(int64_t per) { return per < 32 ? 1 : per < 128 ? static_cast<int>(per / 16) : 8; }

template <ColsKind KIND, int BP, int BQ, int kBk>
__device__ inline bool my_tile(const ColsArgs &a, int block, ColsTile &t) {
    const int tp = KIND == ColsKind::kLowP ? a.blocks : (a.np + BP - 1) / BP;
    const int tq = KIND == ColsKind::kLowQ ? a.blocks : (a.nq + BQ - 1) / BQ;
    const int per = tp * tq * a.parts, shares = cols_shares(per), share = (per + shares - 1) / shares;
    const int at = block >> 3, turn = at / share * 8 + (block & 7);
    const int in_group = turn % shares * share + at % share;
    if (turn >= a.g.G * shares || in_group >= per) return false;
    t.g = largest_group(a.g, turn / shares);
    const int tile = in_group / a.parts;
    t.part = in_group % a.parts;
    const int panel = tile / (4 * tq) * 4, in = tile - panel * tq, rp = min(4, tp - panel);
    t.ip = panel + in % rp;
    t.iq = in / rp;
    t.p0 = place_of(a.g, t.g);
    t.p1 = place_of(a.g, t.g + 1);
    if (a.parts > 1) {                     // whole stages each
        const int stages = max(0, t.p1 - t.p0 + kBk - 1) / kBk;
        const int s0 = static_cast<int>(static_cast<int64_t>(stages) * t.part / a.parts),
                  s1 = static_cast<int>(static_cast<int64_t>(stages) * (t.part + 1) / a.parts);
        t.p1 = min(t.p1, t.p0 + s1 * kBk);
        t.p0 += s0 * kBk;
    }
    return true;
}

// Lane: P column l % 16 of fragment i, four Q columns of fragment j.
template <class E, ColsKind KIND, int BP, int BQ, int WP, int WQ>
__device__ inline void store_tile(const ColsArgs &a, const ColsTile &t, const f32x4 (&acc)[BP / WP / 16][BQ / WQ / 16],
                                  int lane, int wp, int wq) {
    using El = Elem<E>;
    constexpr int PF = BP / WP / 16, QF = BQ / WQ / 16;
    constexpr bool kPair = sizeof(E) == 2;    // low-rank sides hold hi and lo columns
    constexpr int PN = KIND == ColsKind::kLowP ? 2 : PF, QN = KIND == ColsKind::kLowQ ? 2 : QF;
    const int p_first = KIND == ColsKind::kLowP ? t.ip * kRankBlock : t.ip * BP + wp * PF * 16;
    const int q_first = KIND == ColsKind::kLowQ ? t.iq * kRankBlock : t.iq * BQ + wq * QF * 16;
    const int64_t each = static_cast<int64_t>(a.np) * a.nq;
    E *out = static_cast<E *>(a.out) + t.g * each;
    float *part = a.partial + (static_cast<int64_t>(t.part) * a.g.G + t.g) * each;
#pragma unroll
    for (int i = 0; i < PN; ++i) {
        const int pr = p_first + i * 16 + (lane & 15);
        if (pr >= a.np) continue;
#pragma unroll
        for (int j = 0; j < QN; ++j) {
            f32x4 v = acc[i][j];
            if constexpr (KIND != ColsKind::kDense && kPair) {
                // hi + lo; where an infinite factor made hi infinite, lo could make it NaN
                const f32x4 lo = KIND == ColsKind::kLowP ? acc[(i + 2) % PF][j] : acc[i][(j + 2) % QF];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = __builtin_isfinite(v[e]) ? v[e] + lo[e] : v[e];
            }
            const int c = q_first + j * 16 + (lane >> 4) * 4;
            const int64_t line = static_cast<int64_t>(pr) * a.nq;
            if (a.parts > 1) store_four<float>(part + line, c, a.nq, v);
            else store_four<E>(out + line, c, a.nq, v);
        }
    }
}

template <class E, ColsKind KIND, int BP, int BQ>
struct ColsTiles {
    using PT = Tile<E, true, BP>;
    using QT = Tile<E, true, BQ>;
    // a rank block as a tile: 32 columns, in bf16 hi then lo
    static constexpr int kLowCols = kLowBytes / sizeof(E);
    static constexpr bool kLowP = KIND == ColsKind::kLowP, kLowQ = KIND == ColsKind::kLowQ;
    static_assert(!kLowP || BP == kLowCols);
    static_assert(!kLowQ || BQ == kLowCols);
};

template <class E, class PT, class QT, int PF, int QF>
__device__ inline void multiply_tile(const char *lds, int at_q, int p0, int q0, int lane, f32x4 (&acc)[PF][QF]) {
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
        typename Elem<E>::Frag fq[QF], fp[PF];
#pragma unroll
        for (int j = 0; j < QF; ++j) fq[j] = QT::frag(lds, at_q, q0 + j * 16, sub, QT::base(lane));
#pragma unroll
        for (int i = 0; i < PF; ++i) fp[i] = PT::frag(lds, 0, p0 + i * 16, sub, PT::base(lane));
#pragma unroll
        for (int i = 0; i < PF; ++i)
#pragma unroll
            for (int j = 0; j < QF; ++j) acc[i][j] = Elem<E>::mma(fq[j], fp[i], acc[i][j]);
    }
}

// Any widths, strides and alignment: operands pass through registers.
template <class E, ColsKind KIND, int BP, int BQ, int WP, int WQ>
__global__ void __launch_bounds__(WP *WQ * 64) k_cols(ColsArgs a) {
    using El = Elem<E>;
    using TT = ColsTiles<E, KIND, BP, BQ>;
    using PT = typename TT::PT;
    using QT = typename TT::QT;
    static_assert((!TT::kLowP || WP == 1) && (!TT::kLowQ || WQ == 1));
    constexpr int NT = WP * WQ * 64, PF = BP / WP / 16, QF = BQ / WQ / 16, kBk = El::kBk;
    __shared__ __attribute__((aligned(16))) char buf[PT::kBytes + QT::kBytes];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wp = wave / WQ, wq = wave % WQ;
    ColsTile t;
    if (!my_tile<KIND, BP, BQ, kBk>(a, blockIdx.x, t)) return;

    f32x4 acc[PF][QF] = {};
    constexpr int UP = PT::kChunks / NT, UQ = QT::kChunks / NT;
    static_assert(PT::kChunks % NT == 0 && QT::kChunks % NT == 0);
    auto chunk = [&](const void *src, int64_t ld, int width, int c0, bool low, int block, int place, int c) {
        if (place >= t.p1) return u32x4{0, 0, 0, 0};
        if (low)
            return *reinterpret_cast<const u32x4 *>(static_cast<const char *>(src) +
                                                    (static_cast<int64_t>(place) * a.blocks + block) * kLowBytes + c * 16);
        const int r = row_at(a.g, place);
        return load_chunk<E>(r >= 0 ? static_cast<const E *>(src) + r * ld : nullptr, c0 + c * El::kEpc, width);
    };
    u32x4 vp[UP], vq[UQ];
    auto load = [&](int p) {
#pragma unroll
        for (int i = 0; i < UP; ++i) {
            const int u = i * NT + tid, line = u / PT::kCpl, c = (u % PT::kCpl) ^ PT::swz(line);
            vp[i] = chunk(a.p, a.ldp, a.np, t.ip * BP, TT::kLowP, t.ip, p + line, c);
        }
#pragma unroll
        for (int i = 0; i < UQ; ++i) {
            const int u = i * NT + tid, line = u / QT::kCpl, c = (u % QT::kCpl) ^ QT::swz(line);
            vq[i] = chunk(a.q, a.ldq, a.nq, t.iq * BQ, TT::kLowQ, t.iq, p + line, c);
        }
    };
    if (t.p0 < t.p1) load(t.p0);
    for (int p = t.p0; p < t.p1; p += kBk) {
#pragma unroll
        for (int i = 0; i < UP; ++i) *reinterpret_cast<u32x4 *>(buf + (i * NT + tid) * 16) = vp[i];
#pragma unroll
        for (int i = 0; i < UQ; ++i) *reinterpret_cast<u32x4 *>(buf + PT::kBytes + (i * NT + tid) * 16) = vq[i];
        __syncthreads();
        if (p + kBk < t.p1) load(p + kBk);
        multiply_tile<E, PT, QT, PF, QF>(buf, PT::kBytes, wp * PF * 16, wq * QF * 16, lane, acc);
        __syncthreads();
    }
    store_tile<E, KIND, BP, BQ, WP, WQ>(a, t, acc, lane, wp, wq);
}

// Whole chunks of 16 bytes everywhere: operands go from memory straight into LDS
// (run_stages); a stage's rows are looked up when the stage before it is loaded.  Places past the last are zeros on both sides; columns
// past the last are loaded from a valid place and not stored.
template <class E, ColsKind KIND, int BP, int BQ>
constexpr int kColsBuf = ColsTiles<E, KIND, BP, BQ>::PT::kBytes + ColsTiles<E, KIND, BP, BQ>::QT::kBytes;

template <class E, ColsKind KIND, int BP, int BQ, int WP, int WQ>
__device__ inline void cols_direct(const ColsArgs &a, int block, char *buf0, char *buf1, char *buf2, char *buf3) {
    using El = Elem<E>;
    using TT = ColsTiles<E, KIND, BP, BQ>;
    using PT = typename TT::PT;
    using QT = typename TT::QT;
    static_assert((!TT::kLowP || WP == 1) && (!TT::kLowQ || WQ == 1));
    constexpr int NT = WP * WQ * 64, PF = BP / WP / 16, QF = BQ / WQ / 16, kBk = El::kBk, kEpc = El::kEpc;
    constexpr int UP = PT::kChunks / NT, UQ = QT::kChunks / NT;
    static_assert(PT::kChunks % NT == 0 && QT::kChunks % NT == 0);
    constexpr bool kDeep = BP == 64 && BQ == 64;     // run_stages_deep
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wp = wave / WQ, wq = wave % WQ;
    ColsTile t;
    if (!my_tile<KIND, BP, BQ, kBk>(a, block, t)) return;

    // the thread's chunks: byte within the row.  Lines 16 apart have the same order of chunks.
    constexpr int kLinesP = NT / PT::kCpl, kLinesQ = NT / QT::kCpl;
    constexpr int BPN = kLinesP % 16 ? UP : 1, BQN = kLinesQ % 16 ? UQ : 1;
    int pb[BPN], qb[BQN];
#pragma unroll
    for (int i = 0; i < BPN; ++i) {
        const int u = i * NT + tid, c = (u % PT::kCpl) ^ PT::swz(u / PT::kCpl);
        pb[i] = TT::kLowP ? t.ip * kLowBytes + c * 16 : min(t.ip * BP + c * kEpc, (a.np - 1) / kEpc * kEpc) * (int)sizeof(E);
    }
#pragma unroll
    for (int i = 0; i < BQN; ++i) {
        const int u = i * NT + tid, c = (u % QT::kCpl) ^ QT::swz(u / QT::kCpl);
        qb[i] = TT::kLowQ ? t.iq * kLowBytes + c * 16 : min(t.iq * BQ + c * kEpc, (a.nq - 1) / kEpc * kEpc) * (int)sizeof(E);
    }
    // Rows of a stage's lines, as they stand in the order (checked when they are used:
    // a check here would wait for the loads in flight).  Tiles of one width share them.
    // Looked up one stage before they are loaded, or four (run_stages_deep), in turn.
    constexpr bool kShared = KIND == ColsKind::kDense && BP == BQ;
    constexpr int kSlots = kDeep ? 4 : 1, kLead = kDeep ? 4 : 1;
    int pr[kSlots][UP], qr[kSlots][kShared ? 1 : UQ];
    auto look_up = [&](int stage, int slot) {
        const int p = t.p0 + stage * kBk;
        auto row = [&](int at) {
            at = min(at, t.p1 - 1);
            return a.g.order ? a.g.order[at] : at;
        };
        if constexpr (!TT::kLowP)
#pragma unroll
            for (int i = 0; i < UP; ++i) pr[slot][i] = row(p + i * kLinesP + tid / PT::kCpl);
        if constexpr (!kShared && !TT::kLowQ)
#pragma unroll
            for (int i = 0; i < UQ; ++i) qr[slot][i] = row(p + i * kLinesQ + tid / QT::kCpl);
    };
    const int64_t pld = TT::kLowP ? a.blocks * kLowBytes : a.ldp * (int64_t)sizeof(E);
    const int64_t qld = TT::kLowQ ? a.blocks * kLowBytes : a.ldq * (int64_t)sizeof(E);
    const char *ps = static_cast<const char *>(a.p), *qs = static_cast<const char *>(a.q);
    auto in_range = [&](int row) { return min(static_cast<unsigned>(row), static_cast<unsigned>(a.g.n - 1)); };
    auto issue = [&](char *b, int stage, auto... in_turn) {
        constexpr int slot = kDeep ? (decltype(in_turn)::value + ... + 0) : 0;
        const int p = t.p0 + stage * kBk;
        auto p_row = [&](int i) -> int64_t { return TT::kLowP ? p + i * kLinesP + tid / PT::kCpl : in_range(pr[slot][i]); };
        auto q_row = [&](int i) -> int64_t {
            return TT::kLowQ ? p + i * kLinesQ + tid / QT::kCpl : in_range(kShared ? pr[slot][i] : qr[slot][kShared ? 0 : i]);
        };
        auto to_p = [&](int i, const char *src) { load_lds(src, b + (i * NT + wave * 64) * 16); };
        auto to_q = [&](int i, const char *src) { load_lds(src, b + PT::kBytes + (i * NT + wave * 64) * 16); };
        if (p + kBk <= t.p1) {
#pragma unroll
            for (int i = 0; i < UP; ++i) to_p(i, ps + p_row(i) * pld + pb[i % BPN]);
#pragma unroll
            for (int i = 0; i < UQ; ++i) to_q(i, qs + q_row(i) * qld + qb[i % BQN]);
        } else {                           // lines past the last place are zeros
            const char *zeros = static_cast<const char *>(a.zeros);
#pragma unroll
            for (int i = 0; i < UP; ++i)
                to_p(i, p + i * kLinesP + tid / PT::kCpl < t.p1 ? ps + p_row(i) * pld + pb[i % BPN] : zeros);
#pragma unroll
            for (int i = 0; i < UQ; ++i)
                to_q(i, p + i * kLinesQ + tid / QT::kCpl < t.p1 ? qs + q_row(i) * qld + qb[i % BQN] : zeros);
        }
        look_up(stage + kLead, (slot + kLead) % kSlots);
    };
    f32x4 acc[PF][QF] = {};
    if (t.p0 < t.p1) {
        const int stages = (t.p1 - t.p0 + kBk - 1) / kBk, p_at = wp * PF * 16, q_at = wq * QF * 16;
#pragma unroll
        for (int i = 0; i < kLead; ++i) look_up(i, i);
        if constexpr (kDeep) run_stages_deep<E, PT, QT, PF, QF, UP + UQ>(stages, issue, buf0, buf1, buf2, buf3, p_at, q_at, lane, acc);
        else run_stages<E, PT, QT, PF, QF>(stages, issue, buf0, buf1, p_at, q_at, lane, acc);
    }
    if constexpr (KIND == ColsKind::kDense) {
        if (a.parts == 1) {                // whole rows of the output
            using L = ThroughLds<E, BP, BQ, WP, WQ>;
            const int q = t.iq * BQ + L::column(tid);
            E *out = static_cast<E *>(a.out) + static_cast<int64_t>(t.g) * a.np * a.nq;
            __syncthreads();               // (the last products have read the buffers)
            L::run(buf0, buf1, acc, tid, [](int, int, int) {}, [&](int, int, int row, const float (&v)[L::V]) __attribute__((always_inline)) {
                const int p = t.ip * BP + row;
                if (p < a.np && q < a.nq) Some<E, L::V>(v).store(out + static_cast<int64_t>(p) * a.nq, q, a.nq);
            });
            return;
        }
    }
    store_tile<E, KIND, BP, BQ, WP, WQ>(a, t, acc, lane, wp, wq);
}

template <class E, ColsKind KIND, int BP, int BQ, int WP, int WQ>
__global__ void __launch_bounds__(WP *WQ * 64) k_cols_direct(ColsArgs a) {
    // an array each, so that the compiler sees that reads of one do not depend on the
    // loads in flight into the other
    constexpr int kBuf = kColsBuf<E, KIND, BP, BQ>, kMore = BP == 64 && BQ == 64 ? kBuf : 16;
    __shared__ __attribute__((aligned(16))) char buf0[kBuf], buf1[kBuf], buf2[kMore], buf3[kMore];
    cols_direct<E, KIND, BP, BQ, WP, WQ>(a, blockIdx.x, buf0, buf1, buf2, buf3);
}

// Both low-rank gradients in one launch, eight workgroups (one on each L2) of each in turn.
template <class E>
__global__ void __launch_bounds__(256) k_cols_low_pair(ColsArgs a, ColsArgs b) {
    constexpr int L = kLowBytes / sizeof(E), kBuf = kColsBuf<E, ColsKind::kLowQ, 128, L>;
    static_assert(kBuf == kColsBuf<E, ColsKind::kLowP, L, 128>);
    __shared__ __attribute__((aligned(16))) char buf0[kBuf], buf1[kBuf];
    const int block = blockIdx.x >> 4 << 3 | (blockIdx.x & 7);
    if (blockIdx.x & 8) cols_direct<E, ColsKind::kLowP, L, 128, 1, 4>(b, block, buf0, buf1, nullptr, nullptr);
    else cols_direct<E, ColsKind::kLowQ, 128, L, 4, 1>(a, block, buf0, buf1, nullptr, nullptr);
}

// out = sum of the parts
template <class E>
__device__ inline void sum_parts(const ColsArgs &a, int64_t i) {
    const int64_t count = static_cast<int64_t>(a.g.G) * a.np * a.nq;
    if (i >= count) return;
    if (i + 4 <= count) {
        f32x4 v = {};
#pragma unroll 4
        for (int s = 0; s < a.parts; ++s) v += *reinterpret_cast<const f32x4_a4 *>(a.partial + s * count + i);
        typename Elem<E>::Out4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = static_cast<E>(v[e]);
        *reinterpret_cast<typename Elem<E>::Out4 *>(static_cast<E *>(a.out) + i) = o;
    } else {
        for (int64_t j = i; j < count; ++j) {
            float v = 0.0f;
            for (int s = 0; s < a.parts; ++s) v += a.partial[s * count + j];
            static_cast<E *>(a.out)[j] = static_cast<E>(v);
        }
    }
}

// (of one gradient, or of two: grid.y)
template <class E>
__global__ void __launch_bounds__(256) k_cols_sum(ColsArgs a, ColsArgs b) {
    const int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
    const ColsArgs &c = blockIdx.y ? b : a;
    if (c.parts > 1) sum_parts<E>(c, i);
}

template <class E>
hipError_t sum(const ColsArgs &a, const ColsArgs *b, hipStream_t s) {
    auto blocks = [](const ColsArgs &c) { return c.parts > 1 ? (static_cast<int64_t>(c.g.G) * c.np * c.nq + 1023) / 1024 : 0; };
    const int64_t most = std::max(blocks(a), b ? blocks(*b) : 0);
    if (most == 0) return hipSuccess;
    return launch_kernel(k_cols_sum<E>, dim3(static_cast<uint32_t>(most), b ? 2 : 1), dim3(256), 0, s, a, b ? *b : a);
}

// Rows in whole, aligned chunks of 16 bytes.
template <class E, ColsKind KIND>
bool whole_chunks(const ColsArgs &a) {
    constexpr int kEpc = Elem<E>::kEpc;
    auto whole = [&](const void *p, int64_t ld, int width) {
        return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % kEpc == 0 && (a.padded || width % kEpc == 0);
    };
    return (KIND == ColsKind::kLowP || whole(a.p, a.ldp, a.np)) && (KIND == ColsKind::kLowQ || whole(a.q, a.ldq, a.nq));
}

// Workgroups: a multiple of 8.
int64_t cols_blocks(const ColsArgs &a, int64_t tp, int64_t tq) {
    const int64_t per = tp * tq * a.parts, shares = cols_shares(per), share = (per + shares - 1) / shares;
    return (a.g.G * shares + 7) / 8 * 8 * share;
}

template <class E, ColsKind KIND, int BP, int BQ, int WP, int WQ, bool DIRECT>
hipError_t go(const ColsArgs &a, hipStream_t s) {
    const int64_t blocks = cols_blocks(a, KIND == ColsKind::kLowP ? a.blocks : (a.np + BP - 1) / BP,
                                       KIND == ColsKind::kLowQ ? a.blocks : (a.nq + BQ - 1) / BQ);
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    const dim3 grid(static_cast<uint32_t>(blocks)), block(WP * WQ * 64);
    hipError_t e;
    if constexpr (DIRECT) e = launch_kernel(k_cols_direct<E, KIND, BP, BQ, WP, WQ>, grid, block, 0, s, a);
    else e = launch_kernel(k_cols<E, KIND, BP, BQ, WP, WQ>, grid, block, 0, s, a);
    return e != hipSuccess ? e : sum<E>(a, nullptr, s);
}

template <class E>
hipError_t low_pair(const ColsArgs &a, const ColsArgs &b, hipStream_t s) {
    const int64_t most = std::max(cols_blocks(a, (a.np + 127) / 128, a.blocks), cols_blocks(b, b.blocks, (b.nq + 127) / 128));
    if (2 * most > INT32_MAX) return hipErrorInvalidValue;
    const hipError_t e = launch_kernel(k_cols_low_pair<E>, dim3(static_cast<uint32_t>(2 * most)), dim3(256), 0, s, a, b);
    return e != hipSuccess ? e : sum<E>(a, &b, s);
}

template <class E>
hipError_t pick(ColsKind kind, const ColsPlan &p, const ColsArgs &a, hipStream_t s) {
    constexpr int L = kLowBytes / sizeof(E);
    if (kind == ColsKind::kLowP)
        return p.direct ? go<E, ColsKind::kLowP, L, 128, 1, 4, true>(a, s) : go<E, ColsKind::kLowP, L, 128, 1, 4, false>(a, s);
    if (kind == ColsKind::kLowQ)
        return p.direct ? go<E, ColsKind::kLowQ, 128, L, 4, 1, true>(a, s) : go<E, ColsKind::kLowQ, 128, L, 4, 1, false>(a, s);
    if (p.direct) {
        if constexpr (sizeof(E) == 2)
            if (p.tile == 256) return go<E, ColsKind::kDense, 256, 256, 2, 4, true>(a, s);
        if (p.tile == 128) return go<E, ColsKind::kDense, 128, 128, 2, 2, true>(a, s);
        return go<E, ColsKind::kDense, 64, 64, 2, 2, true>(a, s);
    }
    if (p.tile == 128) return go<E, ColsKind::kDense, 128, 128, 2, 2, false>(a, s);
    return go<E, ColsKind::kDense, 64, 64, 2, 2, false>(a, s);
}

}  // namespace

// The largest tile with which workgroups fill the device, sharing tiles' places if need be:
// each part has at least 8 stages of an average group (4 with the smallest tile; its
// partial sums are written and read once, 1.6 ps an element).  fp32: not 128 for one to three tiles
// a compute unit, whose rounds come out uneven (both gradients, us, 64 / 128: 3,408 x 832 x 320 in 22 groups
// 68 / 80, 2,400 x 1024 x 1536 in 4 175 / 190, 1,455 x 284 x 1160 in 9 43 / 56; one group of 4,096 x 1024 x
// 1024 185 / 162 in parts).
ColsPlan cols_plan(bool bf16, ColsKind kind, const ColsArgs &a, int cus) {
    ColsPlan p{false, 64, 1};
    if (bf16)
        p.direct = kind == ColsKind::kLowP   ? whole_chunks<__bf16, ColsKind::kLowP>(a)
                   : kind == ColsKind::kLowQ ? whole_chunks<__bf16, ColsKind::kLowQ>(a)
                                             : whole_chunks<__bf16, ColsKind::kDense>(a);
    else
        p.direct = kind == ColsKind::kLowP   ? whole_chunks<float, ColsKind::kLowP>(a)
                   : kind == ColsKind::kLowQ ? whole_chunks<float, ColsKind::kLowQ>(a)
                                             : whole_chunks<float, ColsKind::kDense>(a);
    const int64_t stages = a.g.n / (static_cast<int64_t>(a.g.G) * (bf16 ? 64 : 32));
    // parts that bring `items` workgroups to `enough`
    auto parts = [](int64_t items, int64_t enough) {
        int64_t n = 1;
        while (items * n < enough) n *= 2;
        return n;
    };
    auto tiles = [&](int64_t t) { return a.g.G * ((a.np + t - 1) / t) * ((a.nq + t - 1) / t); };
    if (kind == ColsKind::kDense) {
        for (int t = p.direct && bf16 ? 256 : 128; t >= 64; t /= 2) {
            const int64_t n = parts(tiles(t), cus);
            if (!bf16 && t > 64 && tiles(t) >= cus && tiles(t) < 3 * cus) continue;
            if (t > 64 && (a.np < t || a.nq < t || n > std::max<int64_t>(1, stages / 8))) continue;
            p.tile = t;
            p.parts = static_cast<int>(std::min<int64_t>(n, std::max<int64_t>(1, stages / 4)));
            break;
        }
        return p;
    }
    const int64_t wide = kind == ColsKind::kLowP ? a.nq : a.np;
    const int64_t n = parts(a.blocks * ((wide + 127) / 128) * a.g.G, 3 * cus);
    p.parts = static_cast<int>(std::min<int64_t>(n, std::max<int64_t>(1, stages / 4)));
    return p;
}

hipError_t launch_cols(bool bf16, ColsKind kind, const ColsArgs &a, int cus, hipStream_t s) {
    const ColsPlan p = cols_plan(bf16, kind, a, cus);
    return bf16 ? pick<__bf16>(kind, p, a, s) : pick<float>(kind, p, a, s);
}

hipError_t launch_cols_low_pair(bool bf16, const ColsArgs &q, const ColsArgs &p, hipStream_t s) {
    return bf16 ? low_pair<__bf16>(q, p, s) : low_pair<float>(q, p, s);
}

}  // namespace hwr
