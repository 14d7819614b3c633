// Device code of the weight gradients (k_cols.hip; k_grad.hip).
#pragma once

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
__device__ inline bool col_tile(const ColsArgs &a, int block, ColsTile &t) {
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

// Whole chunks of 16 bytes everywhere: operands go from memory straight into LDS
// (run_stages); a stage's rows are looked up when the stage before it is loaded.  Places past the last are zeros on both sides; columns
// past the last are loaded from a valid place and not stored.
template <class E, ColsKind KIND, int BP, int BQ>
constexpr int kColsBuf = ColsTiles<E, KIND, BP, BQ>::PT::kBytes + ColsTiles<E, KIND, BP, BQ>::QT::kBytes;

template <class E, ColsKind KIND, int BP, int BQ, int WP, int WQ, bool DEEP = BP == 64 && BQ == 64>
__device__ inline void cols_direct(const ColsArgs &a, int block, char *buf0, char *buf1, char *buf2, char *buf3) {
    using El = Elem<E>;
    using TT = ColsTiles<E, KIND, BP, BQ>;
    using PT = typename TT::PT;
    using QT = typename TT::QT;
    static_assert((!TT::kLowP || WP == 1) && (!TT::kLowQ || WQ == 1));
    constexpr int NT = WP * WQ * 64, PF = BP / WP / 16, QF = BQ / WQ / 16, kBk = El::kBk, kEpc = El::kEpc;
    constexpr int UP = PT::kChunks / NT, UQ = QT::kChunks / NT;
    static_assert(PT::kChunks % NT == 0 && QT::kChunks % NT == 0);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wp = wave / WQ, wq = wave % WQ;
    ColsTile t;
    if (!col_tile<KIND, BP, BQ, kBk>(a, block, t)) return;

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
    constexpr int kSlots = DEEP ? 4 : 1, kLead = DEEP ? 4 : 1;
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
        constexpr int slot = DEEP ? (decltype(in_turn)::value + ... + 0) : 0;
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
        if constexpr (DEEP) run_stages_deep<E, PT, QT, PF, QF, UP + UQ>(stages, issue, buf0, buf1, buf2, buf3, p_at, q_at, lane, acc);
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

// Workgroups: a multiple of 8.
inline int64_t cols_blocks(const ColsArgs &a, int64_t tp, int64_t tq) {
    const int64_t per = tp * tq * a.parts, shares = cols_shares(per), share = (per + shares - 1) / shares;
    return (a.g.G * shares + 7) / 8 * 8 * share;
}

}  // namespace
}  // namespace hwr
