// Device code of the products by row (k_rows.hip; k_grad.hip).
#pragma once

#include <algorithm>

#include "ops_act.hpp"

namespace hwr {
namespace {

// Operands of one stage on their way from memory through registers: any width,
// row stride and alignment.
template <class E, bool KS, int N, int NT>
struct Staged {
    using T = Tile<E, KS, N>;
    static constexpr int U = (T::kChunks + NT - 1) / NT;
    static_assert(T::kChunks % NT == 0 || U == 1);
    u32x4 v[U];
    // src(line, chunk) -> 16 bytes
    template <class Src>
    __device__ void load(Src src, int tid) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int u = i * NT + tid, line = u / T::kCpl, c = (u % T::kCpl) ^ T::swz(line);
            if (T::kChunks % NT == 0 || u < T::kChunks) v[i] = src(line, c);
        }
    }
    __device__ void store(char *t, int tid) const {
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (T::kChunks % NT == 0 || i * NT + tid < T::kChunks) *reinterpret_cast<u32x4 *>(t + (i * NT + tid) * 16) = v[i];
    }
};

// bf16 infinities and NaNs become zeros.  The low part of a low-rank value
// multiplies such weights by zero: the high part alone gives the infinity (or
// NaN), where hi * inf + lo * inf could be inf - inf.
__device__ inline u32x4 finite_only(u32x4 v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((v[i] & 0x7F80u) == 0x7F80u) v[i] &= 0xFFFF0000u;
        if ((v[i] & 0x7F800000u) == 0x7F800000u) v[i] &= 0x0000FFFFu;
    }
    return v;
}

// The adapters of the tile's groups: one stage for every 32 of the rank, whose
// contraction is hi and lo against the same weights in bf16.  Only the rows of
// the group take the result (a zero would turn another group's infinity into NaN).
template <class E, bool KS, int BM, int BN, int WR, int WC>
__device__ inline void add_adapters(const RowsArgs &a, const RowTile &rt, int c0, char *sx, char *sw,
                                    f32x4 (&acc)[BM / WR / 16][BN / WC / 16], int tid) {
    using El = Elem<E>;
    constexpr int NT = WR * WC * 64, RF = BM / WR / 16, CF = BN / WC / 16;
    using XT = Tile<E, false, BM>;
    using WT = Tile<E, KS, BN>;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave / WC, wc = wave % WC;
    Staged<E, false, BM, NT> gx;
    Staged<E, KS, BN, NT> gw;
    const E *lw = static_cast<const E *>(a.lw);
    const char *low = static_cast<const char *>(a.low);
    const int blocks = (a.rank + kRankBlock - 1) / kRankBlock;
    for (int g = group_of(a.g, rt.p0, lane); g < a.g.G; ++g) {
        const int lo = max(place_of(a.g, g), rt.p0), hi = min(place_of(a.g, g + 1), rt.p1);
        if (place_of(a.g, g) >= rt.p1) break;
        if (lo >= hi) continue;
        const E *gl = lw + static_cast<int64_t>(g) * a.rank * a.m;
        for (int b = 0; b < blocks; ++b) {
            const int r0 = b * kRankBlock;
            gx.load([&](int line, int c) {
                const int p = rt.p0 + line;
                if (p < lo || p >= hi) return u32x4{0, 0, 0, 0};
                return *reinterpret_cast<const u32x4 *>(low + (static_cast<int64_t>(p) * blocks + b) * kLowBytes + c * 16);
            }, tid);
            gx.store(sx, tid);
            gw.load([&](int line, int c) {
                u32x4 v;
                const int e = KS ? line : c * El::kEpc;        // contraction element of the stage
                const int r = r0 + (e & (kRankBlock - 1));
                if constexpr (KS)
                    v = load_chunk<E>(r < a.rank ? gl + static_cast<int64_t>(r) * a.m : nullptr, c0 + c * El::kEpc, a.m);
                else
                    v = load_chunk<E>(c0 + line < a.m ? gl + static_cast<int64_t>(c0 + line) * a.rank : nullptr, r, a.rank);
                return e < kRankBlock ? v : finite_only(v);    // past kRankBlock: the low parts (bf16)
            }, tid);
            gw.store(sw, tid);
            __syncthreads();
#pragma unroll
            for (int sub = 0; sub < 2; ++sub) {
                typename El::Frag fw[CF];
#pragma unroll
                for (int j = 0; j < CF; ++j) fw[j] = WT::frag(sw, 0, (wc * CF + j) * 16, sub, WT::base(lane));
#pragma unroll
                for (int i = 0; i < RF; ++i) {
                    const int f0 = rt.p0 + (wr * RF + i) * 16;
                    if (f0 + 16 <= lo || f0 >= hi) continue;
                    const typename El::Frag fx = XT::frag(sx, 0, (wr * RF + i) * 16, sub, XT::base(lane));
                    const int p = f0 + (lane & 15);
                    const bool in_group = p >= lo && p < hi;
#pragma unroll
                    for (int j = 0; j < CF; ++j) {
                        const f32x4 v = El::mma(fw[j], fx, acc[i][j]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][e] = in_group ? v[e] : acc[i][j][e];
                    }
                }
            }
            __syncthreads();
        }
    }
}

// A lane holds, for row l % 16 of fragment i, four columns of fragment j.
template <class E, int BM, int BN, int WR, int WC>
__device__ inline void store_parts(const RowsArgs &a, const RowTile &rt, int c0, int part,
                                   const f32x4 (&acc)[BM / WR / 16][BN / WC / 16], int tid) {
    constexpr int RF = BM / WR / 16, CF = BN / WC / 16;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave / WC, wc = wave % WC;
    const int q = lane >> 4;
    float *out = a.partial + static_cast<int64_t>(part) * a.g.n * a.m_pad;
#pragma unroll
    for (int i = 0; i < RF; ++i) {
        const int p = rt.p0 + (wr * RF + i) * 16 + (lane & 15);
        if (p >= rt.p1) continue;
#pragma unroll
        for (int j = 0; j < CF; ++j) {
            const int c = c0 + (wc * CF + j) * 16 + q * 4;
            if (c < a.m_pad) *reinterpret_cast<f32x4_a4 *>(out + static_cast<int64_t>(p) * a.m_pad + c) = acc[i][j];
        }
    }
}
template <class E, RowsKind KIND, int BM, int BN, int WR, int WC>
__device__ inline void store_rows(const RowsArgs &a, const RowTile &rt, int c0, int part, const int *rows,
                                  const f32x4 (&acc)[BM / WR / 16][BN / WC / 16], int tid) {
    constexpr int RF = BM / WR / 16, CF = BN / WC / 16;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave / WC, wc = wave % WC;
    const int q = lane >> 4;
    if (a.parts > 1) return store_parts<E, BM, BN, WR, WC>(a, rt, c0, part, acc, tid);
    E *y = static_cast<E *>(a.y);
    if constexpr (KIND == RowsKind::kLinear) {
#pragma unroll
        for (int j = 0; j < CF; ++j) {
            Finish<E, 4> finish(a.end, c0 + (wc * CF + j) * 16 + q * 4, a.m, a.g.G, rt.g);
            int r[RF];
            Some<E, 4> res[RF];
#pragma unroll
            for (int i = 0; i < RF; ++i) {
                r[i] = rows[(wr * RF + i) * 16 + (lane & 15)];
                finish.load(max(r[i], 0), res[i]);
            }
            finish.settle();
#pragma unroll
            for (int i = 0; i < RF; ++i) {
                const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                if (r[i] >= 0) finish.store(r[i], res[i], v, y, a.ldy);
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < RF; ++i) {
        const int r = rows[(wr * RF + i) * 16 + (lane & 15)];
        if (r < 0) continue;
        E *line = y + r * a.ldy;
#pragma unroll
        for (int j = 0; j < CF; ++j) {
            store_four<E>(line, c0 + (wc * CF + j) * 16 + q * 4, a.m, acc[i][j]);
        }
    }
}

// A tile's rows, whole: y and z written, and the residual read, in chunks (through_lds).
template <class E, RowsKind KIND, int BM, int BN, int WR, int WC>
__device__ inline void store_whole_rows(const RowsArgs &a, const RowTile &rt, int c0, const int *rows, char *buf0, char *buf1,
                                        const f32x4 (&acc)[BM / WR / 16][BN / WC / 16], int tid) {
    using T = ThroughLds<E, BM, BN, WR, WC>;
    constexpr int V = T::V;
    constexpr bool kLayer = KIND == RowsKind::kLinear;
    const int c = c0 + T::column(tid);
    Finish<E, V> finish(a.end, c, a.m, a.g.G, rt.g);           // (layers)
    Some<E, V> res[3][T::U];
    int row[3][T::U];
    auto fetch = [&](int turn, int u, int i) __attribute__((always_inline)) {
        row[turn % 3][u] = rows[i];
        if constexpr (kLayer) finish.load(max(row[turn % 3][u], 0), res[turn % 3][u]);
    };
    auto put = [&](int turn, int u, int, const float (&v)[V]) __attribute__((always_inline)) {
        if (kLayer && turn == 0 && u == 0) finish.settle();
        const int r = row[turn % 3][u];
        if (r < 0 || c >= a.m) return;
        if constexpr (kLayer) finish.store(r, res[turn % 3][u], v, static_cast<E *>(a.y), a.ldy);
        else Some<E, V>(v).store(static_cast<E *>(a.y) + r * a.ldy, c, a.m);
    };
    T::run(buf0, buf1, acc, tid, fetch, put);
}

// The workgroup's tile of places, first column and part.  False past the last tile.
template <RowsKind KIND, int BM, int BN>
__device__ inline bool row_tile(const RowsArgs &a, int id, int lane, RowTile &rt, int &c0, int &part) {
    const bool tail = KIND != RowsKind::kAdapter;
    const int tiles = KIND == RowsKind::kAdapter ? (a.g.n + BM - 1) / BM : count_tiles(a.g, BM, tail, lane);
    int t;
    if (!row_item(id, tiles, a.m, a.mw, BN, a.parts, t, c0, part)) return false;
    if (KIND == RowsKind::kAdapter) rt = {0, t * BM, min(t * BM + BM, a.g.n)};
    else rt = find_tile(a.g, t, BM, tail, lane);
    return true;
}

// The same for whole tiles of 256 and quarters of them (cut_item).
__device__ inline bool cut_tile(const RowsArgs &a, int id, int lane, RowTile &rt, int &c0, int &quarter) {
    constexpr int BM = 256, BN = 256;
    const int tiles = count_tiles(a.g, BM, false, lane);
    const int tail = (a.g.n - place_of(a.g, a.g.G) + BM - 1) / BM;
    int t;
    if (!cut_item(id, tiles, tail, a.m, a.mw, BN, a.units, t, c0, quarter)) return false;
    rt = find_tile(a.g, t, BM, true, lane);
    if (quarter < 0) return true;
    c0 += (quarter & 1) * (BN / 2);
    rt.p0 += (quarter >> 1) * (BM / 2);
    rt.p1 = min(rt.p1, rt.p0 + BM / 2);
    return rt.p0 < rt.p1 && c0 < a.m;
}

// Stages of a part of the contraction.
__device__ inline void my_stages(int stages, int part, int parts, int &first, int &last) {
    first = static_cast<int>(static_cast<int64_t>(stages) * part / parts);
    last = static_cast<int>(static_cast<int64_t>(stages) * (part + 1) / parts);
}

// Whole chunks of 16 bytes everywhere (rows padded to them with zeros) and at least BN columns: operands go from
// memory straight into LDS (run_stages).  A place without a row computes one that it
// does not store; contraction elements past the last are zeros on both sides.
// Places rt and columns from c0 on, a part of the contraction; kRowsBuf bytes of LDS each (the last two where kRowsDeep) and
// room for BM row numbers.
template <int BM, int BN>
constexpr int kRowsBuf = (BM + BN) * kStageBytes;
template <int BN>
constexpr bool kRowsDeep = BN == 64;       // run_stages_deep

template <class E, RowsKind KIND, bool KS, int BM, int BN, int WR, int WC, bool DEEP = kRowsDeep<BN>>
__device__ __forceinline__ void rows_direct(const RowsArgs &a, const RowTile &rt, int c0, int part, char *buf0, char *buf1, char *buf2, char *buf3, int *rows) {
    using El = Elem<E>;
    constexpr int NT = WR * WC * 64, RF = BM / WR / 16, CF = BN / WC / 16, kBk = El::kBk, kEpc = El::kEpc;
    using XT = Tile<E, false, BM>;
    using WT = Tile<E, KS, BN>;
    constexpr int UX = XT::kChunks / NT, UW = WT::kChunks / NT;
    static_assert(XT::kChunks % NT == 0 && WT::kChunks % NT == 0);
    // a thread's chunks lie a multiple of 16 lines apart: one order of chunks (not in
    // fp32 tiles of 128 columns)
    constexpr int kLinesX = NT / XT::kCpl, kLinesW = NT / WT::kCpl;
    static_assert(kLinesX % 16 == 0);
    constexpr bool kOneOrder = kLinesW % 16 == 0;
    static_assert(kRowsBuf<BM, BN> == XT::kBytes + WT::kBytes);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave / WC, wc = wave % WC;
    for (int i = tid; i < BM; i += NT) rows[i] = rt.p0 + i < rt.p1 ? row_at(a.g, rt.p0 + i) : -1;
    __syncthreads();

    const int k = KIND != RowsKind::kAdapter && rt.g == a.g.G ? 0 : a.k;
    int first, last;
    my_stages((k + kBk - 1) / kBk, part, a.parts, first, last);
    const int xline = tid / XT::kCpl, xe = ((tid % XT::kCpl) ^ XT::swz(xline)) * kEpc;   // first element of the thread's chunks
    const char *xp[UX];
#pragma unroll
    for (int i = 0; i < UX; ++i) {
        const int r = rows[i * kLinesX + xline];
        xp[i] = reinterpret_cast<const char *>(static_cast<const E *>(a.x) + (r < 0 ? 0 : r) * a.ldx + xe + first * kBk);
    }
    const E *w = static_cast<const E *>(a.w) + (KIND == RowsKind::kAdapter || k == 0 ? 0 : rt.g) * a.w_stride;
    const int wline = tid / WT::kCpl, ldw = a.ldw;
    auto chunk = [&](int i) { return ((tid % WT::kCpl) ^ WT::swz(i * kLinesW + wline)) * kEpc; };
    const int we = KS ? wline : chunk(0);
    const char *wp = reinterpret_cast<const char *>(KS ? w + static_cast<int64_t>(wline) * ldw + c0
                                                       : w + static_cast<int64_t>(c0 + wline) * ldw) +
                     (kOneOrder ? chunk(0) * sizeof(E) : 0);
    auto weight = [&](int i) {
        const char *at = wp + static_cast<int64_t>(i) * kLinesW * ldw * sizeof(E);
        return kOneOrder ? at : at + chunk(i) * sizeof(E);
    };
    const int64_t wstep = KS ? static_cast<int64_t>(kBk) * ldw * sizeof(E) : kStageBytes;
    wp += first * wstep;
    auto issue = [&](char *b, int stage, auto...) {
        const int k0 = (first + stage) * kBk;
        if (k0 + kBk <= k) {
#pragma unroll
            for (int i = 0; i < UX; ++i) load_lds(xp[i], b + (i * NT + wave * 64) * 16);
#pragma unroll
            for (int i = 0; i < UW; ++i) load_lds(weight(i), b + XT::kBytes + (i * NT + wave * 64) * 16);
        } else {
            const char *zeros = static_cast<const char *>(a.zeros);
#pragma unroll
            for (int i = 0; i < UX; ++i) load_lds(k0 + xe < k ? xp[i] : zeros, b + (i * NT + wave * 64) * 16);
#pragma unroll
            for (int i = 0; i < UW; ++i) {
                const int e = KS ? i * kLinesW + we : kOneOrder ? we : chunk(i);
                load_lds(k0 + e < k ? weight(i) : zeros, b + XT::kBytes + (i * NT + wave * 64) * 16);
            }
        }
#pragma unroll
        for (int i = 0; i < UX; ++i) xp[i] += kStageBytes;
        wp += wstep;
    };
    f32x4 acc[RF][CF] = {};
    const int stages = last - first, x0 = wr * RF * 16, w0 = wc * CF * 16;
    if constexpr (DEEP) {
        if (stages > 0) run_stages_deep<E, XT, WT, RF, CF, UX + UW>(stages, issue, buf0, buf1, buf2, buf3, x0, w0, lane, acc);
    } else {
        if (stages > 0) run_stages<E, XT, WT, RF, CF>(stages, issue, buf0, buf1, x0, w0, lane, acc);
    }
    __syncthreads();

    if constexpr (KIND == RowsKind::kAdapter)
        if (part == 0) add_adapters<E, KS, BM, BN, WR, WC>(a, rt, c0, buf0, buf0 + XT::kBytes, acc, tid);
    if (a.parts == 1) store_whole_rows<E, KIND, BM, BN, WR, WC>(a, rt, c0, rows, buf0, buf1, acc, tid);
    else store_parts<E, BM, BN, WR, WC>(a, rt, c0, part, acc, tid);
}

// Workgroups of a product by row: a multiple of 8.
template <RowsKind KIND, int BM, int BN>
int64_t rows_blocks(const RowsArgs &a) {
    const int64_t n = a.g.n;
    // a group adds at most one partial tile, and a tile holds at least one row
    const int64_t tiles = KIND == RowsKind::kAdapter ? (n + BM - 1) / BM : n / BM + (n < a.g.G + 1 ? n : a.g.G + 1);
    return (tiles * ((a.m + BN - 1) / BN) * a.parts + 7) / 8 * 8;
}
// Of tiles of 256, cut (cut_item).
template <RowsKind KIND>
int64_t cut_blocks(const RowsArgs &a) { return rows_blocks<KIND, 256, 256>(a) + (3 * a.units / 4 + 24 + 7) / 8 * 8; }

}  // namespace
}  // namespace hwr
