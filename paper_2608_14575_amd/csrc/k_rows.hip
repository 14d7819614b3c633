// Products by row: every row of a routed batch with the weights of its group
// (kGrouped), or with shared weights plus its group's low-rank adapter (kAdapter).
#include <algorithm>

#include "ops_device.hpp"

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
__device__ inline void store_rows(const RowsArgs &a, const RowTile &rt, int c0, int part, const int *rows,
                                  const f32x4 (&acc)[BM / WR / 16][BN / WC / 16], int tid) {
    constexpr int RF = BM / WR / 16, CF = BN / WC / 16;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave / WC, wc = wave % WC;
    const int q = lane >> 4;
    if (a.parts > 1) {
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
        return;
    }
    E *y = static_cast<E *>(a.y);
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

// The workgroup's tile of places, first column and part.  False past the last tile.
template <RowsKind KIND, int BM, int BN, int NT>
__device__ inline bool my_tile(const RowsArgs &a, int lane, RowTile &rt, int &c0, int &part) {
    const bool tail = KIND == RowsKind::kGrouped;
    const int tiles = KIND == RowsKind::kAdapter ? (a.g.n + BM - 1) / BM : count_tiles(a.g, BM, tail, lane);
    int t;
    if (!row_item(block_id<NT>(), tiles, a.m, a.mw, BN, a.parts, t, c0, part)) return false;
    if (KIND == RowsKind::kAdapter) rt = {0, t * BM, min(t * BM + BM, a.g.n)};
    else rt = find_tile(a.g, t, BM, tail, lane);
    return true;
}

// Stages of a part of the contraction.
__device__ inline void my_stages(int stages, int part, int parts, int &first, int &last) {
    first = static_cast<int>(static_cast<int64_t>(stages) * part / parts);
    last = static_cast<int>(static_cast<int64_t>(stages) * (part + 1) / parts);
}

// Any widths, strides and alignment: operands pass through registers.
template <class E, RowsKind KIND, bool KS, int BM, int BN, int WR, int WC>
__global__ void __launch_bounds__(WR *WC * 64) k_rows(RowsArgs a) {
    using El = Elem<E>;
    constexpr int NT = WR * WC * 64, RF = BM / WR / 16, CF = BN / WC / 16, kBk = El::kBk;
    using XT = Tile<E, false, BM>;
    using WT = Tile<E, KS, BN>;
    __shared__ __attribute__((aligned(16))) char sx[XT::kBytes], sw[WT::kBytes];
    __shared__ int rows[BM];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave / WC, wc = wave % WC;
    RowTile rt;
    int c0, part;
    if (!my_tile<KIND, BM, BN, NT>(a, lane, rt, c0, part)) return;

    for (int i = tid; i < BM; i += NT) rows[i] = rt.p0 + i < rt.p1 ? row_at(a.g, rt.p0 + i) : -1;
    __syncthreads();

    const E *x = static_cast<const E *>(a.x);
    const E *w = static_cast<const E *>(a.w) + (KIND == RowsKind::kAdapter ? 0 : rt.g) * a.w_stride;
    const int k = KIND == RowsKind::kGrouped && rt.g == a.g.G ? 0 : a.k;
    int first, last;
    my_stages((k + kBk - 1) / kBk, part, a.parts, first, last);

    auto weights = [&](const E *base, int k0, int klen) {   // KS: lines are elements; else columns
        return [=, &a](int line, int c) {
            if constexpr (KS) {
                return load_chunk<E>(k0 + line < klen ? base + static_cast<int64_t>(k0 + line) * a.ldw : nullptr,
                                     c0 + c * El::kEpc, a.m);
            } else {
                return load_chunk<E>(c0 + line < a.m ? base + static_cast<int64_t>(c0 + line) * a.ldw : nullptr,
                                     k0 + c * El::kEpc, klen);
            }
        };
    };
    auto inputs = [&](int k0) {
        return [=, &a](int line, int c) {
            const int r = rows[line];
            return load_chunk<E>(r >= 0 ? x + r * a.ldx : nullptr, k0 + c * El::kEpc, k);
        };
    };

    f32x4 acc[RF][CF] = {};
    Staged<E, false, BM, NT> gx;
    Staged<E, KS, BN, NT> gw;
    if (first < last) {
        gx.load(inputs(first * kBk), tid);
        gw.load(weights(w, first * kBk, k), tid);
    }
    for (int stage = first; stage < last; ++stage) {
        gx.store(sx, tid);
        gw.store(sw, tid);
        __syncthreads();
        if (stage + 1 < last) {
            gx.load(inputs((stage + 1) * kBk), tid);
            gw.load(weights(w, (stage + 1) * kBk, k), tid);
        }
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
            typename El::Frag fw[CF], fx[RF];
#pragma unroll
            for (int j = 0; j < CF; ++j) fw[j] = WT::frag(sw, 0, (wc * CF + j) * 16, sub, WT::base(lane));
#pragma unroll
            for (int i = 0; i < RF; ++i) fx[i] = XT::frag(sx, 0, (wr * RF + i) * 16, sub, XT::base(lane));
#pragma unroll
            for (int i = 0; i < RF; ++i)
#pragma unroll
                for (int j = 0; j < CF; ++j) acc[i][j] = El::mma(fw[j], fx[i], acc[i][j]);
        }
        __syncthreads();
    }

    if constexpr (KIND == RowsKind::kAdapter)
        if (part == 0) add_adapters<E, KS, BM, BN, WR, WC>(a, rt, c0, sx, sw, acc, tid);
    store_rows<E, BM, BN, WR, WC>(a, rt, c0, part, rows, acc, tid);
}

// Whole chunks of 16 bytes everywhere (rows padded to them with zeros) and at least BN columns: operands go from
// memory straight into LDS (run_stages).  A place without a row computes one that it
// does not store; contraction elements past the last are zeros on both sides.
template <class E, RowsKind KIND, bool KS, int BM, int BN, int WR, int WC>
__global__ void __launch_bounds__(WR *WC * 64) k_rows_direct(RowsArgs a) {
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
    constexpr int kBuf = XT::kBytes + WT::kBytes;
    // an array each, so that the compiler sees that reads of one do not depend on the
    // loads in flight into the other
    __shared__ __attribute__((aligned(16))) char buf0[kBuf], buf1[kBuf];
    constexpr bool kDeep = BN == 64;       // run_stages_deep
    __shared__ __attribute__((aligned(16))) char buf2[kDeep ? kBuf : 16], buf3[kDeep ? kBuf : 16];
    __shared__ int rows[BM];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave / WC, wc = wave % WC;
    RowTile rt;
    int c0, part;
    if (!my_tile<KIND, BM, BN, NT>(a, lane, rt, c0, part)) return;
    for (int i = tid; i < BM; i += NT) rows[i] = rt.p0 + i < rt.p1 ? row_at(a.g, rt.p0 + i) : -1;
    __syncthreads();

    const int k = KIND == RowsKind::kGrouped && rt.g == a.g.G ? 0 : a.k;
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
    if constexpr (kDeep) {
        if (stages > 0) run_stages_deep<E, XT, WT, RF, CF, UX + UW>(stages, issue, buf0, buf1, buf2, buf3, x0, w0, lane, acc);
    } else {
        if (stages > 0) run_stages<E, XT, WT, RF, CF>(stages, issue, buf0, buf1, x0, w0, lane, acc);
    }
    __syncthreads();

    if constexpr (KIND == RowsKind::kAdapter)
        if (part == 0) add_adapters<E, KS, BM, BN, WR, WC>(a, rt, c0, buf0, buf0 + XT::kBytes, acc, tid);
    store_rows<E, BM, BN, WR, WC>(a, rt, c0, part, rows, acc, tid);
}

template <class E, RowsKind KIND, bool KS, int BM, int BN, int WR, int WC, bool DIRECT>
hipError_t go(const RowsArgs &a, hipStream_t s) {
    const int64_t n = a.g.n;
    // a group adds at most one partial tile, and a tile holds at least one row
    const int64_t tiles = KIND == RowsKind::kAdapter ? (n + BM - 1) / BM : n / BM + (n < a.g.G + 1 ? n : a.g.G + 1);
    const int64_t items = tiles * ((a.m + BN - 1) / BN) * a.parts;
    const int64_t blocks = (items + 7) / 8 * 8;
    if (blocks > INT32_MAX - grid_row(WR * WC * 64)) return hipErrorInvalidValue;
    const dim3 grid = wide_grid(blocks, WR * WC * 64), block(WR * WC * 64);
    if constexpr (DIRECT) return launch_kernel(k_rows_direct<E, KIND, KS, BM, BN, WR, WC>, grid, block, 0, s, a);
    else return launch_kernel(k_rows<E, KIND, KS, BM, BN, WR, WC>, grid, block, 0, s, a);
}

template <class E, RowsKind KIND, bool KS>
hipError_t pick(const RowsPlan &p, const RowsArgs &a, hipStream_t s) {
    if (p.direct) {
        if constexpr (sizeof(E) == 2) {
            if (p.bm == 256) return go<E, KIND, KS, 256, 256, 2, 4, true>(a, s);
        } else {
            if (p.bm == 32) return go<E, KIND, KS, 32, 64, 1, 4, true>(a, s);
        }
        if (p.bm == 128) return go<E, KIND, KS, 128, 128, 2, 2, true>(a, s);
        return go<E, KIND, KS, 64, 64, 2, 2, true>(a, s);
    }
    if (p.bm == 128) return go<E, KIND, KS, 128, 128, 2, 2, false>(a, s);
    return go<E, KIND, KS, 64, 64, 2, 2, false>(a, s);
}

template <class E>
hipError_t pick_kind(RowsKind kind, bool ks, const RowsPlan &p, const RowsArgs &a, hipStream_t s) {
    if (kind == RowsKind::kGrouped)
        return ks ? pick<E, RowsKind::kGrouped, true>(p, a, s) : pick<E, RowsKind::kGrouped, false>(p, a, s);
    return ks ? pick<E, RowsKind::kAdapter, true>(p, a, s) : pick<E, RowsKind::kAdapter, false>(p, a, s);
}

// Rows and weights in whole, aligned chunks of 16 bytes.
bool whole_chunks(bool bf16, bool ks, const RowsArgs &a) {
    const int epc = bf16 ? 8 : 4;
    const auto ptrs = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w);
    return (ptrs & 15) == 0 && a.ldx % epc == 0 && a.ldw % epc == 0 && a.w_stride % epc == 0 && (a.padded || a.k % epc == 0) &&
           (!ks || a.mw % epc == 0);
}

}  // namespace

// The largest tile that gives most compute units a workgroup: 256 half of them with an
// adapter (whose tiles of 128 take 260 to 271 registers in bf16 and so run one workgroup on a
// compute unit; without an adapter 174 and two), three of four without.  us, 256 / 128:
// adapter 2,100 x 2048 x 4096 72 / 98, 3,300 x 1024 x 4096 50 / 80, 4,208 x 2200 x 3226 89 / 153; grouped,
// 4 groups, 2048 x 4096 1,600 rows 56 / 41, 2,100 rows 58 / 61, 3,000 rows 61 / 74.  fp32 128 from three
// a compute unit, for below that rounds and the ends of groups cost more (64 / 128: 4,096 x
// 1536 x 1536 in one group 165 / 202, 4,096 x 1024 x 1024 in 32 115 / 137, with adapters 4,096 x 1024 x
// 1536 in 8 136 / 155; 16,384 x 1024 x 1536 in one 444 / 406).  Where even small tiles leave units
// idle, parts of the contraction of at least four stages.
RowsPlan rows_plan(bool bf16, RowsKind kind, bool ks, const RowsArgs &a, int cus) {
    auto tiles = [&](int64_t bm, int64_t bn) {          // (at most n groups hold a row)
        return (a.g.n / bm + (kind == RowsKind::kAdapter ? 1 : std::min(a.g.n, a.g.G))) * ((a.m + bn - 1) / bn);
    };
    RowsPlan p{whole_chunks(bf16, ks, a) && a.mw >= 64, 64, 64, 1};
    const int stages = (a.k + (bf16 ? 63 : 31)) / (bf16 ? 64 : 32);
    const int enough = kind == RowsKind::kAdapter ? cus / 2 : cus * 3 / 4;
    if (p.direct && bf16 && a.mw >= 256 && tiles(256, 256) >= enough) p.bm = p.bn = 256;
    else if ((!p.direct || a.mw >= 128) && tiles(128, 128) >= (bf16 || !p.direct ? 1 : 3) * cus) p.bm = p.bn = 128;
    else if (p.direct && !bf16 && tiles(64, 64) < 2 * cus) p.bm = 32;
    while (p.bm < 256 && tiles(p.bm, p.bn) * p.parts < cus && stages >= 8 * p.parts) p.parts *= 2;
    return p;
}

hipError_t launch_rows(bool bf16, RowsKind kind, bool ks, const RowsArgs &a, int cus, hipStream_t s) {
    const RowsPlan p = rows_plan(bf16, kind, ks, a, cus);
    return bf16 ? pick_kind<__bf16>(kind, ks, p, a, s) : pick_kind<float>(kind, ks, p, a, s);
}

}  // namespace hwr
