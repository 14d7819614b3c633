// Products by row: every row of a routed batch with the weights of its group
// (kGrouped; kLinear: and what follows in a layer), or with shared weights plus its group's
// low-rank adapter (kAdapter).
#include <algorithm>

#include "rows_device.hpp"

namespace hwr {
namespace {

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
    if (!row_tile<KIND, BM, BN>(a, block_id<NT>(), lane, rt, c0, part)) return;

    for (int i = tid; i < BM; i += NT) rows[i] = rt.p0 + i < rt.p1 ? row_at(a.g, rt.p0 + i) : -1;
    __syncthreads();

    const E *x = static_cast<const E *>(a.x);
    const E *w = static_cast<const E *>(a.w) + (KIND == RowsKind::kAdapter ? 0 : rt.g) * a.w_stride;
    const int k = KIND != RowsKind::kAdapter && rt.g == a.g.G ? 0 : a.k;
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
    store_rows<E, KIND, BM, BN, WR, WC>(a, rt, c0, part, rows, acc, tid);
}

// Tiles of 256 of groups run one to a compute unit, without parts: the last round is cut.
template <RowsKind KIND, int BM>
constexpr bool kCut = BM == 256 && KIND != RowsKind::kAdapter;

template <class E, RowsKind KIND, bool KS, int BM, int BN, int WR, int WC>
__global__ void __launch_bounds__(WR *WC * 64) k_rows_direct(RowsArgs a) {
    // an array each, so that the compiler sees that reads of one do not depend on the
    // loads in flight into the other
    constexpr int kBuf = kRowsBuf<BM, BN>, kMore = kRowsDeep<BN> ? kBuf : 16;
    __shared__ __attribute__((aligned(16))) char buf0[kBuf], buf1[kBuf], buf2[kMore], buf3[kMore];
    __shared__ int rows[BM];
    const int id = block_id<WR * WC * 64>(), lane = threadIdx.x & 63;
    RowTile rt;
    int c0, part = 0;
    if constexpr (kCut<KIND, BM>) {
        int quarter;
        if (!cut_tile(a, id, lane, rt, c0, quarter)) return;
        if (quarter < 0) rows_direct<E, KIND, KS, BM, BN, WR, WC>(a, rt, c0, 0, buf0, buf1, buf2, buf3, rows);
        else rows_direct<E, KIND, KS, BM / 2, BN / 2, WR, WC>(a, rt, c0, 0, buf0, buf1, buf2, buf3, rows);
    } else {
        if (!row_tile<KIND, BM, BN>(a, id, lane, rt, c0, part)) return;
        rows_direct<E, KIND, KS, BM, BN, WR, WC>(a, rt, c0, part, buf0, buf1, buf2, buf3, rows);
    }
}

template <class E, RowsKind KIND, bool KS, int BM, int BN, int WR, int WC, bool DIRECT>
hipError_t go(const RowsArgs &a, hipStream_t s) {
    int64_t blocks = rows_blocks<KIND, BM, BN>(a);
    if constexpr (DIRECT && kCut<KIND, BM>) blocks = cut_blocks<KIND>(a);
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
    if (kind == RowsKind::kLinear) return pick<E, RowsKind::kLinear, true>(p, a, s);
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
// adapter 2,100 x 2048 x 4096 65 / 94, 3,300 x 1024 x 4096 46 / 78, 4,208 x 2200 x 3226 89 / 161; grouped,
// 4 groups, 2048 x 4096 1,600 rows 55 / 39, 2,100 rows 57 / 59, 3,000 rows 58 / 71; layers with gelu, residual and z 1,600 rows
// 71 / 47, 2,100 rows 71 / 72, 3,000 rows 73 / 85, 12,288 rows 512 x 4096 in 8 156 / 153, 2048 x 4096 285 / 322.  fp32 128 from three
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
