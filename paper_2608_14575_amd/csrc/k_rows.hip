// Products by row: every row of a routed batch with the weights of its group
// (kGrouped), with shared weights plus its group's low-rank adapter (kAdapter),
// or into the low-rank intermediate (kShrink).
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

    const bool tail = KIND == RowsKind::kGrouped;
    const int tiles = KIND == RowsKind::kAdapter ? (a.g.n + BM - 1) / BM : count_tiles(a.g, BM, tail, lane);
    const int ct = (a.m + BN - 1) / BN;
    const int item = xcd_item(blockIdx.x, tiles * ct);
    if (item < 0) return;
    const int panel = item / (8 * ct) * 8, in = item - panel * ct, rp = min(8, tiles - panel);
    const int t = panel + in % rp, c0 = in / rp * BN;
    RowTile rt;
    if (KIND == RowsKind::kAdapter) rt = {0, t * BM, min(t * BM + BM, a.g.n)};
    else rt = find_tile(a.g, t, BM, tail, lane);

    for (int i = tid; i < BM; i += NT) rows[i] = rt.p0 + i < rt.p1 ? row_at(a.g, rt.p0 + i) : -1;
    __syncthreads();

    const E *x = static_cast<const E *>(a.x);
    const E *w = static_cast<const E *>(a.w) + (KIND == RowsKind::kAdapter ? 0 : rt.g) * a.w_stride;
    const int k = KIND == RowsKind::kGrouped && rt.g == a.g.G ? 0 : a.k;

    auto weights = [&](const E *base, int k0, int klen) {   // KS: lines are elements; else columns
        return [=, &a](int line, int c) {
            if constexpr (KS) {
                return load_chunk<E>(k0 + line < klen ? base + static_cast<int64_t>(k0 + line) * a.m : nullptr,
                                     c0 + c * El::kEpc, a.m);
            } else {
                return load_chunk<E>(c0 + line < a.m ? base + static_cast<int64_t>(c0 + line) * klen : nullptr,
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
    if (k > 0) {
        gx.load(inputs(0), tid);
        gw.load(weights(w, 0, k), tid);
    }
    for (int k0 = 0; k0 < k; k0 += kBk) {
        gx.store(sx, tid);
        gw.store(sw, tid);
        __syncthreads();
        if (k0 + kBk < k) {
            gx.load(inputs(k0 + kBk), tid);
            gw.load(weights(w, k0 + kBk, k), tid);
        }
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
            typename El::Frag fw[CF], fx[RF];
#pragma unroll
            for (int j = 0; j < CF; ++j) fw[j] = WT::frag(sw, (wc * CF + j) * 16, sub, lane);
#pragma unroll
            for (int i = 0; i < RF; ++i) fx[i] = XT::frag(sx, (wr * RF + i) * 16, sub, lane);
#pragma unroll
            for (int i = 0; i < RF; ++i)
#pragma unroll
                for (int j = 0; j < CF; ++j) acc[i][j] = El::mma(fw[j], fx[i], acc[i][j]);
        }
        __syncthreads();
    }

    // The adapters of the tile's groups: one stage for every 32 of the rank, whose
    // contraction is hi and lo against the same weights in bf16.  Only the rows of
    // the group take the result (a zero would turn another group's infinity into NaN).
    if constexpr (KIND == RowsKind::kAdapter) {
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
                gx.store(sx, tid);
                gw.store(sw, tid);
                __syncthreads();
#pragma unroll
                for (int sub = 0; sub < 2; ++sub) {
                    typename El::Frag fw[CF];
#pragma unroll
                    for (int j = 0; j < CF; ++j) fw[j] = WT::frag(sw, (wc * CF + j) * 16, sub, lane);
#pragma unroll
                    for (int i = 0; i < RF; ++i) {
                        const int f0 = rt.p0 + (wr * RF + i) * 16;
                        if (f0 + 16 <= lo || f0 >= hi) continue;
                        const typename El::Frag fx = XT::frag(sx, (wr * RF + i) * 16, sub, lane);
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

    const int q = lane >> 4;
    if constexpr (KIND == RowsKind::kShrink) {
        const float s = a.scale ? a.scale[rt.g] : 1.0f;
        const int blocks = (a.m + kRankBlock - 1) / kRankBlock;
#pragma unroll
        for (int i = 0; i < RF; ++i) {
            const int p = rt.p0 + (wr * RF + i) * 16 + (lane & 15);
            if (p >= rt.p1) continue;
#pragma unroll
            for (int j = 0; j < CF; ++j) {
                const int c = c0 + (wc * CF + j) * 16 + q * 4;
                if (c >= blocks * kRankBlock) continue;
                char *at = static_cast<char *>(a.y) + (static_cast<int64_t>(p) * blocks + c / kRankBlock) * kLowBytes;
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = c + e < a.m ? acc[i][j][e] * s : 0.0f;   // not 0 * inf past the rank
                if constexpr (sizeof(E) == 4) {
                    *reinterpret_cast<f32x4 *>(at + c % kRankBlock * 4) = v;
                } else {
                    bf16x4 hi, lo;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        hi[e] = static_cast<__bf16>(v[e]);
                        const float h = static_cast<float>(hi[e]);
                        lo[e] = static_cast<__bf16>(__builtin_isfinite(h) ? v[e] - h : 0.0f);
                    }
                    *reinterpret_cast<bf16x4 *>(at + c % kRankBlock * 2) = hi;
                    *reinterpret_cast<bf16x4 *>(at + 64 + c % kRankBlock * 2) = lo;
                }
            }
        }
    } else {
        E *y = static_cast<E *>(a.y);
        const bool vec = (a.m & 3) == 0 && (a.ldy & 3) == 0 && (reinterpret_cast<uintptr_t>(y) & (4 * sizeof(E) - 1)) == 0;
#pragma unroll
        for (int i = 0; i < RF; ++i) {
            const int r = rows[(wr * RF + i) * 16 + (lane & 15)];
            if (r < 0) continue;
            E *line = y + r * a.ldy;
#pragma unroll
            for (int j = 0; j < CF; ++j) {
                const int c = c0 + (wc * CF + j) * 16 + q * 4;
                typename El::Out4 o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = static_cast<E>(acc[i][j][e]);
                if (vec && c < a.m) *reinterpret_cast<typename El::Out4 *>(line + c) = o;
                else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (c + e < a.m) line[c + e] = o[e];
                }
            }
        }
    }
}

template <class E, RowsKind KIND, bool KS, int BM, int BN, int WR, int WC>
hipError_t go(const RowsArgs &a, hipStream_t s) {
    const int64_t n = a.g.n;
    // a group adds at most one partial tile, and a tile holds at least one row
    const int64_t tiles = KIND == RowsKind::kAdapter ? (n + BM - 1) / BM : n / BM + (n < a.g.G + 1 ? n : a.g.G + 1);
    const int64_t items = tiles * ((a.m + BN - 1) / BN);
    const int64_t blocks = (items + 7) / 8 * 8;
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    return launch_kernel(k_rows<E, KIND, KS, BM, BN, WR, WC>, dim3(static_cast<uint32_t>(blocks)), dim3(WR * WC * 64), 0, s, a);
}

template <class E, RowsKind KIND, bool KS>
hipError_t pick(const RowsArgs &a, hipStream_t s) {
    if constexpr (KIND == RowsKind::kShrink) {
        if (a.m <= 32) return go<E, KIND, KS, 32, 32, 2, 1>(a, s);
        return go<E, KIND, KS, 32, 64, 2, 2>(a, s);
    } else {
        const bool small = KIND == RowsKind::kAdapter ? a.g.n <= 64 : a.g.n <= 64 * a.g.G;
        if (small) return go<E, KIND, KS, 16, 64, 1, 4>(a, s);
        return go<E, KIND, KS, 128, 128, 2, 2>(a, s);
    }
}

template <class E>
hipError_t pick_kind(RowsKind kind, bool ks, const RowsArgs &a, hipStream_t s) {
    switch (kind) {
    case RowsKind::kGrouped: return ks ? pick<E, RowsKind::kGrouped, true>(a, s) : pick<E, RowsKind::kGrouped, false>(a, s);
    case RowsKind::kAdapter: return ks ? pick<E, RowsKind::kAdapter, true>(a, s) : pick<E, RowsKind::kAdapter, false>(a, s);
    default: return ks ? pick<E, RowsKind::kShrink, true>(a, s) : pick<E, RowsKind::kShrink, false>(a, s);
    }
}

}  // namespace

hipError_t launch_rows(bool bf16, RowsKind kind, bool ks, const RowsArgs &a, int cus, hipStream_t s) {
    (void)cus;
    return bf16 ? pick_kind<__bf16>(kind, ks, a, s) : pick_kind<float>(kind, ks, a, s);
}

}  // namespace hwr
