// Low-rank intermediates: low[place] = scale[g] x[row] w_g, with w_g [k][rank]
// (KS) or [rank][k].  The rows are read once, straight into matrix operands; the
// narrow weights come from the L2s.  A workgroup takes the places of one group in
// tiles; its waves take every kWaves-th step of the contraction and add up through LDS.
#include "ops_device.hpp"

namespace hwr {
namespace {

constexpr int kWaves = 8;

// KS: fragment j holds the columns m V + j (as in the products of few rows), V
// fragments whatever the rank; else the columns 16 j + m, as many as the rank takes.
template <class E, bool KS, int RB>
__global__ void __launch_bounds__(kWaves * 64) k_shrink(ShrinkArgs a) {
    using El = Elem<E>;
    constexpr int V = El::kEpc, BM = 16 * RB, kStep = 4 * V, kCols = 16 * V;
    constexpr int kAcc = RB * V;
    __shared__ f32x4 part[kWaves / 2 * kAcc * 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m = lane & 15, q = lane >> 4;
    const int ct = (a.rank + kCols - 1) / kCols;
    const int t = blockIdx.x / ct, c0 = blockIdx.x % ct * kCols;
    if (t >= count_tiles(a.g, BM, false, lane)) return;
    const RowTile rt = find_tile(a.g, t, BM, false, lane);
    const E *w = static_cast<const E *>(a.w) + static_cast<int64_t>(rt.g) * a.k * a.rank;
    const int cols = min(a.rank - c0, kCols);

    // (a place without a row takes row 0; its intermediate is never used)
    const E *x[RB];
    bool in_tile[RB];
#pragma unroll
    for (int i = 0; i < RB; ++i) {
        const int p = rt.p0 + i * 16 + m, r = p < rt.p1 ? row_at(a.g, p) : -1;
        in_tile[i] = p < rt.p1;
        x[i] = static_cast<const E *>(a.x) + (r < 0 ? 0 : r) * a.ldx + q * V;
    }
    f32x4 acc[RB][V] = {};
    u32x4 nw[V], nx[RB];
    const int steps = (a.k + kStep - 1) / kStep;
    auto load = [&](int step) {
        const bool whole = (step + 1) * kStep <= a.k;
#pragma unroll
        for (int i = 0; i < RB; ++i) {
            if (whole) nx[i] = *reinterpret_cast<const typename El::Vec *>(x[i] + step * kStep);
            else nx[i] = load_chunk<E>(x[i], step * kStep, a.k - q * V);
        }
        const int e = step * kStep + q * V;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if constexpr (KS) {
                nw[i] = load_chunk<E>(e + i < a.k ? w + static_cast<int64_t>(e + i) * a.rank + c0 : nullptr, m * V, cols);
            } else {
                if (i * 16 >= cols) break;
                nw[i] = load_chunk<E>(i * 16 + m < cols ? w + static_cast<int64_t>(c0 + i * 16 + m) * a.k : nullptr, e, a.k);
            }
        }
    };
    int step = wave;
    if (step < steps) load(step);
    for (; step < steps; step += kWaves) {
        typename El::Frag fw[V];
        union Chunk { u32x4 v; typename El::Frag f; } fx[RB], u;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if constexpr (KS) {
                fw[j] = column(nw, j);
            } else {
                u.v = nw[j];
                fw[j] = u.f;
            }
        }
#pragma unroll
        for (int i = 0; i < RB; ++i) fx[i].v = nx[i];
        if (step + kWaves < steps) load(step + kWaves);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (!KS && j * 16 >= cols) break;
#pragma unroll
            for (int i = 0; i < RB; ++i) acc[i][j] = El::mma(fw[j], fx[i].f, acc[i][j]);
        }
    }

#pragma unroll
    for (int half = kWaves / 2; half; half /= 2) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int i = 0; i < kAcc; ++i) part[((wave - half) * kAcc + i) * 64 + lane] = acc[i / V][i % V];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int i = 0; i < kAcc; ++i) acc[i / V][i % V] += part[(wave * kAcc + i) * 64 + lane];
        __syncthreads();
    }
    if (wave != 0) return;

    // lane: place m of block i; KS: columns (4 q + e) V + j, else 16 j + 4 q + e.
    // Zeros past the rank (not 0 x infinity).
    const float s = a.scale ? a.scale[rt.g] : 1.0f;
    const int blocks = (a.rank + kRankBlock - 1) / kRankBlock;
#pragma unroll
    for (int i = 0; i < RB; ++i) {
        if (!in_tile[i]) continue;
        char *at = static_cast<char *>(a.low) + static_cast<int64_t>(rt.p0 + i * 16 + m) * blocks * kLowBytes;
        auto put = [&](int c, f32x4 v) {
            if (c0 + c >= blocks * kRankBlock) return;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = c + e < cols ? v[e] * s : 0.0f;
            store_low<E>(at + (c0 + c) / kRankBlock * kLowBytes, (c0 + c) % kRankBlock, v);
        };
#pragma unroll
        for (int j = 0; j < V; j += KS ? 4 : 1)
            if constexpr (KS) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    put((4 * q + e) * V + j, f32x4{acc[i][j][e], acc[i][j + 1][e], acc[i][j + 2][e], acc[i][j + 3][e]});
            } else {
                put(j * 16 + 4 * q, acc[i][j]);
            }
    }
}

template <class E, bool KS>
hipError_t go(const ShrinkArgs &a, int cus, hipStream_t s) {
    constexpr int kCols = 16 * Elem<E>::kEpc;
    const int ct = (a.rank + kCols - 1) / kCols;
    auto tiles = [&](int bm) { return static_cast<uint32_t>(a.g.n / bm + (a.g.n < a.g.G ? a.g.n : a.g.G)); };
    // two blocks of rows share the weights' loads where that leaves the device full
    if (a.g.n >= 32 * 2 * cus) return launch_kernel(k_shrink<E, KS, 2>, dim3(tiles(32) * ct), dim3(kWaves * 64), 0, s, a);
    return launch_kernel(k_shrink<E, KS, 1>, dim3(tiles(16) * ct), dim3(kWaves * 64), 0, s, a);
}

}  // namespace

hipError_t launch_shrink(bool bf16, bool ks, const ShrinkArgs &a, int cus, hipStream_t s) {
    if (bf16) return ks ? go<__bf16, true>(a, cus, s) : go<__bf16, false>(a, cus, s);
    return ks ? go<float, true>(a, cus, s) : go<float, false>(a, cus, s);
}

}  // namespace hwr
