// The gradient of a layer's sums: dz = dy act'(z), rounded to the type of the products that
// read it, and dbias[g] = sum over the rows of g of dz (before that rounding).
//
// A workgroup takes kPlaces places of one group and a slab of columns, a wave every fourth place; the
// slab's column sums are written for every tile of places and added, in order, by k_bias.  Bound by memory: dy
// and z are read and dz written once.
#include <algorithm>

#include "ops_act.hpp"

namespace hwr {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64, kPlaces = 64;

template <class E, int ACT>
__global__ void __launch_bounds__(kThreads) k_slope(SlopeArgs a) {
    constexpr int V = Elem<E>::kEpc, kUnroll = 4;
    __shared__ float part[kWaves][64][V];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int slabs = (a.m + 64 * V - 1) / (64 * V);
    const int id = block_id<kThreads>(), t = id / slabs, c = (id % slabs * 64 + lane) * V;
    if (t >= count_tiles(a.g, kPlaces, false, lane)) return;
    const RowTile rt = find_tile(a.g, t, kPlaces, false, lane);
    float sum[V] = {};
    if (c < a.m) {
        for (int p0 = rt.p0 + wave; p0 < rt.p1; p0 += kUnroll * kWaves) {
            int row[kUnroll];
            u32x4 dy[kUnroll], z[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) row[u] = p0 + u * kWaves < rt.p1 ? row_at(a.g, p0 + u * kWaves) : -1;
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int64_t r = row[u];
                dy[u] = load_chunk<E>(r < 0 ? nullptr : static_cast<const E *>(a.dy) + r * a.lddy, c, a.m);
                if constexpr (ACT != HWR_ACT_NONE) z[u] = load_chunk<E>(r < 0 ? nullptr : static_cast<const E *>(a.z) + r * a.ldz, c, a.m);
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                if (row[u] < 0) continue;
                union { u32x4 v; E e[V]; } d, zz, out;
                d.v = dy[u];
                if constexpr (ACT != HWR_ACT_NONE) zz.v = z[u];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float v = static_cast<float>(d.e[i]);
                    if constexpr (ACT != HWR_ACT_NONE) v *= slope<E, ACT>(static_cast<float>(zz.e[i]));
                    // (past the row's end: zeros, which whole chunks of the products go on with)
                    if (c + i >= a.m) v = 0.0f;
                    sum[i] += v;
                    out.e[i] = static_cast<E>(v);
                }
                if (a.dz) *reinterpret_cast<u32x4 *>(static_cast<E *>(a.dz) + static_cast<int64_t>(row[u]) * a.lddz + c) = out.v;
            }
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int i = 0; i < V; ++i) part[wave][lane][i] = sum[i];
    __syncthreads();
    if (wave != 0 || c >= a.m) return;
#pragma unroll
    for (int i = 0; i < V; ++i)
        for (int w = 1; w < kWaves; ++w) sum[i] += part[w][lane][i];
#pragma unroll
    for (int i = 0; i < V; i += 4)
        *reinterpret_cast<f32x4 *>(a.partial + static_cast<int64_t>(t) * a.m_pad + c + i) = f32x4{sum[i], sum[i + 1], sum[i + 2], sum[i + 3]};
}

// dbias[g][c]: the sums of the group's tiles.
template <class E>
__global__ void __launch_bounds__(kThreads) k_bias(SlopeArgs a) {
    __shared__ f32x4 part[kWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int slabs = (a.m + 255) / 256, g = blockIdx.x / slabs, c = (blockIdx.x % slabs * 64 + lane) * 4;
    // (tiles are capped as count_tiles caps them: offsets may hold anything)
    const int all = count_tiles(a.g, kPlaces, false, lane);
    int first = 0, p0, p1;
    for (int b = 0; b < g; b += 64) {
        int mine = b + lane < g ? lane_tiles(a.g, b + lane, kPlaces, false, p0, p1) : 0;
#pragma unroll
        for (int d = 32; d; d >>= 1) mine = min(mine + __shfl_xor(mine, d), all);
        first = min(first + mine, all);
    }
    const int last = min(first + lane_tiles(a.g, g, kPlaces, false, p0, p1), all);
    f32x4 sum = {};
    if (c < a.m) {
#pragma unroll 8
        for (int t = first + wave; t < last; t += kWaves)
            sum += *reinterpret_cast<const f32x4 *>(a.partial + static_cast<int64_t>(t) * a.m_pad + c);
    }
    part[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || c >= a.m) return;
    for (int w = 1; w < kWaves; ++w) sum += part[w][lane];
    store_four<E>(static_cast<E *>(a.dbias) + static_cast<int64_t>(g) * a.m, c, a.m, sum);
}

template <class E>
hipError_t go(const SlopeArgs &a, int act, hipStream_t s) {
    const int64_t blocks = static_cast<int64_t>(slope_tiles(a.g.n, a.g.G)) * ((a.m + 64 * Elem<E>::kEpc - 1) / (64 * Elem<E>::kEpc));
    if (blocks > INT32_MAX - grid_row(kThreads)) return hipErrorInvalidValue;
    if (blocks > 0) {
        const hipError_t e = with_act(act, [&](auto A) {
            return launch_kernel(k_slope<E, A.value>, wide_grid(blocks, kThreads), dim3(kThreads), 0, s, a);
        });
        if (e != hipSuccess) return e;
    }
    if (!a.dbias) return hipSuccess;
    return launch_kernel(k_bias<E>, dim3(static_cast<uint32_t>((a.m + 255) / 256 * a.g.G)), dim3(kThreads), 0, s, a);
}

}  // namespace

// (as many as count_tiles counts at most, whatever offsets hold)
int slope_tiles(int n, int G) { return n / kPlaces + std::min(n, G + 1); }

hipError_t launch_slope(bool bf16, int act, const SlopeArgs &a, hipStream_t s) {
    return bf16 ? go<__bf16>(a, act, s) : go<float>(a, act, s);
}

}  // namespace hwr
