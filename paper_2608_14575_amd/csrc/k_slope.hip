// The gradient of a layer's sums: dz = dy act'(z), rounded to the type of the products that
// read it (bf16 12,000 rows 2048 x 2048: dx and dW are off by 0.0023 of themselves, by 0.0017 with dz in fp32, which is
// their own rounding; a dz of 16 bits would double the products), and dbias[g] = sum over the rows of g of dz (before that rounding).
//
// A workgroup takes a few places of one group and a slab of columns, a wave every fourth place; the
// slab's column sums are written for every tile of places and added, in order, by sum_bias.  Bound by memory: dy
// and z are read and dz written once (12,000 rows of 2,048, bf16: 147 MB in 39 us).  Copies that the products want of
// other operands are made by further workgroups of the same launch.
#include <algorithm>

#include "slope_device.hpp"

namespace hwr {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

template <class E, int ACT>
__global__ void __launch_bounds__(kThreads) k_slope(SlopeArgs a, int tiles, PadArgs pads) {
    constexpr int V = Elem<E>::kEpc, kUnroll = 4;
    __shared__ float part[kWaves][64][V];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int slabs = (a.m + 64 * V - 1) / (64 * V);
    const int id = block_id<kThreads>();
    if (id >= tiles) {
        if (id < tiles + kPadBlocks * pads.count) pad_rows<E, kThreads>(pads.m[(id - tiles) / kPadBlocks], (id - tiles) % kPadBlocks);
        return;
    }
    const int t = id / slabs, c = (id % slabs * 64 + lane) * V;
    const RowTile rt = find_tile(a.g, t, a.places, false, lane);
    if (rt.p0 >= rt.p1) return;            // past the last
    float sum[V] = {};
    const int inside = min(V, a.m - c);    // of the chunk
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
                    sum[i] += v;
                    out.e[i] = static_cast<E>(v);
                }
                if (inside < V)            // past the row's end: zeros, which whole chunks of the products go on with
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (i >= inside) out.e[i] = static_cast<E>(0.0f);
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

template <class E>
__global__ void __launch_bounds__(kThreads) k_bias(SlopeArgs a) {
    __shared__ f32x4 part[kThreads];
    sum_bias<E>(a, blockIdx.x, part);
}

template <class E>
hipError_t go(const SlopeArgs &a, int act, const PadArgs &pads, hipStream_t s) {
    const int64_t tiles = static_cast<int64_t>(slope_tiles(a.g.n, a.g.G, a.places)) * ((a.m + 64 * Elem<E>::kEpc - 1) / (64 * Elem<E>::kEpc));
    const int64_t blocks = tiles + kPadBlocks * pads.count;
    if (blocks > INT32_MAX - grid_row(kThreads)) return hipErrorInvalidValue;
    if (blocks > 0) {
        const hipError_t e = with_act(act, [&](auto A) {
            return launch_kernel(k_slope<E, A.value>, wide_grid(blocks, kThreads), dim3(kThreads), 0, s, a, static_cast<int>(tiles), pads);
        });
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

// (as many as count_tiles counts at most, whatever offsets hold)
int slope_tiles(int n, int G, int places) { return n / places + std::min(n, G + 1); }

// Places of a workgroup: as many as leave four to a compute unit, a load of four rows a wave at least
// (fp32 1,003 rows x 390: 24 us with 64 places, 8 with 16).
int slope_places(bool bf16, int n, int G, int m, int cus) {
    const int slab = bf16 ? 512 : 256;
    int places = 64;
    while (places > 16 && static_cast<int64_t>(slope_tiles(n, G, places)) * ((m + slab - 1) / slab) < 4 * cus) places /= 2;
    return places;
}

hipError_t launch_slope(bool bf16, int act, const SlopeArgs &a, const PadArgs &pads, hipStream_t s) {
    return bf16 ? go<__bf16>(a, act, pads, s) : go<float>(a, act, pads, s);
}
hipError_t launch_bias(bool bf16, const SlopeArgs &a, hipStream_t s) {
    const dim3 grid(static_cast<uint32_t>(bias_blocks(a))), block(kThreads);
    return bf16 ? launch_kernel(k_bias<__bf16>, grid, block, 0, s, a) : launch_kernel(k_bias<float>, grid, block, 0, s, a);
}

}  // namespace hwr
