// Device code of a layer's gradient before and beside its products (k_slope.hip, k_pad.hip; k_grad.hip).
#pragma once

#include "ops_act.hpp"

namespace hwr {
namespace {

// Rows padded to whole chunks: workgroup `block` of kPadBlocks.  (us, 2,048 / 1,024 of them: gradients of bf16 9,000 x 1024 x 2050 in 4
// groups 193.9 / 197.3, of layers 9,000 x 1023 x 2048 161.2 / 162.6.)
constexpr int kPadBlocks = 2048;
template <class E, int NT>
__device__ inline void pad_rows(const PadArgs::Matrix &m, int block) {
    constexpr int kEpc = Elem<E>::kEpc;
    const int per = (m.width + kEpc - 1) / kEpc;            // chunks of a row
    const int64_t chunks = m.rows * per, step = static_cast<int64_t>(kPadBlocks) * NT;
    for (int64_t i = static_cast<int64_t>(block) * NT + threadIdx.x; i < chunks; i += step) {
        const int64_t row = i / per;
        const int c = static_cast<int>(i - row * per) * kEpc;
        reinterpret_cast<u32x4 *>(m.dst)[i] = load_chunk<E>(static_cast<const E *>(m.src) + row * m.ld, c, m.width);
    }
}

// dbias[g][c]: the sums of the group's tiles.  Workgroup `id` of bias_blocks, 256 f32x4 of LDS.  The first four waves
// add them up in workgroups of any size: the order of additions, and so the bits, are the same.
template <class E>
__device__ inline void sum_bias(const SlopeArgs &a, int id, f32x4 *part) {
    constexpr int kWaves = 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int slabs = (a.m + 255) / 256, g = id / slabs, c = (id % slabs * 64 + lane) * 4;
    // (tiles are capped as count_tiles caps them: offsets may hold anything)
    const int all = count_tiles(a.g, a.places, false, lane);
    int first = 0, p0, p1;
    for (int b = 0; b < g; b += 64) {
        int mine = b + lane < g ? lane_tiles(a.g, b + lane, a.places, false, p0, p1) : 0;
#pragma unroll
        for (int d = 32; d; d >>= 1) mine = min(mine + __shfl_xor(mine, d), all);
        first = min(first + mine, all);
    }
    const int last = min(first + lane_tiles(a.g, g, a.places, false, p0, p1), all);
    f32x4 sum = {};
    if (wave < kWaves && c < a.m) {
#pragma unroll 8
        for (int t = first + wave; t < last; t += kWaves)
            sum += *reinterpret_cast<const f32x4 *>(a.partial + static_cast<int64_t>(t) * a.m_pad + c);
    }
    if (wave < kWaves) part[wave * 64 + lane] = sum;
    __syncthreads();
    if (wave != 0 || c >= a.m) return;
    for (int w = 1; w < kWaves; ++w) sum += part[w * 64 + lane];
    store_four<E>(static_cast<E *>(a.dbias) + static_cast<int64_t>(g) * a.m, c, a.m, sum);
}

__host__ __device__ inline int bias_blocks(const SlopeArgs &a) { return (a.m + 255) / 256 * a.g.G; }

}  // namespace
}  // namespace hwr
