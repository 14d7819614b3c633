// Rows by group: a stable counting sort of the routed rows.
#include "ops_device.hpp"

namespace hwr {
namespace {

constexpr int kGroupThreads = 256;
constexpr int kGroupRows = 4096;      // rows of a workgroup

__device__ inline int group_key(const GroupRowsArgs &a, int row) {
    int c = a.choice[row];
    if (a.table) c = static_cast<unsigned>(c) < static_cast<unsigned>(a.n_table) ? a.table[c] : -1;
    return static_cast<unsigned>(c) < static_cast<unsigned>(a.G) ? c : a.G;
}

// hist[key][block]: rows of each key in the block's range
__global__ void __launch_bounds__(kGroupThreads) k_group_count(GroupRowsArgs a) {
    __shared__ int h[kMaxPairs + 1];
    for (int i = threadIdx.x; i <= a.G; i += kGroupThreads) h[i] = 0;
    __syncthreads();
    const int r0 = blockIdx.x * kGroupRows, r1 = min(r0 + kGroupRows, a.n);
    for (int r = r0 + threadIdx.x; r < r1; r += kGroupThreads) atomicAdd(&h[group_key(a, r)], 1);
    __syncthreads();
    for (int i = threadIdx.x; i <= a.G; i += kGroupThreads) a.hist[static_cast<int64_t>(i) * a.blocks + blockIdx.x] = h[i];
}

// hist in place: place of each block's first row of each key; offsets
__global__ void __launch_bounds__(1024) k_group_scan(GroupRowsArgs a) {
    __shared__ int part[16], total;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int count = (a.G + 1) * a.blocks;
    int base = 0;
    for (int i0 = 0; i0 < count; i0 += 1024) {
        const int i = i0 + threadIdx.x;
        const int v = i < count ? a.hist[i] : 0;
        const int upto = wave_scan(v, lane);
        if (lane == 63) part[wave] = upto;
        __syncthreads();
        int before = base;
        for (int w = 0; w < wave; ++w) before += part[w];
        if (i < count) {
            a.hist[i] = before + upto - v;
            if (i % a.blocks == 0 && i / a.blocks <= a.G) a.offsets[i / a.blocks] = before + upto - v;
        }
        if (threadIdx.x == 1023) total = before + upto;
        __syncthreads();
        base = total;
    }
}

__global__ void __launch_bounds__(64) k_group_place(GroupRowsArgs a) {
    __shared__ int next[kMaxPairs + 1];
    const int lane = threadIdx.x;
    for (int i = lane; i <= a.G; i += 64) next[i] = a.hist[static_cast<int64_t>(i) * a.blocks + blockIdx.x];
    __syncthreads();
    const int r0 = blockIdx.x * kGroupRows, r1 = min(r0 + kGroupRows, a.n);
    for (int b = r0; b < r1; b += 64) {
        const int r = b + lane;
        const int key = r < r1 ? group_key(a, r) : -1;
        // lanes of the same key: rank among them, and the last one advances the counter
        uint64_t same = __ballot(key >= 0);
        for (int bit = 0; (a.G >> bit) != 0; ++bit) {
            const uint64_t set = __ballot((key >> bit) & 1);
            same &= ((key >> bit) & 1) ? set : ~set;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        const int at = key >= 0 ? next[key] : 0;
        __syncthreads();
        if (key >= 0) {
            a.order[at + rank] = r;
            if (rank == __popcll(same) - 1) next[key] = at + rank + 1;
        }
        __syncthreads();
    }
}

}  // namespace

int group_rows_blocks(int n) { return n > 0 ? (n + kGroupRows - 1) / kGroupRows : 1; }

hipError_t launch_group_rows(const GroupRowsArgs &a, hipStream_t s) {
    hipError_t e = launch_kernel(k_group_count, dim3(a.blocks), dim3(kGroupThreads), 0, s, a);
    if (e != hipSuccess) return e;
    e = launch_kernel(k_group_scan, dim3(1), dim3(1024), 0, s, a);
    if (e != hipSuccess) return e;
    return launch_kernel(k_group_place, dim3(a.blocks), dim3(64), 0, s, a);
}

}  // namespace hwr
