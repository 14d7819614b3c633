// Rows by group: a stable counting sort of the routed rows.
//
// A wave takes 512 (several blocks: 256) rows in order, 64 at a time, and counts them by
// key in LDS.  A row's place is where its key begins, plus the rows of the key before
// the wave, plus those before the row in the wave: lanes of one key find each other by
// a ballot for each bit of the key.  Up to 8,192 rows fit one workgroup and one
// launch; more take two, counts by block and the places, or three with a scan over the
// blocks of every key between them (two_launches).  Latency bounds the small form,
// the launches and the scattered row numbers the large one (8 MB for a million rows).
#include "ops_device.hpp"

namespace hwr {
namespace {

constexpr int kSmallWaves = 4, kWaves = 16;
constexpr int kChunks = 8;                                               // one workgroup: 64 rows each
constexpr int kSmallRows = kSmallWaves * 64 * kChunks, kOneRows = kWaves * 64 * kChunks;
constexpr int kBlockChunks = 4, kBlockRows = kWaves * 64 * kBlockChunks; // several

__device__ inline int group_key(const GroupRowsArgs &a, int c) {
    if (a.table) c = static_cast<unsigned>(c) < static_cast<unsigned>(a.n_table) ? a.table[c] : -1;
    return static_cast<unsigned>(c) < static_cast<unsigned>(a.G) ? c : a.G;
}

// Exclusive prefix over i < count of value(i), handed to use(i, before).
template <int WAVES, class Value, class Use>
__device__ inline void scan_keys(int count, Value value, Use use) {
    __shared__ int part[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int base = 0;
    for (int i0 = 0; i0 < count; i0 += WAVES * 64) {
        const int i = i0 + tid, v = i < count ? value(i) : 0, upto = wave_scan(v, lane);
        if (lane == 63) part[wave] = upto;
        __syncthreads();
        int before = base;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) before += part[w];
            base += part[w];
        }
        if (i < count) use(i, before + upto - v);
        __syncthreads();
    }
}

enum class Step { kAll, kCount, kPlace, kSumAndPlace };

// total and before of every key, from the counts by block: all of its rows, and those in
// the blocks before this one.  A wave takes four keys at a time.
template <int WAVES>
__device__ inline void sum_blocks(const GroupRowsArgs &a, int keys, int *total, int *before) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i0 = wave; i0 < keys; i0 += 4 * WAVES) {
        int t[4] = {}, b[4] = {};
#pragma unroll 4
        for (int at = lane; at < a.blocks; at += 64)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int key = i0 + j * WAVES;
                const int v = key < keys ? a.hist[static_cast<int64_t>(key) * a.blocks + at] : 0;
                t[j] += v;
                b[j] += at < static_cast<int>(blockIdx.x) ? v : 0;
            }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int d = 32; d; d >>= 1) {
                t[j] += __shfl_xor(t[j], d);
                b[j] += __shfl_xor(b[j], d);
            }
            if (lane == 0 && i0 + j * WAVES < keys) {
                total[i0 + j * WAVES] = t[j];
                before[i0 + j * WAVES] = b[j];
            }
        }
    }
}

template <Step STEP, int WAVES, int kChunks>
__global__ void __launch_bounds__(WAVES * 64) k_group(GroupRowsArgs a) {
    constexpr int kWaveRows = 64 * kChunks;
    constexpr bool kSum = STEP == Step::kSumAndPlace;
    // counts by wave, then the place of the wave's next row of each key
    __shared__ int count[WAVES][kMaxPairs + 1];
    __shared__ int total[kSum ? kMaxPairs + 1 : 1], in_blocks[kSum ? kMaxPairs + 1 : 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, keys = a.G + 1;
    const int64_t r0 = (static_cast<int64_t>(blockIdx.x) * WAVES + wave) * kWaveRows + lane;
    int key[kChunks];
#pragma unroll
    for (int j = 0; j < kChunks; ++j) key[j] = r0 + j * 64 < a.n ? a.choice[r0 + j * 64] : -1;
    if constexpr (kSum) sum_blocks<WAVES>(a, keys, total, in_blocks);    // while the choices are on their way
#pragma unroll
    for (int j = 0; j < kChunks; ++j) key[j] = r0 + j * 64 < a.n ? group_key(a, key[j]) : -1;
    for (int i = lane; i < keys; i += 64) count[wave][i] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kChunks; ++j)
        if (key[j] >= 0) atomicAdd(&count[wave][key[j]], 1);
    __syncthreads();
    auto in_block = [&](int i) {
        int v = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += count[w][i];
        return v;
    };
    if constexpr (STEP == Step::kCount) {
        for (int i = tid; i < keys; i += WAVES * 64) a.hist[static_cast<int64_t>(i) * a.blocks + blockIdx.x] = in_block(i);
        return;
    }
    scan_keys<WAVES>(
        keys, [&](int i) { return STEP == Step::kAll ? in_block(i) : kSum ? total[i] : a.totals[i]; },
        [&](int i, int before) {
            if (blockIdx.x == 0 && i <= a.G) a.offsets[i] = before;
            if (STEP == Step::kPlace) before += a.hist[static_cast<int64_t>(i) * a.blocks + blockIdx.x];
            if (kSum) before += in_blocks[i];
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const int c = count[w][i];
                count[w][i] = before;
                before += c;
            }
        });
    int *next = count[wave];
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
        const int k = key[j];
        uint64_t same = __ballot(k >= 0);
        for (int bit = 0; (a.G >> bit) != 0; ++bit) {
            const uint64_t set = __ballot((k >> bit) & 1);
            same &= ((k >> bit) & 1) ? set : ~set;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1)), at = k < 0 ? 0 : next[k];
        if (k >= 0) a.order[at + rank] = static_cast<int>(r0 + j * 64);
        wave_lds();                                      // every lane has its place: the first moves it on
        if (k >= 0 && rank == 0) next[k] = at + __popcll(same);
        wave_lds();
    }
}

// hist of a key: rows in the blocks before each; totals: its rows.  A wave to a key.
__global__ void __launch_bounds__(256) k_group_scan(GroupRowsArgs a) {
    const int lane = threadIdx.x & 63, key = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (key > a.G) return;
    int *h = a.hist + static_cast<int64_t>(key) * a.blocks;
    int base = 0;
    for (int b0 = 0; b0 < a.blocks; b0 += 64 * 8) {
        int v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = b0 + j * 64 + lane < a.blocks ? h[b0 + j * 64 + lane] : 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int upto = wave_scan(v[j], lane);
            if (b0 + j * 64 + lane < a.blocks) h[b0 + j * 64 + lane] = base + upto - v[j];
            base += __builtin_amdgcn_readlane(upto, 63);
        }
    }
    if (lane == 0) a.totals[key] = base;
}

}  // namespace

int group_rows_blocks(int n) { return n > kOneRows ? static_cast<int>((static_cast<int64_t>(n) + kBlockRows - 1) / kBlockRows) : 1; }

// Whether every block of the places sums the counts of the blocks itself, rather than a
// launch between: one round of 64 keys and 256 blocks.  (us, two / three launches: 100,000
// rows 5 keys 9.8 / 12.3, 64 keys 10.8 / 12.0, 201 keys 17.6 / 13.0; 1,048,576 rows 33 keys
// 12.4 / 13.6, 64 keys 13.5 / 14.5, 201 keys 21.4 / 16.5; 3,145,728 rows 33 keys 33.9 / 26.3.)
static bool two_launches(const GroupRowsArgs &a) { return a.G < 64 && a.blocks <= 256; }

hipError_t launch_group_rows(const GroupRowsArgs &a, hipStream_t s) {
    if (a.n <= kSmallRows)
        return launch_kernel(k_group<Step::kAll, kSmallWaves, kChunks>, dim3(1), dim3(kSmallWaves * 64), 0, s, a);
    const dim3 grid(a.blocks), block(kWaves * 64);
    if (a.blocks == 1) return launch_kernel(k_group<Step::kAll, kWaves, kChunks>, grid, block, 0, s, a);
    hipError_t e = launch_kernel(k_group<Step::kCount, kWaves, kBlockChunks>, grid, block, 0, s, a);
    if (e != hipSuccess) return e;
    if (two_launches(a)) return launch_kernel(k_group<Step::kSumAndPlace, kWaves, kBlockChunks>, grid, block, 0, s, a);
    e = launch_kernel(k_group_scan, dim3((a.G + 4) / 4), dim3(256), 0, s, a);
    if (e != hipSuccess) return e;
    return launch_kernel(k_group<Step::kPlace, kWaves, kBlockChunks>, grid, block, 0, s, a);
}

}  // namespace hwr
