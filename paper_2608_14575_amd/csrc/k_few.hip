// Products of few rows: the weights are streamed once, straight from memory
// into matrix operands, and the contraction is split over waves and workgroups.
//
// A lane (m = l % 16, q = l / 16) loads 16 bytes of V columns from each of V
// weight rows, V = 8 (bf16) or 4 (fp32): rows q V .. q V + V - 1 of a step of 4 V,
// columns m V .. m V + V - 1.  Its V x V block transposed is the lane's share of V
// A-operand fragments: fragment j holds the columns m V + j.  The steps need no LDS and
// no barrier: a wave has the next step's loads in flight while it multiplies one.
// The waves of a workgroup take every kWaves-th step and add up through LDS at the end;
// workgroups that share a tile write fp32 partial sums that k_join adds, in order.
//
// A tile is 16 rows: tiles of the same weights run side by side on one L2 (48
// rows, 4096 x 4096 bf16: 14.8 us; with tiles of 32 rows 17.0, of 64 rows 20.7, for
// want of registers to load ahead: the loads of cut columns and of a last cut step stand
// in the same loop, which takes all 128 registers in bf16 and spills 14 to 16 of them, read
// back on those paths alone).
#include "ops_device.hpp"

namespace hwr {
namespace {

constexpr int kWaves = 8;

// low[s][place][r]: partial sums of x[row] a_g over the s-th part of the contraction
template <class E>
__device__ void few_shrink(const FewArgs &a, int item, float *lds) {
    constexpr int V = Elem<E>::kEpc, NT = kWaves * 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int p = item % a.g.n, s = item / a.g.n;
    const int g = group_of(a.g, p, lane);
    if (g == a.g.G) return;
    const int row = row_at(a.g, p);
    const E *x = static_cast<const E *>(a.x) + (row < 0 ? 0 : row) * a.ldx;
    const E *w = static_cast<const E *>(a.a) + static_cast<int64_t>(g) * a.k * a.rank;
    int lanes = 1;                               // lanes of a weight row, V columns each
    while (lanes * V < a.rank) lanes *= 2;
    const int c = tid % lanes * V;
    const int k0 = static_cast<int>(static_cast<int64_t>(a.k) * s / a.low_parts),
              k1 = static_cast<int>(static_cast<int64_t>(a.k) * (s + 1) / a.low_parts);
    float acc[V] = {};
#pragma unroll 4
    for (int k = k0 + tid / lanes; k < k1; k += NT / lanes) {
        union { u32x4 v; E e[V]; } u;
        u.v = load_chunk<E>(w + static_cast<int64_t>(k) * a.rank, c, a.rank);
        const float xv = row < 0 ? 0.0f : static_cast<float>(x[k]);
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = fmaf(xv, static_cast<float>(u.e[i]), acc[i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        for (int d = 32; d >= lanes; d >>= 1) acc[i] += __shfl_xor(acc[i], d);
    if (lane < lanes)
#pragma unroll
        for (int i = 0; i < V; ++i) lds[(wave * lanes + lane) * V + i] = acc[i];
    __syncthreads();
    if (tid < a.rank) {
        float v = 0.0f;
        for (int w2 = 0; w2 < kWaves; ++w2) v += lds[w2 * lanes * V + tid];
        a.low[(static_cast<int64_t>(s) * a.g.n + p) * a.rank + tid] = v;
    }
}

template <class E, bool ADAPTER>
__global__ void __launch_bounds__(kWaves * 64, 4) k_few(FewArgs a) {   // two workgroups on a compute unit
    using El = Elem<E>;
    constexpr int V = El::kEpc, BM = kFewTile, BN = 16 * V, kStep = 4 * V;
    __shared__ f32x4 part[kWaves / 2 * V * 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m = lane & 15, q = lane >> 4;

    int item = blockIdx.x;
    if (ADAPTER) {
        if (item < a.g.n * a.low_parts) return few_shrink<E>(a, item, reinterpret_cast<float *>(part));
        item -= a.g.n * a.low_parts;
    }
    const int ct = (a.m + BN - 1) / BN;
    const int s = item % a.parts, tc = item / a.parts, t = tc / ct;
    // the last tile of columns ends with the row: it shares columns with the one before
    // (both give them the same bits), and no chunk is cut
    const int c0 = a.m < BN ? 0 : min(tc % ct * BN, a.m - BN);
    RowTile rt;
    if (ADAPTER) {
        rt = {0, t * BM, min(t * BM + BM, a.g.n)};
    } else {
        if (t >= count_tiles(a.g, BM, true, lane)) return;
        rt = find_tile(a.g, t, BM, true, lane);
    }
    const int k = !ADAPTER && rt.g == a.g.G ? 0 : a.k;
    const E *w = static_cast<const E *>(a.w) + (ADAPTER || k == 0 ? 0 : rt.g) * a.w_stride;

    // the wave's steps: first, first + stride, ... < steps
    const int steps = (k + kStep - 1) / kStep, stride = a.parts * kWaves;
    f32x4 acc[V] = {};
    u32x4 nw[V], nx;
    // whole steps of whole columns: one lane offset, the rest of the address is uniform
    const uint32_t lane_at = static_cast<uint32_t>((q * V * a.m + c0 + m * V) * sizeof(E));
    const bool columns = c0 + BN <= a.m;
    auto load_weights = [&](int step) {
        if (columns && (step + 1) * kStep <= k) {
            const char *base = reinterpret_cast<const char *>(w + static_cast<int64_t>(step) * kStep * a.m);
#pragma unroll
            for (int i = 0; i < V; ++i)
                nw[i] = *reinterpret_cast<const typename El::Vec *>(base + static_cast<int64_t>(i) * a.m * sizeof(E) + lane_at);
            return;
        }
        const int e = step * kStep + q * V;
#pragma unroll
        for (int i = 0; i < V; ++i)
            nw[i] = load_chunk<E>(e + i < k ? w + static_cast<int64_t>(e + i) * a.m : nullptr, c0 + m * V, a.m);
    };
    int step = s * kWaves + wave;
    if (step < steps) load_weights(step);        // on their way while the rows are looked up
    const int place = rt.p0 + m, row = place < rt.p1 ? row_at(a.g, place) : -1;
    // (a place without a row computes one that it does not store)
    const E *x = static_cast<const E *>(a.x) + (row < 0 ? 0 : row) * a.ldx + q * V;
    auto load_row = [&](int step) {
        if ((step + 1) * kStep <= k) nx = *reinterpret_cast<const typename El::Vec *>(x + step * kStep);
        else nx = load_chunk<E>(x, step * kStep, k - q * V);
    };
    if (step < steps) load_row(step);
    for (; step < steps; step += stride) {
        typename El::Frag fw[V];
        union { u32x4 v; typename El::Frag f; } fx;
        fx.v = nx;
#pragma unroll
        for (int j = 0; j < V; ++j) fw[j] = column(nw, j);
        if (step + stride < steps) {
            load_weights(step + stride);
            load_row(step + stride);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = El::mma(fw[j], fx.f, acc[j]);
    }

    // sum over the waves, halving; wave 0 ends with the total
#pragma unroll
    for (int half = kWaves / 2; half; half /= 2) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int j = 0; j < V; ++j) part[((wave - half) * V + j) * 64 + lane] = acc[j];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] += part[(wave * V + j) * 64 + lane];
        __syncthreads();
    }
    if (wave != 0 || place >= rt.p1) return;

    // lane: the place, columns (4 q + e) V + j
    if (ADAPTER || a.parts > 1) {
        float *out = a.partial + (static_cast<int64_t>(s) * a.g.n + place) * a.m_pad;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int j = 0; j < V; j += 4) {
                const int c = c0 + (4 * q + e) * V + j;
                if (c < a.m_pad)
                    *reinterpret_cast<f32x4_a4 *>(out + c) = f32x4{acc[j][e], acc[j + 1][e], acc[j + 2][e], acc[j + 3][e]};
            }
    } else if (row >= 0) {
        E *y = static_cast<E *>(a.y) + row * a.ldy;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = c0 + (4 * q + e) * V;
            union { u32x4 v; E o[V]; } u;
#pragma unroll
            for (int j = 0; j < V; ++j) u.o[j] = static_cast<E>(acc[j][e]);
            if (c + V <= a.m) {
                *reinterpret_cast<typename El::Vec *>(y + c) = u.v;
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (c + j < a.m) y[c + j] = u.o[j];
            }
        }
    }
}

// y[row] = sum of the parts, plus scale[g] low[place] b_g: a thread per four columns of a place
constexpr int kJoinThreads = 128;
template <class E, bool ADAPTER>
__global__ void __launch_bounds__(kJoinThreads) k_join(FewArgs a) {
    __shared__ float low[128];
    const int tid = threadIdx.x, lane = tid & 63;
    const int ct = (a.m_pad / 4 + kJoinThreads - 1) / kJoinThreads;
    const int p = blockIdx.x / ct, c = (blockIdx.x % ct * kJoinThreads + tid) * 4;
    // everything that the place alone says first: the row, its group and that group's
    // weights are looked up while it is on its way
    f32x4 v = {};
    if (c < a.m)
#pragma unroll 4
        for (int s = 0; s < a.parts; ++s)
            v += *reinterpret_cast<const f32x4 *>(a.partial + (static_cast<int64_t>(s) * a.g.n + p) * a.m_pad + c);
    const int row = row_at(a.g, p);
    int g = a.g.G;
    if (ADAPTER) {
        float t = 0.0f;
        g = group_of(a.g, p, lane);
        if (g < a.g.G && tid < a.rank) {
#pragma unroll 4
            for (int s = 0; s < a.low_parts; ++s) t += a.low[(static_cast<int64_t>(s) * a.g.n + p) * a.rank + tid];
            low[tid] = a.scale ? a.scale[g] * t : t;
        }
        __syncthreads();
    }
    if (row < 0 || c >= a.m) return;
    if (ADAPTER && g < a.g.G) {
        // (the row's last columns, where they are cut: the four that end with the row)
        const int first = a.m < 4 ? c : min(c, a.m - 4);
        const E *b = static_cast<const E *>(a.b) + static_cast<int64_t>(g) * a.rank * a.m + first;
        f32x4 add = {};
        if (a.m >= 4) {
            struct __attribute__((packed, aligned(sizeof(E)))) Four { E e[4]; };
#pragma unroll 16
            for (int r = 0; r < a.rank; ++r) {
                const Four f = *reinterpret_cast<const Four *>(b + static_cast<int64_t>(r) * a.m);
#pragma unroll
                for (int e = 0; e < 4; ++e) add[e] = fmaf(low[r], static_cast<float>(f.e[e]), add[e]);
            }
        } else {
            for (int r = 0; r < a.rank; ++r)
                for (int e = 0; e < 4; ++e)
                    if (c + e < a.m) add[e] = fmaf(low[r], static_cast<float>(b[static_cast<int64_t>(r) * a.m + e]), add[e]);
        }
        for (int skip = first; skip < c; ++skip) add = f32x4{add[1], add[2], add[3], 0.0f};
        v += add;
    }
    store_four<E>(static_cast<E *>(a.y) + row * a.ldy, c, a.m, v);
}

template <class E, bool ADAPTER>
hipError_t join(const FewArgs &a, hipStream_t s) {
    const int64_t blocks = static_cast<int64_t>((a.m_pad / 4 + kJoinThreads - 1) / kJoinThreads) * a.g.n;
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    return launch_kernel(k_join<E, ADAPTER>, dim3(static_cast<uint32_t>(blocks)), dim3(kJoinThreads), 0, s, a);
}

template <class E, bool ADAPTER>
hipError_t go(const FewArgs &a, hipStream_t s) {
    const int ct = (a.m + 16 * Elem<E>::kEpc - 1) / (16 * Elem<E>::kEpc);
    const int64_t items = static_cast<int64_t>(few_tiles(a.g.n, a.g.G, ADAPTER)) * ct * a.parts +
                          (ADAPTER ? static_cast<int64_t>(a.g.n) * a.low_parts : 0);
    if (items > INT32_MAX) return hipErrorInvalidValue;
    const dim3 grid(static_cast<uint32_t>(items)), block(kWaves * 64);
    const hipError_t e = launch_kernel(k_few<E, ADAPTER>, grid, block, 0, s, a);
    if (e != hipSuccess || (!ADAPTER && a.parts == 1)) return e;
    return join<E, ADAPTER>(a, s);
}

}  // namespace

// Up to where 16-row tiles that read the weights once each beat larger tiles (which
// take a launch or two more with an adapter).  us, few / larger: adapter bf16 1024 x 1024
// 192 rows 17.0 / 18.2; 2048 x 2048 130 rows 19.4 / 23.0, 192 rows 20.8 / 22.8, 256 rows 28.1 / 27.7;
// 2752 x 3712 80 rows 24.9 / 27.2, 130 rows 45.4 / 30.5; 4096 x 4096 96 rows 27.8 / 34.6, 130 rows
// 41.8 / 36.8; fp32 2048 x 2048 256 rows 37 / 44; grouped (2 groups) bf16 4096 x 4096 33 rows 18.7 / 19.5,
// 48 rows 18.6 / 19.5, 64 rows 19.0 to 26.7 / 19.9, 1024 x 2048 48 rows 9.7 to 10.3 / 8.6, 64 rows 10.2 / 8.6 (beside
// 8 to 10 of the call's host time): three tiles; fp32 2048 x 2048 256 rows 38 / 44, 384 rows 48 / 44.
// And where groups have at most 16 rows on average, for a larger tile's other rows are then
// empty: 32 groups evenly, bf16 1024 x 2048 128 rows 25.4 / 30.8, 512 rows 26.3 / 30.8, 2048 x 2048 47.5 / 55.2,
// fp32 1024 x 1024 512 rows 26.2 / 41.3; 1,024 groups 512 x 512 16,384 rows bf16 200 / 216, fp32 326 / 610; 8 groups bf16
// 1024 x 2048 96 rows 13.0 / 9.5, 128 rows 9.3 / 9.5.  The rule does not see how rows lie: all in one
// group of 32, 512 rows 12.8 / 30.7; of 1,024, 16,384 rows 112 / 47, fp32 203 / 105.
bool few_rows(int n, int G, int k, int m, bool adapter, bool bf16) {
    const int most = !bf16 ? 256 : !adapter ? 48 : static_cast<int64_t>(k) * m <= 1 << 22 ? 192 : 96;
    return n <= most || (!adapter && n <= kFewTile * G);
}

int few_tiles(int n, int G, bool adapter) {
    return adapter ? (n + kFewTile - 1) / kFewTile : n / kFewTile + (n < G + 1 ? n : G + 1);
}

// Workgroups that share a tile's contraction: enough to occupy the compute units (half of
// them beside the shrink's workgroups), while every wave has a step of its own (4096 x 4096 bf16: one row 21.4 /
// 13.6 / 10.7 / 10.6 us in 1 / 2 / 4 / 8 parts, 48 rows 14.8 / 18.5 / 22.1 in 2 / 4 / 8).
int few_parts(int n, int G, int k, int m, bool bf16, bool adapter, int cus) {
    const int v = bf16 ? 8 : 4, steps = (k + 4 * v - 1) / (4 * v);
    const int64_t tiles = static_cast<int64_t>(few_tiles(n, G, adapter)) * ((m + 16 * v - 1) / (16 * v));
    int parts = 1;
    const int enough = adapter ? cus / 2 : cus;
    while (tiles * parts < enough && parts * 2 * kWaves <= steps) parts *= 2;
    return parts;
}

hipError_t launch_few(bool bf16, bool adapter, const FewArgs &a, hipStream_t s) {
    if (bf16) return adapter ? go<__bf16, true>(a, s) : go<__bf16, false>(a, s);
    return adapter ? go<float, true>(a, s) : go<float, false>(a, s);
}

hipError_t launch_join(bool bf16, const FewArgs &a, hipStream_t s) {
    return bf16 ? join<__bf16, false>(a, s) : join<float, false>(a, s);
}

}  // namespace hwr
