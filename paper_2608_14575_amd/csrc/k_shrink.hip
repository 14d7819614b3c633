// Low-rank intermediates: low[place] = scale[g] x[row] w_g, with w_g [k][rank]
// or [rank][k].
//
// The rows are read once, straight into matrix operands; the narrow weights come
// from the L2s.  A workgroup takes a tile of places of one group; its waves take every
// kWaves-th step of the contraction and add up through LDS.  A wave waits for
// no other until then, and keeps the loads of several steps in flight: that, and not
// the L2s, bounded a form with one step ahead (12,288 rows of 4096 bf16: 75 us).
#include "ops_device.hpp"

namespace hwr {
namespace {

constexpr int kWaves = 8;

// (stored and read as different types)
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), may_alias));

// How the weights come into operand form.  kDirect: [rank][k], 16 bytes of a lane are
// its operand.  Else [k][rank]: a step's rows are one piece of memory, which goes
// through a part of LDS that is the wave's own and is read by columns: kTurned with
// the transposing read (bf16, ranks that are multiples of 4), kPicked by single elements.
enum class From { kDirect, kTurned, kPicked };

template <class E, From FROM, int NF, int RB>
struct Sizes {
    static constexpr int kStep = 4 * Elem<E>::kEpc;
    // a step's weights for each wave, or half of the waves' sums
    static constexpr int kOwn = FROM != From::kDirect ? kStep * 16 * NF * (int)sizeof(E) : 0, kSums = RB * NF * 64 * 16;
    static constexpr int kLds = kWaves * kOwn > kWaves / 2 * kSums ? kWaves * kOwn : kWaves / 2 * kSums;
    static constexpr int kMinWaves = NF == 8 || (FROM == From::kPicked && NF * RB == 8) ? 2 : 4;   // a SIMD
};

// NF column fragments, RB row fragments; tile t of the batch.
template <class E, From FROM, int NF, int RB>
__device__ inline void shrink_tile(const ShrinkArgs &a, int t, char *lds) {
    using El = Elem<E>;
    using Sz = Sizes<E, FROM, NF, RB>;
    constexpr int V = El::kEpc, BM = 16 * RB, kStep = Sz::kStep, kOwn = Sz::kOwn;
    constexpr int kAcc = RB * NF, kDeep = NF <= 2 ? 4 : 2;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m = lane & 15, q = lane >> 4;
    if (t >= count_tiles(a.g, BM, false, lane)) return;
    const RowTile rt = find_tile(a.g, t, BM, false, lane);
    const E *w = static_cast<const E *>(a.w) + static_cast<int64_t>(rt.g) * a.k * a.rank;

    // (a place without a row takes row 0; its intermediate is never used)
    const E *x[RB];
    bool in_tile[RB];
#pragma unroll
    for (int i = 0; i < RB; ++i) {
        const int p = rt.p0 + i * 16 + m, r = p < rt.p1 ? row_at(a.g, p) : -1;
        in_tile[i] = p < rt.p1;
        x[i] = static_cast<const E *>(a.x) + (r < 0 ? 0 : r) * a.ldx + q * V;
    }
    f32x4 acc[RB][NF] = {};
    u32x4 nw[kDeep][NF], nx[kDeep][RB];
    const int steps = (a.k + kStep - 1) / kStep;
    auto load = [&](u32x4 (&lw)[NF], u32x4 (&lx)[RB], int step) {
        const bool whole = (step + 1) * kStep <= a.k;
#pragma unroll
        for (int i = 0; i < RB; ++i) {
            if (whole) lx[i] = *reinterpret_cast<const typename El::Vec *>(x[i] + step * kStep);
            else lx[i] = load_chunk<E>(x[i], step * kStep, a.k - q * V);
        }
        const int e = step * kStep + q * V;
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            if constexpr (FROM == From::kDirect) {
                const E *line = w + static_cast<int64_t>(min(i * 16 + m, a.rank - 1)) * a.k;   // past the rank: not used
                if (whole) lw[i] = *reinterpret_cast<const typename El::Vec *>(line + e);
                else lw[i] = load_chunk<E>(line, e, a.k);
            } else {
                const int at = step * kStep * a.rank + (i * 64 + lane) * V, all = a.k * a.rank;
                lw[i] = u32x4{0, 0, 0, 0};
                if ((i * 64 + lane) * V < kStep * a.rank) {
                    if (at + V <= all) lw[i] = *reinterpret_cast<const typename El::Vec *>(w + at);
                    else lw[i] = load_chunk<E>(w, at, all);
                }
            }
        }
    };
    auto consume = [&](const u32x4 (&lw)[NF], const u32x4 (&lx)[RB]) {
        union Chunk { u32x4 v; typename El::Frag f; E e[V]; } u;
        typename El::Frag fw[NF];
        char *own = lds + wave * kOwn;
        if constexpr (FROM != From::kDirect) {
#pragma unroll
            for (int i = 0; i < NF; ++i)
                if ((i * 64 + lane) * V < kStep * a.rank) *reinterpret_cast<u32x4_any *>(own + (i * 64 + lane) * 16) = lw[i];
            wave_lds();
        }
#pragma unroll
        for (int j = 0; j < NF; ++j) {
            if constexpr (FROM == From::kDirect) {
                u.v = lw[j];
            } else {
                // (columns past the rank take what follows in LDS, and are not used)
                const int line = a.rank * (int)sizeof(E);
                if constexpr (FROM == From::kTurned) {
                    typedef __attribute__((address_space(3))) i16x4 lds_v;
                    union { i16x4 h[2]; u32x4 v; } r;
                    const int o = (q * 8 + (m >> 2)) * line + (j * 16 + (m & 3) * 4) * 2;
                    r.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v *)(own + min(o, kOwn - 8)));
                    r.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v *)(own + min(o + 4 * line, kOwn - 8)));
                    u.v = r.v;
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        u.e[i] = *reinterpret_cast<const E *>(own + min((q * V + i) * line + (j * 16 + m) * (int)sizeof(E),
                                                                        kOwn - (int)sizeof(E)));
                }
            }
            fw[j] = u.f;
        }
        if constexpr (FROM != From::kDirect) wave_lds();       // before the next step overwrites it
#pragma unroll
        for (int i = 0; i < RB; ++i) {
            u.v = lx[i];
#pragma unroll
            for (int j = 0; j < NF; ++j) acc[i][j] = El::mma(fw[j], u.f, acc[i][j]);
        }
    };
    // kDeep steps in flight, in turn (a step past the last is zeros on both sides)
#pragma unroll
    for (int d = 0; d < kDeep; ++d) load(nw[d], nx[d], wave + d * kWaves);
    for (int step = wave; step < steps; step += kDeep * kWaves) {
#pragma unroll
        for (int d = 0; d < kDeep; ++d) {
            consume(nw[d], nx[d]);
            load(nw[d], nx[d], step + (kDeep + d) * kWaves);
        }
    }

    f32x4 *part = reinterpret_cast<f32x4 *>(lds);
    __syncthreads();
#pragma unroll
    for (int half = kWaves / 2; half; half /= 2) {
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int i = 0; i < kAcc; ++i) part[((wave - half) * kAcc + i) * 64 + lane] = acc[i / NF][i % NF];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int i = 0; i < kAcc; ++i) acc[i / NF][i % NF] += part[(wave * kAcc + i) * 64 + lane];
        __syncthreads();
    }
    if (wave != 0) return;

    // lane: place m of block i, columns 16 j + 4 q + e.  Zeros past the rank (not 0 x infinity).
    const float s = a.scale ? a.scale[rt.g] : 1.0f;
    const int blocks = (a.rank + kRankBlock - 1) / kRankBlock;
#pragma unroll
    for (int i = 0; i < RB; ++i) {
        if (!in_tile[i]) continue;
        char *at = static_cast<char *>(a.low) + static_cast<int64_t>(rt.p0 + i * 16 + m) * blocks * kLowBytes;
        auto put = [&](int c, f32x4 v) {
            if (c >= blocks * kRankBlock) return;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = c + e < a.rank ? v[e] * s : 0.0f;
            store_low<E>(at + c / kRankBlock * kLowBytes, c % kRankBlock, v);
        };
#pragma unroll
        for (int j = 0; j < NF; ++j) put(j * 16 + 4 * q, acc[i][j]);
        if constexpr (NF == 1) put(16 + 4 * q, f32x4{});       // the block's other half
    }
}

template <class E, From FROM, int NF, int RB>
__global__ void __launch_bounds__(kWaves * 64, (Sizes<E, FROM, NF, RB>::kMinWaves)) k_shrink(ShrinkArgs a) {
    __shared__ __attribute__((aligned(16))) char lds[Sizes<E, FROM, NF, RB>::kLds];
    shrink_tile<E, FROM, NF, RB>(a, block_id<kWaves * 64>(), lds);
}

// Two in one launch: the first's tiles take the even workgroups.
template <class E, From FROM, int NF, int RB>
__global__ void __launch_bounds__(kWaves * 64, (Sizes<E, FROM, NF, RB>::kMinWaves)) k_shrink_pair(ShrinkArgs a, ShrinkArgs b) {
    constexpr int kA = Sizes<E, From::kDirect, NF, RB>::kLds, kB = Sizes<E, FROM, NF, RB>::kLds;
    __shared__ __attribute__((aligned(16))) char lds[kA > kB ? kA : kB];
    const int id = block_id<kWaves * 64>();
    if (id & 1) shrink_tile<E, FROM, NF, RB>(b, id >> 1, lds);
    else shrink_tile<E, From::kDirect, NF, RB>(a, id >> 1, lds);
}

// One (pair null), or with it [rank][k] weights beside `pair`'s [k][rank].
template <class E, From FROM, int NF, int RB>
hipError_t go(const ShrinkArgs &a, const ShrinkArgs *pair, hipStream_t s) {
    const int64_t tiles = a.g.n / (16 * RB) + (a.g.n < a.g.G ? a.g.n : a.g.G);
    constexpr int NT = kWaves * 64;
    if constexpr (FROM != From::kDirect)
        if (pair) return launch_kernel(k_shrink_pair<E, FROM, NF, RB>, wide_grid(2 * tiles, NT), dim3(NT), 0, s, a, *pair);
    return launch_kernel(k_shrink<E, FROM, NF, RB>, wide_grid(tiles, NT), dim3(NT), 0, s, a);
}

template <class E, From FROM, int NF>
hipError_t rows(const ShrinkArgs &a, const ShrinkArgs *pair, int cus, hipStream_t s) {
    // two blocks of rows share the weights' loads where the device stays full
    if constexpr (NF <= 4)
        if (a.g.n >= 32 * cus) return go<E, FROM, NF, 2>(a, pair, s);
    return go<E, FROM, NF, 1>(a, pair, s);
}

template <class E, From FROM>
hipError_t ranks(const ShrinkArgs &a, const ShrinkArgs *pair, int cus, hipStream_t s) {
    if (a.rank <= 16) return rows<E, FROM, 1>(a, pair, cus, s);
    if (a.rank <= 32) return rows<E, FROM, 2>(a, pair, cus, s);
    if (a.rank <= 64) return rows<E, FROM, 4>(a, pair, cus, s);
    return rows<E, FROM, 8>(a, pair, cus, s);
}

template <class E>
hipError_t pick(bool ks, const ShrinkArgs &a, const ShrinkArgs *pair, int cus, hipStream_t s) {
    if (!ks && !pair) return ranks<E, From::kDirect>(a, nullptr, cus, s);
    if constexpr (sizeof(E) == 2)
        if (a.rank % 4 == 0) return ranks<E, From::kTurned>(a, pair, cus, s);
    return ranks<E, From::kPicked>(a, pair, cus, s);
}

}  // namespace

hipError_t launch_shrink(bool bf16, bool ks, const ShrinkArgs &a, int cus, hipStream_t s) {
    return bf16 ? pick<__bf16>(ks, a, nullptr, cus, s) : pick<float>(ks, a, nullptr, cus, s);
}

hipError_t launch_shrink_pair(bool bf16, const ShrinkArgs &direct, const ShrinkArgs &ks, int cus, hipStream_t s) {
    return bf16 ? pick<__bf16>(false, direct, &ks, cus, s) : pick<float>(false, direct, &ks, cus, s);
}

}  // namespace hwr
