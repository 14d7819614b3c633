// Weight gradients of a routed batch: out[g] = P^T Q over the places of group
// g, with P and Q rows of the batch (through the row order) or low-rank
// intermediates (by place).
//
// Both factors are staged by place, 64 (bf16) or 32 (fp32) places to a stage, and
// read by columns.  Where the output has few tiles, workgroups share a tile's
// places and write fp32 partial sums that k_cols_sum adds, in order.
#include <algorithm>

#include "cols_device.hpp"

namespace hwr {
namespace {

template <class E, class PT, class QT, int PF, int QF>
__device__ inline void multiply_tile(const char *lds, int at_q, int p0, int q0, int lane, f32x4 (&acc)[PF][QF]) {
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
        typename Elem<E>::Frag fq[QF], fp[PF];
#pragma unroll
        for (int j = 0; j < QF; ++j) fq[j] = QT::frag(lds, at_q, q0 + j * 16, sub, QT::base(lane));
#pragma unroll
        for (int i = 0; i < PF; ++i) fp[i] = PT::frag(lds, 0, p0 + i * 16, sub, PT::base(lane));
#pragma unroll
        for (int i = 0; i < PF; ++i)
#pragma unroll
            for (int j = 0; j < QF; ++j) acc[i][j] = Elem<E>::mma(fq[j], fp[i], acc[i][j]);
    }
}

// Any widths, strides and alignment: operands pass through registers.
template <class E, ColsKind KIND, int BP, int BQ, int WP, int WQ>
__global__ void __launch_bounds__(WP *WQ * 64) k_cols(ColsArgs a) {
    using El = Elem<E>;
    using TT = ColsTiles<E, KIND, BP, BQ>;
    using PT = typename TT::PT;
    using QT = typename TT::QT;
    static_assert((!TT::kLowP || WP == 1) && (!TT::kLowQ || WQ == 1));
    constexpr int NT = WP * WQ * 64, PF = BP / WP / 16, QF = BQ / WQ / 16, kBk = El::kBk;
    __shared__ __attribute__((aligned(16))) char buf[PT::kBytes + QT::kBytes];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wp = wave / WQ, wq = wave % WQ;
    ColsTile t;
    if (!col_tile<KIND, BP, BQ, kBk>(a, blockIdx.x, t)) return;

    f32x4 acc[PF][QF] = {};
    constexpr int UP = PT::kChunks / NT, UQ = QT::kChunks / NT;
    static_assert(PT::kChunks % NT == 0 && QT::kChunks % NT == 0);
    auto chunk = [&](const void *src, int64_t ld, int width, int c0, bool low, int block, int place, int c) {
        if (place >= t.p1) return u32x4{0, 0, 0, 0};
        if (low)
            return *reinterpret_cast<const u32x4 *>(static_cast<const char *>(src) +
                                                    (static_cast<int64_t>(place) * a.blocks + block) * kLowBytes + c * 16);
        const int r = row_at(a.g, place);
        return load_chunk<E>(r >= 0 ? static_cast<const E *>(src) + r * ld : nullptr, c0 + c * El::kEpc, width);
    };
    u32x4 vp[UP], vq[UQ];
    auto load = [&](int p) {
#pragma unroll
        for (int i = 0; i < UP; ++i) {
            const int u = i * NT + tid, line = u / PT::kCpl, c = (u % PT::kCpl) ^ PT::swz(line);
            vp[i] = chunk(a.p, a.ldp, a.np, t.ip * BP, TT::kLowP, t.ip, p + line, c);
        }
#pragma unroll
        for (int i = 0; i < UQ; ++i) {
            const int u = i * NT + tid, line = u / QT::kCpl, c = (u % QT::kCpl) ^ QT::swz(line);
            vq[i] = chunk(a.q, a.ldq, a.nq, t.iq * BQ, TT::kLowQ, t.iq, p + line, c);
        }
    };
    if (t.p0 < t.p1) load(t.p0);
    for (int p = t.p0; p < t.p1; p += kBk) {
#pragma unroll
        for (int i = 0; i < UP; ++i) *reinterpret_cast<u32x4 *>(buf + (i * NT + tid) * 16) = vp[i];
#pragma unroll
        for (int i = 0; i < UQ; ++i) *reinterpret_cast<u32x4 *>(buf + PT::kBytes + (i * NT + tid) * 16) = vq[i];
        __syncthreads();
        if (p + kBk < t.p1) load(p + kBk);
        multiply_tile<E, PT, QT, PF, QF>(buf, PT::kBytes, wp * PF * 16, wq * QF * 16, lane, acc);
        __syncthreads();
    }
    store_tile<E, KIND, BP, BQ, WP, WQ>(a, t, acc, lane, wp, wq);
}

template <class E, ColsKind KIND, int BP, int BQ, int WP, int WQ>
__global__ void __launch_bounds__(WP *WQ * 64) k_cols_direct(ColsArgs a) {
    // an array each, so that the compiler sees that reads of one do not depend on the
    // loads in flight into the other
    constexpr int kBuf = kColsBuf<E, KIND, BP, BQ>, kMore = BP == 64 && BQ == 64 ? kBuf : 16;
    __shared__ __attribute__((aligned(16))) char buf0[kBuf], buf1[kBuf], buf2[kMore], buf3[kMore];
    cols_direct<E, KIND, BP, BQ, WP, WQ>(a, blockIdx.x, buf0, buf1, buf2, buf3);
}

// Both low-rank gradients in one launch, eight workgroups (one on each L2) of each in turn.
template <class E>
__global__ void __launch_bounds__(256) k_cols_low_pair(ColsArgs a, ColsArgs b) {
    constexpr int L = kLowBytes / sizeof(E), kBuf = kColsBuf<E, ColsKind::kLowQ, 128, L>;
    static_assert(kBuf == kColsBuf<E, ColsKind::kLowP, L, 128>);
    __shared__ __attribute__((aligned(16))) char buf0[kBuf], buf1[kBuf];
    const int block = blockIdx.x >> 4 << 3 | (blockIdx.x & 7);
    if (blockIdx.x & 8) cols_direct<E, ColsKind::kLowP, L, 128, 1, 4>(b, block, buf0, buf1, nullptr, nullptr);
    else cols_direct<E, ColsKind::kLowQ, 128, L, 4, 1>(a, block, buf0, buf1, nullptr, nullptr);
}

// out = sum of the parts
template <class E>
__device__ inline void sum_parts(const ColsArgs &a, int64_t i) {
    const int64_t count = static_cast<int64_t>(a.g.G) * a.np * a.nq;
    if (i >= count) return;
    if (i + 4 <= count) {
        f32x4 v = {};
#pragma unroll 4
        for (int s = 0; s < a.parts; ++s) v += *reinterpret_cast<const f32x4_a4 *>(a.partial + s * count + i);
        typename Elem<E>::Out4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = static_cast<E>(v[e]);
        *reinterpret_cast<typename Elem<E>::Out4 *>(static_cast<E *>(a.out) + i) = o;
    } else {
        for (int64_t j = i; j < count; ++j) {
            float v = 0.0f;
            for (int s = 0; s < a.parts; ++s) v += a.partial[s * count + j];
            static_cast<E *>(a.out)[j] = static_cast<E>(v);
        }
    }
}

// (of one gradient, or of two: grid.y)
template <class E>
__global__ void __launch_bounds__(256) k_cols_sum(ColsArgs a, ColsArgs b) {
    const int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
    const ColsArgs &c = blockIdx.y ? b : a;
    if (c.parts > 1) sum_parts<E>(c, i);
}

template <class E>
hipError_t sum(const ColsArgs &a, const ColsArgs *b, hipStream_t s) {
    auto blocks = [](const ColsArgs &c) { return c.parts > 1 ? (static_cast<int64_t>(c.g.G) * c.np * c.nq + 1023) / 1024 : 0; };
    const int64_t most = std::max(blocks(a), b ? blocks(*b) : 0);
    if (most == 0) return hipSuccess;
    return launch_kernel(k_cols_sum<E>, dim3(static_cast<uint32_t>(most), b ? 2 : 1), dim3(256), 0, s, a, b ? *b : a);
}

// Rows in whole, aligned chunks of 16 bytes.
template <class E, ColsKind KIND>
bool whole_chunks(const ColsArgs &a) {
    constexpr int kEpc = Elem<E>::kEpc;
    auto whole = [&](const void *p, int64_t ld, int width) {
        return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % kEpc == 0 && (a.padded || width % kEpc == 0);
    };
    return (KIND == ColsKind::kLowP || whole(a.p, a.ldp, a.np)) && (KIND == ColsKind::kLowQ || whole(a.q, a.ldq, a.nq));
}

template <class E, ColsKind KIND, int BP, int BQ, int WP, int WQ, bool DIRECT>
hipError_t go(const ColsArgs &a, hipStream_t s) {
    const int64_t blocks = cols_blocks(a, KIND == ColsKind::kLowP ? a.blocks : (a.np + BP - 1) / BP,
                                       KIND == ColsKind::kLowQ ? a.blocks : (a.nq + BQ - 1) / BQ);
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    const dim3 grid(static_cast<uint32_t>(blocks)), block(WP * WQ * 64);
    hipError_t e;
    if constexpr (DIRECT) e = launch_kernel(k_cols_direct<E, KIND, BP, BQ, WP, WQ>, grid, block, 0, s, a);
    else e = launch_kernel(k_cols<E, KIND, BP, BQ, WP, WQ>, grid, block, 0, s, a);
    return e != hipSuccess ? e : sum<E>(a, nullptr, s);
}

template <class E>
hipError_t low_pair(const ColsArgs &a, const ColsArgs &b, hipStream_t s) {
    const int64_t most = std::max(cols_blocks(a, (a.np + 127) / 128, a.blocks), cols_blocks(b, b.blocks, (b.nq + 127) / 128));
    if (2 * most > INT32_MAX) return hipErrorInvalidValue;
    const hipError_t e = launch_kernel(k_cols_low_pair<E>, dim3(static_cast<uint32_t>(2 * most)), dim3(256), 0, s, a, b);
    return e != hipSuccess ? e : sum<E>(a, &b, s);
}

template <class E>
hipError_t pick(ColsKind kind, const ColsPlan &p, const ColsArgs &a, hipStream_t s) {
    constexpr int L = kLowBytes / sizeof(E);
    if (kind == ColsKind::kLowP)
        return p.direct ? go<E, ColsKind::kLowP, L, 128, 1, 4, true>(a, s) : go<E, ColsKind::kLowP, L, 128, 1, 4, false>(a, s);
    if (kind == ColsKind::kLowQ)
        return p.direct ? go<E, ColsKind::kLowQ, 128, L, 4, 1, true>(a, s) : go<E, ColsKind::kLowQ, 128, L, 4, 1, false>(a, s);
    if (p.direct) {
        if constexpr (sizeof(E) == 2)
            if (p.tile == 256) return go<E, ColsKind::kDense, 256, 256, 2, 4, true>(a, s);
        if (p.tile == 128) return go<E, ColsKind::kDense, 128, 128, 2, 2, true>(a, s);
        return go<E, ColsKind::kDense, 64, 64, 2, 2, true>(a, s);
    }
    if (p.tile == 128) return go<E, ColsKind::kDense, 128, 128, 2, 2, false>(a, s);
    return go<E, ColsKind::kDense, 64, 64, 2, 2, false>(a, s);
}

}  // namespace

// The largest tile with which workgroups fill the device, sharing tiles' places if need be:
// each part has at least 8 stages of an average group (4 with the smallest tile; its
// partial sums are written and read once, 1.6 ps an element).  fp32: not 128 for one to three tiles
// a compute unit, whose rounds come out uneven (both gradients, us, 64 / 128: 3,408 x 832 x 320 in 22 groups
// 68 / 80, 2,400 x 1024 x 1536 in 4 175 / 190, 1,455 x 284 x 1160 in 9 43 / 56; one group of 4,096 x 1024 x
// 1024 185 / 162 in parts).
ColsPlan cols_plan(bool bf16, ColsKind kind, const ColsArgs &a, int cus) {
    ColsPlan p{false, 64, 1};
    if (bf16)
        p.direct = kind == ColsKind::kLowP   ? whole_chunks<__bf16, ColsKind::kLowP>(a)
                   : kind == ColsKind::kLowQ ? whole_chunks<__bf16, ColsKind::kLowQ>(a)
                                             : whole_chunks<__bf16, ColsKind::kDense>(a);
    else
        p.direct = kind == ColsKind::kLowP   ? whole_chunks<float, ColsKind::kLowP>(a)
                   : kind == ColsKind::kLowQ ? whole_chunks<float, ColsKind::kLowQ>(a)
                                             : whole_chunks<float, ColsKind::kDense>(a);
    const int64_t stages = a.g.n / (static_cast<int64_t>(a.g.G) * (bf16 ? 64 : 32));
    // parts that bring `items` workgroups to `enough`
    auto parts = [](int64_t items, int64_t enough) {
        int64_t n = 1;
        while (items * n < enough) n *= 2;
        return n;
    };
    auto tiles = [&](int64_t t) { return a.g.G * ((a.np + t - 1) / t) * ((a.nq + t - 1) / t); };
    if (kind == ColsKind::kDense) {
        for (int t = p.direct && bf16 ? 256 : 128; t >= 64; t /= 2) {
            const int64_t n = parts(tiles(t), cus);
            if (!bf16 && t > 64 && tiles(t) >= cus && tiles(t) < 3 * cus) continue;
            if (t > 64 && (a.np < t || a.nq < t || n > std::max<int64_t>(1, stages / 8))) continue;
            p.tile = t;
            p.parts = static_cast<int>(std::min<int64_t>(n, std::max<int64_t>(1, stages / 4)));
            break;
        }
        return p;
    }
    const int64_t wide = kind == ColsKind::kLowP ? a.nq : a.np;
    const int64_t n = parts(a.blocks * ((wide + 127) / 128) * a.g.G, 3 * cus);
    p.parts = static_cast<int>(std::min<int64_t>(n, std::max<int64_t>(1, stages / 4)));
    return p;
}

hipError_t launch_cols(bool bf16, ColsKind kind, const ColsArgs &a, int cus, hipStream_t s) {
    const ColsPlan p = cols_plan(bf16, kind, a, cus);
    return bf16 ? pick<__bf16>(kind, p, a, s) : pick<float>(kind, p, a, s);
}

hipError_t launch_cols_sum(bool bf16, const ColsArgs &a, hipStream_t s) {
    return bf16 ? sum<__bf16>(a, nullptr, s) : sum<float>(a, nullptr, s);
}

hipError_t launch_cols_low_pair(bool bf16, const ColsArgs &q, const ColsArgs &p, hipStream_t s) {
    return bf16 ? low_pair<__bf16>(q, p, s) : low_pair<float>(q, p, s);
}

}  // namespace hwr
