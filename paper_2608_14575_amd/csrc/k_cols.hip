// Weight gradients of a routed batch: out[g] = P^T Q over the places of group
// g, with P and Q rows of the batch (through the row order) or low-rank
// intermediates (by place).
#include "ops_device.hpp"

namespace hwr {
namespace {

template <class E, ColsKind KIND, int BP, int BQ, int WP, int WQ>
__global__ void __launch_bounds__(WP *WQ * 64) k_cols(ColsArgs a) {
    using El = Elem<E>;
    constexpr int NT = WP * WQ * 64, PF = BP / WP / 16, QF = BQ / WQ / 16, kBk = El::kBk;
    using PT = Tile<E, true, BP>;
    using QT = Tile<E, true, BQ>;
    // a rank block as a tile: 32 columns, in bf16 hi then lo
    constexpr int kLowCols = kLowBytes / sizeof(E);
    static_assert(KIND != ColsKind::kLowP || (BP == kLowCols && WP == 1));
    static_assert(KIND != ColsKind::kLowQ || (BQ == kLowCols && WQ == 1));
    __shared__ __attribute__((aligned(16))) char sp[PT::kBytes], sq[QT::kBytes];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wp = wave / WQ, wq = wave % WQ;
    const int g = blockIdx.y;
    const int tp = KIND == ColsKind::kLowP ? a.blocks : (a.np + BP - 1) / BP;
    const int ip = blockIdx.x % tp, iq = blockIdx.x / tp;
    const int pc = ip * BP, qc = iq * BQ;
    const int p0 = place_of(a.g, g), p1 = place_of(a.g, g + 1);

    f32x4 acc[PF][QF] = {};
    constexpr int UP = PT::kChunks / NT, UQ = QT::kChunks / NT;
    static_assert(PT::kChunks % NT == 0 && QT::kChunks % NT == 0);
    auto chunk = [&](const void *src, int64_t ld, int width, int c0, bool low, int block, int place, int c) {
        if (place >= p1) return u32x4{0, 0, 0, 0};
        if (low)
            return *reinterpret_cast<const u32x4 *>(static_cast<const char *>(src) +
                                                    (static_cast<int64_t>(place) * a.blocks + block) * kLowBytes + c * 16);
        const int r = row_at(a.g, place);
        return load_chunk<E>(r >= 0 ? static_cast<const E *>(src) + r * ld : nullptr, c0 + c * El::kEpc, width);
    };
    for (int p = p0; p < p1; p += kBk) {
        u32x4 vp[UP], vq[UQ];
#pragma unroll
        for (int i = 0; i < UP; ++i) {
            const int u = i * NT + tid, line = u / PT::kCpl, c = (u % PT::kCpl) ^ PT::swz(line);
            vp[i] = chunk(a.p, a.ldp, a.np, pc, KIND == ColsKind::kLowP, ip, p + line, c);
        }
#pragma unroll
        for (int i = 0; i < UQ; ++i) {
            const int u = i * NT + tid, line = u / QT::kCpl, c = (u % QT::kCpl) ^ QT::swz(line);
            vq[i] = chunk(a.q, a.ldq, a.nq, qc, KIND == ColsKind::kLowQ, iq, p + line, c);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < UP; ++i) *reinterpret_cast<u32x4 *>(sp + (i * NT + tid) * 16) = vp[i];
#pragma unroll
        for (int i = 0; i < UQ; ++i) *reinterpret_cast<u32x4 *>(sq + (i * NT + tid) * 16) = vq[i];
        __syncthreads();
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
            typename El::Frag fq[QF], fp[PF];
#pragma unroll
            for (int j = 0; j < QF; ++j) fq[j] = QT::frag(sq, 0, (wq * QF + j) * 16, sub, lane);
#pragma unroll
            for (int i = 0; i < PF; ++i) fp[i] = PT::frag(sp, 0, (wp * PF + i) * 16, sub, lane);
#pragma unroll
            for (int i = 0; i < PF; ++i)
#pragma unroll
                for (int j = 0; j < QF; ++j) acc[i][j] = El::mma(fq[j], fp[i], acc[i][j]);
        }
    }

    // lane: P column l % 16 of fragment i, four Q columns of fragment j
    E *out = static_cast<E *>(a.out) + static_cast<int64_t>(g) * a.np * a.nq;
    constexpr bool kPair = sizeof(E) == 2;    // low-rank sides hold hi and lo columns
    constexpr int PN = KIND == ColsKind::kLowP ? 2 : PF, QN = KIND == ColsKind::kLowQ ? 2 : QF;
    const int p_first = KIND == ColsKind::kLowP ? ip * kRankBlock : pc + wp * PF * 16;
    const int q_first = KIND == ColsKind::kLowQ ? iq * kRankBlock : qc + wq * QF * 16;
    const bool vec = (a.nq & 3) == 0 && (reinterpret_cast<uintptr_t>(a.out) & (4 * sizeof(E) - 1)) == 0;
#pragma unroll
    for (int i = 0; i < PN; ++i) {
        const int pr = p_first + i * 16 + (lane & 15);
        if (pr >= a.np) continue;
#pragma unroll
        for (int j = 0; j < QN; ++j) {
            f32x4 v = acc[i][j];
            if constexpr (KIND != ColsKind::kDense && kPair) {
                // hi + lo; where an infinite factor made hi infinite, lo could make it NaN
                const f32x4 lo = KIND == ColsKind::kLowP ? acc[(i + 2) % PF][j] : acc[i][(j + 2) % QF];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = __builtin_isfinite(v[e]) ? v[e] + lo[e] : v[e];
            }
            const int c = q_first + j * 16 + (lane >> 4) * 4;
            E *line = out + static_cast<int64_t>(pr) * a.nq;
            typename El::Out4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = static_cast<E>(v[e]);
            if (vec && c < a.nq) *reinterpret_cast<typename El::Out4 *>(line + c) = o;
            else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + e < a.nq) line[c + e] = o[e];
            }
        }
    }
}

template <class E, ColsKind KIND, int BP, int BQ, int WP, int WQ>
hipError_t go(const ColsArgs &a, hipStream_t s) {
    const int64_t tp = KIND == ColsKind::kLowP ? a.blocks : (a.np + BP - 1) / BP;
    const int64_t tq = KIND == ColsKind::kLowQ ? a.blocks : (a.nq + BQ - 1) / BQ;
    return launch_kernel(k_cols<E, KIND, BP, BQ, WP, WQ>, dim3(static_cast<uint32_t>(tp * tq), a.g.G), dim3(WP * WQ * 64), 0, s, a);
}

template <class E>
hipError_t pick(ColsKind kind, const ColsArgs &a, hipStream_t s) {
    constexpr int L = kLowBytes / sizeof(E);
    switch (kind) {
    case ColsKind::kDense: return go<E, ColsKind::kDense, 128, 128, 2, 2>(a, s);
    case ColsKind::kLowP: return go<E, ColsKind::kLowP, L, 128, 1, 4>(a, s);
    default: return go<E, ColsKind::kLowQ, 128, L, 4, 1>(a, s);
    }
}

}  // namespace

hipError_t launch_cols(bool bf16, ColsKind kind, const ColsArgs &a, int cus, hipStream_t s) {
    (void)cus;
    return bf16 ? pick<__bf16>(kind, a, s) : pick<float>(kind, a, s);
}

}  // namespace hwr
