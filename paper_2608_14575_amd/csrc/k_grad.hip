// Both gradients of a product, of the rows and of the weights, in one launch: they read the same rows and do
// not depend on each other, and apart each would fill its last round of tiles on its own.
#include "cols_device.hpp"
#include "rows_device.hpp"
#include "slope_device.hpp"

namespace hwr {
namespace {

// Workgroups [0, first) make tiles of dx, those to `second` tiles of dW, the largest groups' first: tiles of dx take the longest
// but for those, and short ones fill the end.  The others add up the bias gradient's partial sums.  Two stage buffers, tiles of 64
// too: there are many workgroups, and more of them on a compute unit hide more than more stages of each (us, two / four: fp32
// 2,051 rows 771 x 390 53 / 61, 4,096 x 1024 x 1024 173 / 188; bf16 2,000 x 512 x 512 9.2 / 13.7, 700 x 256 x 512 9.5 / 8.8).
template <class E, int BM, int BN, int WR, int WC, int BP, int WP, int WQ>
__global__ void __launch_bounds__(WR *WC * 64) k_grad(RowsArgs a, ColsArgs b, SlopeArgs c, int first, int second) {
    static_assert(WR * WC == WP * WQ);
    constexpr int kCols = kColsBuf<E, ColsKind::kDense, BP, BP>, kBuf = std::max(kRowsBuf<BM, BN>, kCols);
    __shared__ __attribute__((aligned(16))) char buf0[kBuf], buf1[kBuf];
    __shared__ int rows[BM];
    const int id = block_id<WR * WC * 64>();
    if (id < first) {
        RowTile rt;
        int c0, part;
        if (row_tile<RowsKind::kGrouped, BM, BN>(a, id, threadIdx.x & 63, rt, c0, part))
            rows_direct<E, RowsKind::kGrouped, false, BM, BN, WR, WC, false>(a, rt, c0, part, buf0, buf1, nullptr, nullptr, rows);
    } else if (id < second) {
        cols_direct<E, ColsKind::kDense, BP, BP, WP, WQ, false>(b, id - first, buf0, buf1, nullptr, nullptr);
    } else if (c.dbias && id - second < bias_blocks(c)) {
        sum_bias<E>(c, id - second, reinterpret_cast<f32x4 *>(buf0));
    }
}

template <class E, int BM, int BN, int WR, int WC, int BP, int WP, int WQ>
hipError_t go(const RowsArgs &a, const ColsArgs &b, const SlopeArgs &c, hipStream_t s) {
    constexpr int NT = WR * WC * 64;
    const int64_t first = rows_blocks<RowsKind::kGrouped, BM, BN>(a);
    const int64_t second = first + cols_blocks(b, (b.np + BP - 1) / BP, (b.nq + BP - 1) / BP);
    const int64_t blocks = second + (c.dbias ? bias_blocks(c) : 0);
    if (blocks > INT32_MAX - grid_row(NT)) return hipErrorInvalidValue;
    return launch_kernel(k_grad<E, BM, BN, WR, WC, BP, WP, WQ>, wide_grid(blocks, NT), dim3(NT), 0, s, a, b, c, static_cast<int>(first),
                         static_cast<int>(second));
}

}  // namespace

// Both in whole chunks, and tiles of one size: of others the larger one's LDS would leave room for one
// workgroup on a compute unit.
bool grad_pair(const RowsPlan &p, const ColsPlan &q) { return p.direct && q.direct && p.bn == q.tile; }

hipError_t launch_grad(bool bf16, const RowsPlan &p, const RowsArgs &a, const ColsArgs &b, const SlopeArgs &c, hipStream_t s) {
    if (bf16) {
        if (p.bm == 256) return go<__bf16, 256, 256, 2, 4, 256, 2, 4>(a, b, c, s);
        return p.bm == 128 ? go<__bf16, 128, 128, 2, 2, 128, 2, 2>(a, b, c, s) : go<__bf16, 64, 64, 2, 2, 64, 2, 2>(a, b, c, s);
    }
    if (p.bm == 128) return go<float, 128, 128, 2, 2, 128, 2, 2>(a, b, c, s);
    return p.bm == 64 ? go<float, 64, 64, 2, 2, 64, 2, 2>(a, b, c, s) : go<float, 32, 64, 1, 4, 64, 2, 2>(a, b, c, s);
}

}  // namespace hwr
