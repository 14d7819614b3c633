// Both gradients of a product, of the rows and of the weights, in one launch: they read the same rows and do
// not depend on each other, and apart each would fill its last round of tiles on its own.
#include "cols_device.hpp"
#include "rows_device.hpp"

namespace hwr {
namespace {

// Workgroups [0, first) make tiles of dx, the others of dW, the largest groups' first: tiles of dx take the longest but for those,
// and short ones fill the end.
template <class E, int BM, int BN, int WR, int WC, int BP, int WP, int WQ>
__global__ void __launch_bounds__(WR *WC * 64) k_grad(RowsArgs a, ColsArgs b, int first) {
    static_assert(WR * WC == WP * WQ);
    constexpr int kCols = kColsBuf<E, ColsKind::kDense, BP, BP>, kBuf = std::max(kRowsBuf<BM, BN>, kCols);
    constexpr int kMore = std::max(kRowsDeep<BN> ? kRowsBuf<BM, BN> : 16, BP == 64 ? kCols : 16);
    __shared__ __attribute__((aligned(16))) char buf0[kBuf], buf1[kBuf], buf2[kMore], buf3[kMore];
    __shared__ int rows[BM];
    const int id = block_id<WR * WC * 64>();
    if (id < first) rows_direct<E, RowsKind::kGrouped, false, BM, BN, WR, WC>(a, id, buf0, buf1, buf2, buf3, rows);
    else cols_direct<E, ColsKind::kDense, BP, BP, WP, WQ>(b, id - first, buf0, buf1, buf2, buf3);
}

template <class E, int BM, int BN, int WR, int WC, int BP, int WP, int WQ>
hipError_t go(const RowsArgs &a, const ColsArgs &b, hipStream_t s) {
    constexpr int NT = WR * WC * 64;
    const int64_t first = rows_blocks<RowsKind::kGrouped, BM, BN>(a);
    const int64_t blocks = first + cols_blocks(b, (b.np + BP - 1) / BP, (b.nq + BP - 1) / BP);
    if (blocks > INT32_MAX - grid_row(NT)) return hipErrorInvalidValue;
    return launch_kernel(k_grad<E, BM, BN, WR, WC, BP, WP, WQ>, wide_grid(blocks, NT), dim3(NT), 0, s, a, b, static_cast<int>(first));
}

}  // namespace

// Both in whole chunks, and tiles of one size: of others the larger one's LDS would leave room for one
// workgroup on a compute unit.
bool grad_pair(const RowsPlan &p, const ColsPlan &q) { return p.direct && q.direct && p.bn == q.tile; }

hipError_t launch_grad(bool bf16, const RowsPlan &p, const RowsArgs &a, const ColsArgs &b, hipStream_t s) {
    if (bf16) {
        if (p.bm == 256) return go<__bf16, 256, 256, 2, 4, 256, 2, 4>(a, b, s);
        return p.bm == 128 ? go<__bf16, 128, 128, 2, 2, 128, 2, 2>(a, b, s) : go<__bf16, 64, 64, 2, 2, 64, 2, 2>(a, b, s);
    }
    if (p.bm == 128) return go<float, 128, 128, 2, 2, 128, 2, 2>(a, b, s);
    return p.bm == 64 ? go<float, 64, 64, 2, 2, 64, 2, 2>(a, b, s) : go<float, 32, 64, 1, 4, 64, 2, 2>(a, b, s);
}

}  // namespace hwr
