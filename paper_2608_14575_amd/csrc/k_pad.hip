// Copies with rows padded to whole chunks: products of odd widths are worth a pass over
// their operands when they are large (hwr_ops.hip says when).  Bound by memory.
#include "slope_device.hpp"

namespace hwr {
namespace {

constexpr int kThreads = 256;

template <class E>
__global__ void __launch_bounds__(kThreads) k_pad(PadArgs a) {
    pad_rows<E, kThreads>(a.m[blockIdx.y], blockIdx.x);
}

}  // namespace

int64_t padded_width(bool bf16, int width) {
    const int epc = bf16 ? 8 : 4;
    return (width + epc - 1) / epc * epc;
}

hipError_t launch_pad(bool bf16, const PadArgs &a, hipStream_t s) {
    const dim3 grid(kPadBlocks, a.count), block(kThreads);
    return bf16 ? launch_kernel(k_pad<__bf16>, grid, block, 0, s, a) : launch_kernel(k_pad<float>, grid, block, 0, s, a);
}

}  // namespace hwr
