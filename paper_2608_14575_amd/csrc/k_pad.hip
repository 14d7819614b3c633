// Copies with rows padded to whole chunks: products of odd widths are worth a pass over
// their operands when they are large (hwr_ops.hip says when).  Bound by memory.
#include "ops_device.hpp"

namespace hwr {
namespace {

constexpr int kThreads = 256;

template <class E>
__global__ void __launch_bounds__(kThreads) k_pad(PadArgs a) {
    constexpr int kEpc = Elem<E>::kEpc;
    const PadArgs::Matrix &m = a.m[blockIdx.y];
    const int per = (m.width + kEpc - 1) / kEpc;            // chunks of a row
    const int64_t chunks = m.rows * per, step = static_cast<int64_t>(gridDim.x) * kThreads;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < chunks; i += step) {
        const int64_t row = i / per;
        const int c = static_cast<int>(i - row * per) * kEpc;
        reinterpret_cast<u32x4 *>(m.dst)[i] = load_chunk<E>(static_cast<const E *>(m.src) + row * m.ld, c, m.width);
    }
}

}  // namespace

int64_t padded_width(bool bf16, int width) {
    const int epc = bf16 ? 8 : 4;
    return (width + epc - 1) / epc * epc;
}

hipError_t launch_pad(bool bf16, const PadArgs &a, hipStream_t s) {
    const dim3 grid(2048, a.count), block(kThreads);
    return bf16 ? launch_kernel(k_pad<__bf16>, grid, block, 0, s, a) : launch_kernel(k_pad<float>, grid, block, 0, s, a);
}

}  // namespace hwr
