// One step of AdamW over many tensors in one launch:
//   m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2,
//   p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt v / sqrt(1 - b2^t) + eps)
// in fp32.  Weights are fp32, bf16 with an fp32 master, or bf16 alone; states fp32 or 8 bits.
//
// States of 8 bits are e4m3 values with a scale for every 256: the largest of the block is 448
// scales.  The root of v is held in place of v (whose range would not fit), and is never rounded
// down to 0, which would make a step of lr m / eps.  A change of a state in one step is mostly
// smaller than half a step of e4m3 (2^-4 of the value), and of bf16 weights that have no
// master smaller than 2^-9: rounded to nearest they would stand still, so they are rounded up or
// down with the probability of the remainder.  The noise is a hash of the seed, the step
// and the value's place.  The root is without a bias then, its square is not: it grows by the variance of the
// rounding, in a step at most the root's way (half of 1 - b2 of |g^2 / v - 1|) times the codes' distance (an eighth of the root), over the
// 1 / (1 - b2) steps that v remembers by some 5% of v, with a standard deviation of 0.35.
//
// Bound by memory: 28 bytes a value with fp32 states (bf16 without masters 22), 16 with 8 bits (bf16 without masters 10).  A workgroup takes 8
// blocks of a tensor, a thread 8 values (16 bytes of bf16 at a time), a half-wave a block, so that a scale takes five
// exchanges.  67.6 M values in 16 tensors: fp32 states, bf16 with masters 357 us (5.3 TB/s), fp32 353,
// bf16 alone 273; states of 8 bits, bf16 with masters 200, fp32 198 (5.5 TB/s), bf16 alone 133 to 138 (5.0 TB/s; 180 when the
// roundings were made of integer steps, at 105 instructions a value); 466,000 fp32 values in 48
// tensors 5 us, which is one wave of workgroups.
#include <cmath>
#include <utility>

#include "ops_device.hpp"

namespace hwr {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = kAdamwChunk / kThreads;     // values of a thread
constexpr int kBlockLanes = kAdamwBlock / kPer;  // threads of a block
static_assert(kPer == 8 && kBlockLanes == 32);

typedef uint32_t u32x2_a1 __attribute__((ext_vector_type(2), aligned(1)));

// Values [e, e + 8) of a line of len, zeros past it.
template <class E>
__device__ inline void load8(const E *line, int e, int len, float (&f)[kPer]) {
    constexpr int kEpc = Elem<E>::kEpc;
#pragma unroll
    for (int i = 0; i < kPer / kEpc; ++i) {
        const u32x4 v = load_chunk<E>(line, e + i * kEpc, len);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(E) == 2) {
                f[2 * j] = __uint_as_float(v[j] << 16);
                f[2 * j + 1] = __uint_as_float(v[j] & 0xFFFF0000u);
            } else {
                f[i * 4 + j] = __uint_as_float(v[j]);
            }
        }
    }
}
__device__ inline void store8(float *line, int e, int len, const float (&f)[kPer]) {
#pragma unroll
    for (int i = 0; i < kPer; i += 4) store_four<float>(line, e + i, len, f32x4{f[i], f[i + 1], f[i + 2], f[i + 3]});
}
// (rounded to nearest; values that are bf16 already stay what they are)
__device__ inline void store8(__bf16 *line, int e, int len, const float (&f)[kPer]) {
    union { u32x4_a2 v; __bf16 s[kPer]; } u;
#pragma unroll
    for (int i = 0; i < kPer; ++i) u.s[i] = static_cast<__bf16>(f[i]);
    if (e + kPer <= len) {
        *reinterpret_cast<u32x4_a2 *>(line + e) = u.v;
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (e + i < len) line[e + i] = u.s[i];
    }
}
__device__ inline u32x2_a1 load8_bytes(const uint8_t *line, int e, int len) {
    if (e + kPer <= len) return *reinterpret_cast<const u32x2_a1 *>(line + e);
    uint32_t v[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (e + i < len) v[i / 4] |= static_cast<uint32_t>(line[e + i]) << (i % 4 * 8);
    return u32x2_a1{v[0], v[1]};
}
__device__ inline void store8_bytes(uint8_t *line, int e, int len, const uint32_t (&v)[2]) {
    if (e + kPer <= len) {
        *reinterpret_cast<u32x2_a1 *>(line + e) = u32x2_a1{v[0], v[1]};
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (e + i < len) line[e + i] = static_cast<uint8_t>(v[i / 4] >> (i % 4 * 8));
    }
}
__device__ inline void from_e4m3(u32x2_a1 v, float scale, float (&f)[kPer]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(v[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(v[i], true);
        f[4 * i] = lo[0] * scale, f[4 * i + 1] = lo[1] * scale;
        f[4 * i + 2] = hi[0] * scale, f[4 * i + 3] = hi[1] * scale;
    }
}

// Byte SEL of `into` becomes x (at most 448 in magnitude) in e4m3, up or down by the 16 bits of noise at the top of
// `noise`: the instruction adds the noise's upper 20 bits to the bits of x below those that stay (below 2^-6, where
// steps no longer shrink with the value, to the bits below that step), and cuts them.
template <int SEL>
__device__ inline uint32_t to_e4m3(float x, uint32_t noise, uint32_t into) {
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_sr_fp8_f32(x, static_cast<int>(noise), static_cast<int>(into), SEL));
}
// fp32 to the bits of a bf16, as fp32.  (One that would round past the largest stays below; the sum of a NaN's bits and
// the noise may pass all ones, and be a zero's.)
__device__ inline float to_bf16(float x, uint32_t noise) {
    const uint32_t bits = __float_as_uint(x), up = bits + noise;
    return __uint_as_float((x != x || (up & 0x7F800000u) == 0x7F800000u ? bits : up) & 0xFFFF0000u);
}

// sqrt(v), one step of the residual's correction after the hardware's reciprocal root: rounded right but for
// values within 2^-20 of the middle of two.  (The library's takes twice as many instructions, for denormal v; less than
// the root comes out there, below 2^-63.)
__device__ inline float root_of(float v) {
    const float y = __builtin_amdgcn_rsqf(fmaxf(v, 0x1p-126f)), s = v * y;
    return fmaf(fmaf(-s, s, v), 0.5f * y, s);
}

// Scale of a block, and what values are multiplied with.  Blocks of less than 2^-100 become zeros (the factor would
// pass the largest fp32 value).  With a NaN among them all become NaN: it stays in the scale.
__device__ inline float block_scale(const float (&f)[kPer], float &factor) {
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) most = __builtin_elementwise_maximum(most, fabsf(f[i]));
#pragma unroll
    for (int d = 1; d < kBlockLanes; d <<= 1) most = __builtin_elementwise_maximum(most, __shfl_xor(most, d));
    const bool none = most < 0x1p-100f;
    factor = none ? 0.0f : 1.0f / most * 448.0f;       // (products may round past 448: they are cut there)
    return none ? 0.0f : most * (1.0f / 448.0f);
}

template <class F, int... I>
__device__ inline void each_of(F f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}

template <class E, bool MASTER, bool STATES8>
__global__ void __launch_bounds__(kThreads, 8) k_adamw(AdamwArgs a) {   // as many waves as there may be
    const int id = block_id<kThreads>();
    if (id >= a.n_chunks) return;
    const AdamwTensor &t = a.tensors[a.chunks[id]];
    const AdamwCoef &c = a.coef_device ? *a.coef_device : a.coef;
    const int64_t at = (id - t.first) * kAdamwChunk;
    const int len = static_cast<int>(min(t.count - at, static_cast<int64_t>(kAdamwChunk)));
    const int e = threadIdx.x * kPer;
    const int64_t block = at / kAdamwBlock + threadIdx.x / kBlockLanes;
    const bool has_block = e / kAdamwBlock * kAdamwBlock < len;

    float g[kPer], p[kPer], m[kPer], v[kPer], root[kPer];
    load8<E>(static_cast<const E *>(t.g) + at, e, len, g);
    if constexpr (MASTER) load8<float>(t.master + at, e, len, p);
    else load8<E>(static_cast<const E *>(t.p) + at, e, len, p);
    if constexpr (STATES8) {
        const u32x2_a1 mb = load8_bytes(static_cast<const uint8_t *>(t.m) + at, e, len),
                       vb = load8_bytes(static_cast<const uint8_t *>(t.v) + at, e, len);
        const float ms = has_block ? t.m_scale[block] : 0.0f, vs = has_block ? t.v_scale[block] : 0.0f;
        from_e4m3(mb, ms, m);
        from_e4m3(vb, vs, v);
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] *= v[i];
    } else {
        load8<float>(static_cast<const float *>(t.m) + at, e, len, m);
        load8<float>(static_cast<const float *>(t.v) + at, e, len, v);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        m[i] = m[i] * c.beta1 + g[i] * c.beta1_rest;
        v[i] = v[i] * c.beta2 + g[i] * g[i] * c.beta2_rest;
        if constexpr (STATES8) {               // (the hardware's reciprocal, 1 ulp)
            root[i] = root_of(v[i]);
            p[i] = p[i] * c.decay - m[i] * __builtin_amdgcn_rcpf(fmaf(root[i], c.root_rate, c.eps)) * c.rate;
        } else {
            root[i] = sqrtf(v[i]);
            p[i] = p[i] * c.decay - m[i] / (root[i] * c.root_rate + c.eps) * c.rate;
        }
    }
    uint32_t noise[kPer], more[kPer];
    if constexpr (STATES8 || (!MASTER && sizeof(E) == 2)) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            uint32_t h = (static_cast<uint32_t>(t.place + at) + e + i + c.key) * 0x9E3779B9u;
            h = (h ^ h >> 15) * 0xBB67AE85u;
            noise[i] = h ^ h >> 16;
            h = noise[i] * 0x510E527Fu;
            more[i] = h ^ h >> 16;
        }
    }
    if constexpr (MASTER) {
        store8(t.master + at, e, len, p);
    } else if constexpr (sizeof(E) == 2) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) p[i] = to_bf16(p[i], more[i] >> 16);
    }
    store8(static_cast<E *>(t.p) + at, e, len, p);
    if constexpr (STATES8) {
        float mf, vf;
        const float ms = block_scale(m, mf), vs = block_scale(root, vf);
        uint32_t mb[2] = {0, 0}, vb[2] = {0, 0};
        auto encode = [&](auto at) {
            constexpr int i = decltype(at)::value;
            mb[i / 4] = to_e4m3<i % 4>(__builtin_amdgcn_fmed3f(m[i] * mf, -448.0f, 448.0f), noise[i] << 16, mb[i / 4]);
            // (a root is never rounded down to 0)
            const float y = fminf(root[i] * vf, 448.0f);
            vb[i / 4] = to_e4m3<i % 4>(y > 0.0f && y < 0x1p-9f ? 0x1p-9f : y, noise[i] & 0xFFFF0000u, vb[i / 4]);
        };
        each_of(encode, std::make_integer_sequence<int, kPer>{});
        store8_bytes(static_cast<uint8_t *>(t.m) + at, e, len, mb);
        store8_bytes(static_cast<uint8_t *>(t.v) + at, e, len, vb);
        if (has_block && threadIdx.x % kBlockLanes == 0) {
            t.m_scale[block] = ms;
            t.v_scale[block] = vs;
        }
    } else {
        store8(static_cast<float *>(t.m) + at, e, len, m);
        store8(static_cast<float *>(t.v) + at, e, len, v);
    }
}

__host__ __device__ inline AdamwCoef coefficients(double lr, double beta1, double beta2, double eps, double weight_decay,
                                                  uint64_t seed, int64_t step) {
    AdamwCoef c;
    c.decay = static_cast<float>(1.0 - lr * weight_decay);
    c.beta1 = static_cast<float>(beta1);
    c.beta1_rest = static_cast<float>(1.0 - beta1);
    c.beta2 = static_cast<float>(beta2);
    c.beta2_rest = static_cast<float>(1.0 - beta2);
    c.rate = static_cast<float>(lr / (1.0 - pow(beta1, static_cast<double>(step))));
    c.root_rate = static_cast<float>(1.0 / sqrt(1.0 - pow(beta2, static_cast<double>(step))));
    // (the hardware's reciprocal takes smaller ones for 0, and the conversion may: 0 / 0 is for an eps of 0 alone)
    c.eps = eps > 0.0 ? fmaxf(static_cast<float>(eps), 0x1p-126f) : 0.0f;
    c.key = static_cast<uint32_t>((seed * 0x9E3779B97F4A7C15u + static_cast<uint64_t>(step)) * 0xBB67AE8584CAA73Bu >> 32);
    return c;
}

__global__ void k_adamw_coef(AdamwRates a, AdamwCoef *out) {
    if (blockIdx.x || threadIdx.x) return;
    const int64_t step = *a.steps + 1;
    *a.steps = step;
    *out = coefficients(a.lr_device ? *a.lr_device : a.lr, a.beta1, a.beta2, a.eps, a.weight_decay, a.seed, step);
}

template <class E, bool MASTER, bool STATES8>
hipError_t go(const AdamwArgs &a, hipStream_t s) {
    return launch_kernel(k_adamw<E, MASTER, STATES8>, wide_grid(a.n_chunks, kThreads), dim3(kThreads), 0, s, a);
}

}  // namespace

AdamwCoef adamw_coef(double lr, double beta1, double beta2, double eps, double weight_decay, uint64_t seed, int64_t step) {
    return coefficients(lr, beta1, beta2, eps, weight_decay, seed, step);
}

hipError_t launch_adamw_coef(const AdamwRates &a, AdamwCoef *out, hipStream_t s) {
    return launch_kernel(k_adamw_coef, dim3(1), dim3(64), 0, s, a, out);
}

hipError_t launch_adamw(bool bf16, bool master, bool states8, const AdamwArgs &a, hipStream_t s) {
    if (!bf16) return states8 ? go<float, false, true>(a, s) : go<float, false, false>(a, s);
    if (master) return states8 ? go<__bf16, true, true>(a, s) : go<__bf16, true, false>(a, s);
    return states8 ? go<__bf16, false, true>(a, s) : go<__bf16, false, false>(a, s);
}

}  // namespace hwr
