// Activations and their derivatives, in fp32.
//
// gelu is z Phi(z) with the normal distribution's Phi.  fp32 calls take the library's erfcf and
// expf.  For bf16 results, off by 2^-9 for their rounding alone, these would cost 40 to 60
// instructions a value where a product's epilogue has the matrix units wait; there
//   Phi(-a) = exp(-a^2 / 2) R(t), t = 1 / (1 + 0.38 a), a >= 0,
// with R of five powers of t, fitted here to erfc over 0 <= a <= 14 by least squares reweighted towards
// the smallest largest relative error (3.6e-5, 2^-14.8; past 14 Phi(-a) is below the smallest
// normal fp32 value), and the hardware's exp2 and reciprocal (1 ulp).
#pragma once

#include "ops_device.hpp"

namespace hwr {

constexpr float kActLog2e = 1.44269504088896340736f;

// exp(-z^2 / 2) and, of it, Phi(z) = 1 - phi r or phi r
template <class E>
struct Normal {
    float density, upto;          // exp(-z^2 / 2), Phi(z)
    __device__ explicit Normal(float z) {
        if constexpr (sizeof(E) == 2) {
            const float a = fabsf(z), t = __builtin_amdgcn_rcpf(fmaf(0.38f, a, 1.0f));
            float r = fmaf(t, -0.08993185f, 0.18888356f);
            r = fmaf(t, r, 0.09197541f);
            r = fmaf(t, r, 0.15783013f);
            r = fmaf(t, r, 0.15122521f);
            density = __builtin_amdgcn_exp2f(z * z * (-0.5f * kActLog2e));
            const float tail = density * (t * r);
            upto = z > 0.0f ? 1.0f - tail : tail;
        } else {
            density = expf(-0.5f * z * z);
            upto = 0.5f * erfcf(z * -0.70710678118654752440f);
        }
    }
};

template <class E>
__device__ inline float logistic(float z) {
    if constexpr (sizeof(E) == 2) return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kActLog2e * z));
    else return 1.0f / (1.0f + expf(-z));
}

template <class E, int ACT>
__device__ inline float activate(float z) {
    if constexpr (ACT == HWR_ACT_RELU) return z < 0.0f ? 0.0f : z;        // (a NaN stays)
    else if constexpr (ACT == HWR_ACT_SILU) return z * logistic<E>(z);
    else if constexpr (ACT == HWR_ACT_GELU) return z * Normal<E>(z).upto;
    else return z;
}

template <class E, int ACT>
__device__ inline float slope(float z) {
    if constexpr (ACT == HWR_ACT_RELU) {
        return z > 0.0f ? 1.0f : z == z ? 0.0f : z;
    } else if constexpr (ACT == HWR_ACT_SILU) {
        const float h = logistic<E>(z);
        return h * fmaf(z, 1.0f - h, 1.0f);
    } else if constexpr (ACT == HWR_ACT_GELU) {
        const Normal<E> d(z);
        return fmaf(z * 0.39894228040143267794f, d.density, d.upto);
    } else {
        return 1.0f;
    }
}

// run(constant) with the activation as a constant.
template <class Run>
__device__ __host__ __forceinline__ auto with_act(int act, Run &&run) {
    if (act == HWR_ACT_RELU) return run(std::integral_constant<int, HWR_ACT_RELU>{});
    if (act == HWR_ACT_SILU) return run(std::integral_constant<int, HWR_ACT_SILU>{});
    if (act == HWR_ACT_GELU) return run(std::integral_constant<int, HWR_ACT_GELU>{});
    return run(std::integral_constant<int, HWR_ACT_NONE>{});
}

// What follows a product for V neighbouring columns c (below m) of rows of one group (g == G: of none: their
// sums are zeros, and stay so without a bias, whatever the activation).
template <class E, int V>
struct Finish {
    Some<E, V> b;                 // the bias as it stands in memory, until settle(): no one waits for it here
    float bias[V];
    const Epilogue &a;
    int c, m;
    bool biased;
    __device__ __forceinline__ Finish(const Epilogue &end, int c_, int m_, int G, int g) : a(end), c(c_), m(m_), biased(g < G && end.bias && c_ < m_) {
        if (biased) b.load(static_cast<const E *>(a.bias) + static_cast<int64_t>(g) * m, c, m);
    }
    __device__ __forceinline__ void settle() {
#pragma unroll
        for (int i = 0; i < V; ++i) bias[i] = biased ? static_cast<float>(b.e[i]) : 0.0f;
    }
    // the residual of row r
    __device__ __forceinline__ void load(int64_t r, Some<E, V> &res) const {
        if (a.residual && c < m) res.load(static_cast<const E *>(a.residual) + r * a.ldr, c, m);
    }
    // z = v + bias and y = act(z) + residual of row r
    __device__ __forceinline__ void store(int64_t r, const Some<E, V> &res, const float (&v)[V], E *y, int64_t ldy) const {
        if (c >= m) return;
        float z[V], o[V];
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = v[i] + bias[i];
        if (a.z) Some<E, V>(z).store(static_cast<E *>(a.z) + r * a.ldz, c, m);
        with_act(a.act, [&](auto A) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = activate<E, A.value>(z[i]);
        });
        if (a.residual) {
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] += static_cast<float>(res.e[i]);
        }
        Some<E, V>(o).store(y + r * ldy, c, m);
    }
};

}  // namespace hwr
