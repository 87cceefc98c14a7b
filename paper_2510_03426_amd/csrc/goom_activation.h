// Parameters of the norms and their activations.
#pragma once

#include "goom_real.h"

namespace goom_layer {

__device__ inline float param(const void *p, int type, int i, float otherwise)
{
    if (!p) return otherwise;
    return type == GOOM_REAL_F32 ? reinterpret_cast<const float *>(p)[i] : type == GOOM_REAL_BF16 ? (float)reinterpret_cast<const bf16 *>(p)[i] : (float)reinterpret_cast<const f16 *>(p)[i];
}

// V parameters of neighbouring channels
template <int V> __device__ inline void params(const void *p, int type, int i, float otherwise, float (&x)[V])
{
    if (p && type == GOOM_REAL_F32) {
        constexpr int N = V > 4 ? 4 : V;
#pragma unroll
        for (int e = 0; e < V; e += N) {
            float y[N];
            load_floats_unaligned<float, N>(reinterpret_cast<const float *>(p) + i + e, y);
#pragma unroll
            for (int k = 0; k < N; k++) x[e + k] = y[k];
        }
    } else {
#pragma unroll
        for (int e = 0; e < V; e++) x[e] = param(p, type, i + e, otherwise);
    }
}

// 1 / (1 + e^-z) by the hardware's exponential and reciprocal (1 ulp each; the exponent's rounding adds |z| u where the value
// is near e^z): library exp and division were 25 of the 40 instructions an element and took longer than its bytes
__device__ inline float logistic(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504088896341f)); }

// Phi(z) = (1 + erf(z / sqrt 2)) / 2 and phi(z) = Phi'(z), from one exponential: the rational approximation 7.1.26 of Abramowitz
// and Stegun, Handbook of Mathematical Functions (absolute error of erf at most 1.5e-7, about one unit of a float near 1).  With
// the library's erf and exp the kernels were bound by some 80 instructions an element.
__device__ inline void normal(float z, float &cdf, float &density)
{
    const float x = fabsf(z) * 0.70710678118654752f, e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f), t = __builtin_amdgcn_rcpf(1.0f + 0.3275911f * x);
    const float tail = 0.5f * e * t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
    cdf = z < 0.0f ? tail : 1.0f - tail; // (a NaN stays one)
    density = e * 0.39894228040143268f;
}

__device__ inline float activate(float z, int act)
{
    if (act == GOOM_ACT_SILU) return z * logistic(z);
    if (act == GOOM_ACT_GELU) {
        float cdf, density;
        normal(z, cdf, density);
        return z * cdf;
    }
    return z;
}

__device__ inline float activate_slope(float z, int act)
{
    if (act == GOOM_ACT_SILU) {
        const float p = logistic(z);
        return p * (1.0f + z * (1.0f - p));
    }
    if (act == GOOM_ACT_GELU) {
        float cdf, density;
        normal(z, cdf, density);
        return cdf + z * density;
    }
    return 1.0f;
}

} // namespace goom_layer
