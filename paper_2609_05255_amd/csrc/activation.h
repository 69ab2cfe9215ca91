// Activations of the linear operators and their derivatives, fp32, without
// branches. exp is the hardware's exp2 of a scaled argument.
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/gsraster.h"

namespace gsr {

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

// Normal distribution function Phi(z), and its density's exp(-z^2 / 2).
// Phi(-|z|) exp(z^2 / 2) is t P(t), t = 1 / (1 + 0.3005204 |z|), with P fitted by
// weighted least squares to a relative error of 8e-8 over |z| < 12; in fp32 the
// result is within 2e-7.
__device__ __forceinline__ float normal_cdf(float z, float* density)
{
    const float t = __builtin_amdgcn_rcpf(1.f + 0.3005204f * fabsf(z));
    float p = 0.036853787f;
    p = fmaf(p, t, -0.16124097f);
    p = fmaf(p, t, 0.21188542f);
    p = fmaf(p, t, -0.05911236f);
    p = fmaf(p, t, 0.13154161f);
    p = fmaf(p, t, 0.09912653f);
    p = fmaf(p, t, 0.12111989f);
    p = fmaf(p, t, 0.11982605f);
    const float e = exp_of(-0.5f * z * z);
    *density = e * 0.39894228f;
    const float q = p * t * e;
    return z > 0.f ? 1.f - q : q;
}

__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.f + exp_of(-z)); }

// 1 - 2 / (1 + exp(2 z)); below 0.6, where that cancels, z + z^3 P(z^2) with P
// fitted to a relative error of 2e-7.
__device__ __forceinline__ float tanh_of(float z)
{
    const float s = z * z;
    float p = 0.015876217f;
    p = fmaf(p, s, -0.05237579f);
    p = fmaf(p, s, 0.13316134f);
    p = fmaf(p, s, -0.3333275f);
    const float large = 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + exp_of(2.f * z));
    return s < 0.36f ? fmaf(z * s, p, z) : large;
}

// v[k] = act(v[k]); an undefined value stays one
template <int N>
__device__ __forceinline__ void activate(int act, float* v)
{
    float unused;
    switch (act) {
    case GS_ACT_RELU:
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = v[k] <= 0.f ? 0.f : v[k];
        break;
    case GS_ACT_GELU:
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] *= normal_cdf(v[k], &unused);
        break;
    case GS_ACT_SILU:
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] *= logistic(v[k]);
        break;
    case GS_ACT_TANH:
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = tanh_of(v[k]);
        break;
    case GS_ACT_SIGMOID:
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = logistic(v[k]);
        break;
    default: break;
    }
}

// v[k] *= act'(z[k]). A stored z may be infinite where the type's range ends before that of the layer's own sums: the
// slope there is its limit, where the formula has infinity times 0. (Chosen by a comparison: bounding z instead takes
// registers for the bounds, which cost the narrow backward of 128 x 128 with relu 20 of 204 us.)
template <int N>
__device__ __forceinline__ void times_slope(int act, float* v, const float* z)
{
    switch (act) {
    case GS_ACT_RELU:
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = z[k] > 0.f ? v[k] : 0.f;
        break;
    case GS_ACT_GELU:
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float density;
            const float phi = normal_cdf(z[k], &density);
            v[k] *= fabsf(z[k]) < __builtin_inff() ? fmaf(z[k], density, phi) : phi;
        }
        break;
    case GS_ACT_SILU:
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float p = logistic(z[k]);
            v[k] *= fabsf(z[k]) < __builtin_inff() ? p * fmaf(z[k], 1.f - p, 1.f) : p;
        }
        break;
    case GS_ACT_TANH:
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float t = tanh_of(z[k]);
            v[k] *= 1.f - t * t;
        }
        break;
    case GS_ACT_SIGMOID:
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float p = logistic(z[k]);
            v[k] *= p * (1.f - p);
        }
        break;
    default: break;
    }
}

}  // namespace gsr
