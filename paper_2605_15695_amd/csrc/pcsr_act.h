// Activations and their slopes in 32 bits: what kernels that end in one share (pcsr_norm.hip, pcsr_linear.hip).
#pragma once
#include <hip/hip_runtime.h>

#include "pcsr_train.h"

namespace pcsr {
namespace {

// The share of the normal distribution below z; bell: exp(-z^2 / 2), which the slope of gelu needs as well.  Below zero the share over the
// bell is t P(t) with t = 1 / (1 + 0.346 |z|), P of degree 8 by weighted least squares for the smallest relative error over z from -14 to 0 (3.5e-8;
// in fp32 5 u (1 + z^2), u = 2^-24, of which z^2 is the exponential's), so that gelu keeps its digits far below zero, where it is small.
__device__ __forceinline__ float below_normal(float z, float bell)
{
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.346f, fabsf(z), 1.0f));
    constexpr float P[8] = {0.14520301f, -0.26838204f, 0.18176714f, -0.03471449f, 0.1105235f, 0.11777047f, 0.13838688f, 0.13801986f};
    float h = -0.02857433f;
#pragma unroll
    for (int k = 0; k < 8; ++k) h = __builtin_fmaf(h, t, P[k]);
    const float q = bell * t * h;
    return z < 0.0f ? q : 1.0f - q;
}
template <int N> __device__ __forceinline__ void activate(float (&z)[N], int act)
{
    switch (act) { // the same for the whole launch
    case PCSR_ACT_RELU:
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = z[i] < 0.0f ? 0.0f : z[i]; // a NaN stays one
        break;
    case PCSR_ACT_SILU:
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = z[i] * __builtin_amdgcn_rcpf(1.0f + __expf(-z[i]));
        break;
    case PCSR_ACT_GELU:
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = z[i] * below_normal(z[i], __expf(-0.5f * z[i] * z[i]));
        break;
    }
}
// z becomes the activation's slope there
template <int N> __device__ __forceinline__ void slopes(float (&z)[N], int act)
{
    switch (act) {
    case PCSR_ACT_RELU:
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = z[i] > 0.0f ? 1.0f : z[i] <= 0.0f ? 0.0f : z[i];
        break;
    case PCSR_ACT_SILU:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float p = __builtin_amdgcn_rcpf(1.0f + __expf(-z[i]));
            z[i] = p * (1.0f + z[i] * (1.0f - p));
        }
        break;
    case PCSR_ACT_GELU:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float bell = __expf(-0.5f * z[i] * z[i]);
            z[i] = below_normal(z[i], bell) + z[i] * 0.39894228f * bell;
        }
        break;
    default:
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = 1.0f;
    }
}

// both: z becomes the activation, s its slope
template <int N> __device__ __forceinline__ void activate(float (&z)[N], float (&s)[N], int act)
{
    switch (act) {
    case PCSR_ACT_RELU:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s[i] = z[i] > 0.0f ? 1.0f : z[i] <= 0.0f ? 0.0f : z[i];
            z[i] = z[i] < 0.0f ? 0.0f : z[i];
        }
        break;
    case PCSR_ACT_SILU:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float p = __builtin_amdgcn_rcpf(1.0f + __expf(-z[i]));
            s[i] = p * (1.0f + z[i] * (1.0f - p));
            z[i] *= p;
        }
        break;
    case PCSR_ACT_GELU:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float bell = __expf(-0.5f * z[i] * z[i]), p = below_normal(z[i], bell);
            s[i] = p + z[i] * 0.39894228f * bell;
            z[i] *= p;
        }
        break;
    }
}

} // namespace
} // namespace pcsr
