// Activations and their slopes in 32 bits: what kernels that end in one share (pcsr_norm.hip, pcsr_linear_kernels.h).
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

// The same share for results of 16 bits: P of degree 4, good to 2^-14 of itself, where fp16 rounds by up to 2^-11 (five operations and a
// constant less, of nineteen).  The slope of gelu, whose share this is, is 1.15 2^-16 off at most, at 0.
__device__ __forceinline__ float below_normal16(float z, float bell)
{
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.38f, fabsf(z), 1.0f));
    float h = __builtin_fmaf(-0.089927018f, t, 0.188873593f);
    h = __builtin_fmaf(h, t, 0.0919819028f);
    h = __builtin_fmaf(h, t, 0.157828814f);
    h = __builtin_fmaf(h, t, 0.151225205f);
    const float q = bell * t * h;
    return z < 0.0f ? q : 1.0f - q;
}
// z becomes the activation, and s its slope where asked for.  FEW: for results of 16 bits.
template <bool FEW, bool SLOPE, int N> __device__ __forceinline__ void activate_for(float (&z)[N], float (&s)[N], int act)
{
    switch (act) {
    case PCSR_ACT_RELU:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (SLOPE) s[i] = z[i] > 0.0f ? 1.0f : z[i] <= 0.0f ? 0.0f : z[i];
            z[i] = z[i] < 0.0f ? 0.0f : z[i];
        }
        break;
    case PCSR_ACT_SILU:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float p = __builtin_amdgcn_rcpf(1.0f + __expf(-z[i]));
            if (SLOPE) s[i] = p * (1.0f + z[i] * (1.0f - p));
            z[i] *= p;
        }
        break;
    case PCSR_ACT_GELU:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float bell = __builtin_amdgcn_exp2f(z[i] * z[i] * -0.72134752f), p = FEW ? below_normal16(z[i], bell) : below_normal(z[i], bell);
            if (SLOPE) s[i] = p + z[i] * 0.39894228f * bell;
            z[i] *= p;
        }
        break;
    }
}

} // namespace
} // namespace pcsr
