// Numbers of 32 and 16 bits in memory, 32 bits in registers: what the kernels of the training step share
// (pcsr_embed.hip, pcsr_norm.hip, pcsr_ortho.hip, pcsr_drop.hip, pcsr_linear_kernels.h).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "pcsr_train.h"

namespace pcsr {
namespace {

typedef _Float16 half_t;
typedef __bf16 bfloat_t;

// N numbers at an address that is a multiple of one number's size alone: the memory unit takes 16 bytes from there
// in one access, so that rows of odd widths move as fast as others
template <typename T, int N> struct Pack {
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
template <typename T> constexpr int kPer16 = 16 / (int)sizeof(T);

template <typename T, int N> __device__ __forceinline__ void load(const T *p, float (&x)[N])
{
    const typename Pack<T, N>::type v = *reinterpret_cast<const typename Pack<T, N>::type *>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (float)v[i];
}
// rounded to nearest, once
template <typename T, int N> __device__ __forceinline__ void store(T *p, const float (&x)[N])
{
    typename Pack<T, N>::type v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (T)x[i];
    *reinterpret_cast<typename Pack<T, N>::type *>(p) = v;
}
// the first m of N, zeros behind them: the end of a row
template <typename T, int N> __device__ __forceinline__ void load_some(const T *p, int m, float (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = i < m ? (float)p[i] : 0.0f;
}
template <typename T, int N> __device__ __forceinline__ void store_some(T *p, int m, const float (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < m) p[i] = (T)x[i];
}
template <typename T, int N> __device__ __forceinline__ void load_upto(const T *p, int m, float (&x)[N])
{
    if (m >= N)
        load<T, N>(p, x);
    else
        load_some<T, N>(p, m, x);
}
template <typename T, int N> __device__ __forceinline__ void store_upto(T *p, int m, const float (&x)[N])
{
    if (m >= N)
        store<T, N>(p, x);
    else
        store_some<T, N>(p, m, x);
}

// Lets a kernel have so much LDS beside what it declares; more than 64 KB have to be asked for.
template <typename K> bool allow_lds(K *kernel, size_t bytes)
{
    if (bytes <= 64 * 1024) return true;
    const bool ok = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == hipSuccess;
    if (!ok) (void)hipGetLastError(); // the caller reports it: not the next call's
    return ok;
}
inline int launched() { return hipGetLastError() == hipSuccess ? PCSR_OK : PCSR_E_HIP; }

// f(a number of the type that `type` names), for kernels that are made for each
template <typename F> int for_type(int type, F f)
{
    switch (type) {
    case PCSR_F32: return f(float{});
    case PCSR_BF16: return f(bfloat_t{});
    case PCSR_F16: return f(half_t{});
    }
    return PCSR_E_UNSUPPORTED;
}

} // namespace
} // namespace pcsr
