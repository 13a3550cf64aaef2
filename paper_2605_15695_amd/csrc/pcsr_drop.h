// What is dropped, as a function of a seed, an offset and a number's place: nothing is stored (pcsr_drop.hip, pcsr_linear_kernels.h).
//
// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel Random Numbers: As Easy as 1, 2, 3", SC 2011) with the seed as key and the
// counter (column / 8, row, offset) gives 128 bits: 16 for each of 8 columns side by side, word by word, low half first.  A number is
// dropped where its 16 bits are below T = 65536 p, rounded, and multiplied by 65536 / (65536 - T) otherwise, so that the mean stays
// whatever p was rounded by.  16 bits and not 32: a call is 20 wide multiplications, which take a quarter of the rate, some 640 cycles of a SIMD in all;
// for 8 numbers each that is 60 % of the time that memory takes for 16-bit numbers, for 4 it would be the bound.
#pragma once
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "pcsr_train.h"

namespace pcsr {
namespace {

struct Drop {
    uint32_t seed[2], offset[2];
    const int64_t *state; // seed and offset in device memory instead
    int64_t *used;        // what was used is written there
    uint32_t threshold;   // 0: nothing is dropped
    float keep;
};
inline Drop drop_of(const pcsr_drop_t *d)
{
    Drop r = {};
    r.keep = 1.0f;
    if (!d || !(d->p > 0.0)) return r;
    r.seed[0] = (uint32_t)d->seed, r.seed[1] = (uint32_t)(d->seed >> 32);
    r.offset[0] = (uint32_t)d->offset, r.offset[1] = (uint32_t)(d->offset >> 32);
    r.state = d->state, r.used = d->used;
    r.threshold = (uint32_t)std::llrint(d->p * 65536.0); // ties to even, as Python's round
    r.keep = r.threshold < 65536 ? (float)(65536.0 / (65536 - r.threshold)) : 0.0f;
    return r;
}

struct DropKey {
    uint32_t k0, k1, o0, o1;
};
__device__ __forceinline__ DropKey key_of(const Drop &d)
{
    if (!d.state) return {d.seed[0], d.seed[1], d.offset[0], d.offset[1]};
    const uint64_t s = (uint64_t)d.state[0], o = (uint64_t)d.state[1]; // the same for all threads
    return {(uint32_t)s, (uint32_t)(s >> 32), (uint32_t)o, (uint32_t)(o >> 32)};
}
// by one thread of the launch
__device__ __forceinline__ void tell_key(const Drop &d, const DropKey &k)
{
    if (!d.used) return;
    d.used[0] = (int64_t)((uint64_t)k.k1 << 32 | k.k0);
    d.used[1] = (int64_t)((uint64_t)k.o1 << 32 | k.o0);
}

__device__ __forceinline__ void philox(const DropKey &key, uint32_t group, uint32_t row, uint32_t (&w)[4])
{
    uint32_t c0 = group, c1 = row, c2 = key.o0, c3 = key.o1, k0 = key.k0, k1 = key.k1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        // 0x96: exclusive or of three in one instruction
        c0 = __builtin_amdgcn_bitop3_b32((uint32_t)(b >> 32), c1, k0, 0x96), c1 = (uint32_t)b;
        c2 = __builtin_amdgcn_bitop3_b32((uint32_t)(a >> 32), c3, k1, 0x96), c3 = (uint32_t)a;
        k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
    }
    w[0] = c0, w[1] = c1, w[2] = c2, w[3] = c3;
}

// 8 columns from 8 group on, of a row: multiplied (TIMES) or dropped.  What is dropped is 0 whatever it was.
template <bool TIMES = true> __device__ __forceinline__ void drop8(const Drop &d, const DropKey &key, uint32_t group, uint32_t row, float (&x)[8])
{
    uint32_t w[4];
    philox(key, group, row, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
        x[i] = bits >= d.threshold ? TIMES ? x[i] * d.keep : x[i] : 0.0f;
    }
}

} // namespace
} // namespace pcsr
