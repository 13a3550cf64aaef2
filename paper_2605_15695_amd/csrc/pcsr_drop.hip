// Dropout of rows of features, with a residual that is added (see pcsr_train.h; pcsr_drop.h says what is dropped).
//
// y = r + f x, dx = f dy, f = 0 or 1 / (1 - p): one pass over the arrays either way, bound by memory.
#include <hip/hip_runtime.h>

#include "pcsr_drop.h"
#include "pcsr_num.h"

namespace pcsr {
namespace {

constexpr int kT = 256;

struct DropArgs {
    const void *x, *residual;
    void *out;
    int64_t x_stride, r_stride, cols;
    uint32_t first, groups, all; // first row, groups of 8 columns, their number in all rows of the launch
    uint32_t magic, shift;       // t / groups = t * magic >> shift for t below 2^31
    Drop drop;
};

// A thread takes 8 numbers of a row, what one call of the generator gives: nothing waits for anything but its own loads.
// 2,000,000 x 64 in fp32 with a residual 269 us (1.54 GB, 5.7 TB/s), without 173 (5.9); 250,000 x 512 in bf16 87 us (5.9 TB/s), vector units 58 % busy with the
// generator.  One row: 1.7 us of a launch of 4.5.
template <typename T, bool RESIDUAL> __global__ void __launch_bounds__(kT) dropout_kernel(DropArgs a)
{
    const uint32_t t = blockIdx.x * kT + threadIdx.x;
    const DropKey key = key_of(a.drop);
    if (t == 0 && a.first == 0) tell_key(a.drop, key);
    if (t >= a.all) return;
    const uint32_t r = (uint32_t)((uint64_t)t * a.magic >> a.shift), g = t - r * a.groups, row = a.first + r;
    const int64_t c = (int64_t)g * 8;
    const int m = a.cols - c < 8 ? (int)(a.cols - c) : 8;
    float x[8], y[8];
    load_upto<T, 8>(static_cast<const T *>(a.x) + (int64_t)row * a.x_stride + c, m, x);
    if (RESIDUAL) load_upto<T, 8>(static_cast<const T *>(a.residual) + (int64_t)row * a.r_stride + c, m, y);
    if (a.drop.threshold) drop8(a.drop, key, g, row, x);
    if (RESIDUAL)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] += y[i];
    store_upto<T, 8>(static_cast<T *>(a.out) + (int64_t)row * a.cols + c, m, x);
}

} // namespace
} // namespace pcsr

using namespace pcsr;

extern "C" int pcsr_dropout(int64_t rows, int64_t cols, int32_t type, const void *x, int64_t x_stride, const void *residual, int64_t r_stride,
                            const pcsr_drop_t *how, void *out, void *stream)
{
    if (rows < 0 || cols < 1 || !how || !(how->p >= 0.0 && how->p <= 1.0)) return PCSR_E_INVALID_ARG;
    if (type < PCSR_F32 || type > PCSR_F16) return PCSR_E_UNSUPPORTED;
    if (rows >= int64_t(1) << 32 || cols >= int64_t(1) << 31) return PCSR_E_TOO_LARGE;
    if (rows == 0) return PCSR_OK;
    if (!x || !out || x_stride < cols || (residual && r_stride < cols)) return PCSR_E_INVALID_ARG;
    DropArgs a = {x, residual, out, x_stride, r_stride, cols, 0, (uint32_t)((cols + 7) / 8), 0, 0, 0, drop_of(how)};
    uint32_t l = 0;
    while ((uint32_t(1) << l) < a.groups) ++l;
    // for t below 2^31 and 2^l >= groups the quotient is exact with m = ceil(2^(31 + l) / groups), which is below 2^32
    a.magic = (uint32_t)(((uint64_t(1) << (31 + l)) + a.groups - 1) / a.groups), a.shift = 31 + l;
    const int64_t most = ((int64_t(1) << 31) - kT) / a.groups;
    for (int64_t r = 0; r < rows; r += most) {
        a.first = (uint32_t)r;
        a.all = (uint32_t)((rows - r < most ? rows - r : most) * a.groups);
        const unsigned blocks = (a.all + kT - 1) / kT;
        const int rc = for_type(type, [&](auto z) {
            typedef decltype(z) T;
            if (residual) hipLaunchKernelGGL((dropout_kernel<T, true>), dim3(blocks), dim3(kT), 0, (hipStream_t)stream, a);
            else hipLaunchKernelGGL((dropout_kernel<T, false>), dim3(blocks), dim3(kT), 0, (hipStream_t)stream, a);
            return launched();
        });
        if (rc != PCSR_OK) return rc;
    }
    return PCSR_OK;
}
