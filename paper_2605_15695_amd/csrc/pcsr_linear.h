// The calls of linear layers for one type of numbers, their arguments checked (pcsr_linear.hip).
#pragma once
#include <hip/hip_runtime.h>

#include "pcsr_num.h"

namespace pcsr {

template <typename T> struct LinearOf {
    static int64_t workspace(const pcsr_linear_t &a, bool backward);
    static int forward(const pcsr_linear_t &a, void *y, void *slope, void *ws, hipStream_t stream);
    static int backward(const pcsr_linear_t &a, const void *slope, const void *dy, int64_t dy_stride, void *dx, void *dw, void *db, void *ws, hipStream_t stream);
    static void uses(const pcsr_linear_t &a, const void *dy, int64_t dy_stride, int64_t (&ends)[4][2]); // pcsr_linear_uses
};

} // namespace pcsr
