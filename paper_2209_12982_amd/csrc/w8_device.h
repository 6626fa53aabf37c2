// Products of rows with 8-bit weights, on the device: y[r][c] = (sum_k x[r][k]
// w[c][k]) x_scale[r] w_scale[c] + bias[c].  Shared by the dense product and
// the experts' one, which differ in where a row comes from and goes to.
//
// Sums are exact in int32: k < 131072 of products of at most 2^14.  Their order
// is free, so parts of k may be added in any order with the same result.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mx4.h"
#include "wino_device.h"
#include "winof4.h"

namespace w8 {
using namespace mx4;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(16))) int i32x16;

struct Args {
    const int8_t *x, *w;
    const float *x_scales, *w_scales;
    const void* bias;       // dense: [n] in the type of y, or null
    void* y;
    int64_t x_stride, y_stride;
    int32_t m, n, k;        // m: rows of x (dense)
    int32_t* part;          // dense: sums of parts of k, [parts][m][n], or null
    int32_t steps;          // of k in a part
    int32_t* tail;          // sums of the last tiles' parts of k, or null
    // experts: routes in the order of their experts, where each expert's begin; x has a row for `share` routes
    const int32_t *order, *ends;
    int32_t experts, routes;
    winof4::FastDiv share;
    float* products;        // [routes][n] where they are added up with weights, or null
};

typedef u32x4 __attribute__((aligned(2))) Anywhere;      // 16 bytes that begin at any 16-bit number

constexpr int kMostParts = 8;           // of k, of the last tiles

__device__ const uint32_t kZeros[4] = {0, 0, 0, 0};     // what lies behind the end of k

// An expert's rows: the routes order[begin .. end), cut to the tensors.
__device__ inline void rows_of(const Args& a, int expert, int& begin, int& end) {
    begin = min(max(a.ends[expert], 0), a.routes);
    end = min(max(a.ends[expert + 1], begin), a.routes);
}

// Which row of x a route reads; routes out of range (which are not stored either) read row 0.
__device__ inline int64_t x_row(const Args& a, int route) {
    return (uint32_t)route < (uint32_t)a.routes ? winof4::fast_div((uint32_t)route, a.share) : 0;
}

// The result of a sum, the same bits in every kernel: the last step is kept apart from a conversion to fp16 after it, which
// the compiler would otherwise take together with it in some kernels (v_fma_mixlo_f16, one rounding instead of two).
__device__ inline float finish(int sum, float x_scale, float w_scale, float bias) {
    float y = __builtin_fmaf((float)sum * x_scale, w_scale, bias);
    asm("" : "+v"(y));
    return y;
}

// Whether a launch holds so many workgroups (of 512 threads; it counts threads in 32 bits).
inline bool launch_holds(int64_t groups) { return groups < 1 << 23; }

}  // namespace w8
