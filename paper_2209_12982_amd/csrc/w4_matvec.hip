// y = x W^T + b with W in the 4-bit format (mx4.h).
#include <hip/hip_runtime.h>

#include "mx4.h"
#include "winof4.h"

namespace {
using namespace mx4;

struct MatvecArgs {
    const void* x;
    const uint8_t* codes;
    const uint8_t* scales;
    const void* bias;
    void* y;
    int64_t x_stride, y_stride;
    int32_t m, n, k;
};

// One wave per output row of W and row of x: lanes take groups of 32 in turn.
template <int TYPE>
__global__ __launch_bounds__(64) void w4_matvec_kernel(MatvecArgs a) {
    typedef typename Half<TYPE>::type T;
    const int64_t row = blockIdx.x;
    const int32_t tok = blockIdx.y;
    const int groups = a.k / kGroup;
    const T* x = (const T*)a.x + (int64_t)tok * a.x_stride;
    float acc = 0.f;
    for (int g = threadIdx.x; g < groups; g += 64) {
        const uint8_t* c = a.codes + (row * groups + g) * 16;
        float part = 0.f;
        for (int i = 0; i < 16; ++i) {
            part += code_value(c[i] & 15u) * (float)x[g * kGroup + 2 * i];
            part += code_value(c[i] >> 4) * (float)x[g * kGroup + 2 * i + 1];
        }
        acc += part * scale_value(a.scales[row * groups + g]);
    }
    for (int o = 32; o; o >>= 1) acc += __shfl_xor(acc, o);
    if (threadIdx.x == 0) {
        if (a.bias) acc += (float)((const T*)a.bias)[row];
        ((T*)a.y)[(int64_t)tok * a.y_stride + row] = (T)acc;
    }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace

extern "C" size_t w4_matvec_workspace_bytes(int32_t m, int32_t n, int32_t k) {
    (void)m;
    (void)n;
    (void)k;
    return 0;
}

extern "C" wino_status w4_matvec(const void* x, int64_t x_stride, const uint8_t* codes, const uint8_t* scales,
                                 const void* bias, void* y, int64_t y_stride, int32_t m, int32_t n, int32_t k,
                                 wino_float_type type, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    (void)workspace;
    (void)workspace_bytes;
    if (type != WINO_BF16 && type != WINO_FP16) return WINO_EINVAL;
    if (m < 0 || n < 0 || k < 0 || k % kGroup != 0) return WINO_EINVAL;
    if (m == 0 || n == 0) return WINO_OK;
    if (!y || (k > 0 && (!x || !codes || !scales))) return WINO_EINVAL;
    if (m > 1 && (x_stride < k || y_stride < n)) return WINO_EINVAL;
    if (m > 65535 || n > (1 << 24) || k > (1 << 20)) return WINO_EUNSUPPORTED;
    if (!aligned16(x) || !aligned16(codes) || (k > 0 && m > 1 && (x_stride & 7))) return WINO_EUNSUPPORTED;
    MatvecArgs a = {x, codes, scales, bias, y, x_stride, y_stride, m, n, k};
    const dim3 grid((unsigned)n, (unsigned)m);
    if (type == WINO_BF16)
        hipLaunchKernelGGL(w4_matvec_kernel<WINO_BF16>, grid, dim3(64), 0, stream, a);
    else
        hipLaunchKernelGGL(w4_matvec_kernel<WINO_FP16>, grid, dim3(64), 0, stream, a);
    return hipGetLastError() == hipSuccess ? WINO_OK : WINO_EHIP;
}
