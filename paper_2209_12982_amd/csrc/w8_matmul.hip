// w8_matmul: rows of 8-bit codes times a matrix of 8-bit weights, with a scale for each row and each output.
#include <algorithm>

#include "w8_rows.h"
#include "w8_tiles.h"

namespace {
using namespace w8;

// Adds up the parts of k (whole numbers: any order gives the same) and finishes the outputs.
template <int TYPE> __global__ __launch_bounds__(256) void w8_join_kernel(Args a, int parts) {
    typedef typename Half<TYPE>::type T;
    const int64_t o = (int64_t)blockIdx.x * 256 + threadIdx.x, all = (int64_t)a.m * a.n;
    if (o >= all) return;
    int sum = 0;
    for (int p = 0; p < parts; ++p) sum += a.part[p * all + o];
    const int row = (int)(o / a.n), col = (int)(o - (int64_t)row * a.n);
    ((T*)a.y)[row * a.y_stride + col] =
        (T)finish(sum, a.x_scales[row], a.w_scales[col], a.bias ? (float)((const T*)a.bias)[col] : 0.f);
}

template <int TYPE, int MT, int NT> void launch_rows(const Args& a, hipStream_t stream) {
    const dim3 grid((unsigned)((a.n + 16 * NT - 1) / (16 * NT)), (unsigned)((a.m + 16 * MT - 1) / (16 * MT)), 1);
    hipLaunchKernelGGL((w8_rows_kernel<TYPE, MT, NT, 8, false>), grid, dim3(512), 0, stream, a);
}
template <int TYPE, class S> void launch_tiles(const Args& a, hipStream_t stream) {
    const int n_tiles = (a.n + S::kOuts - 1) / S::kOuts, m_tiles = (a.m + S::kRows - 1) / S::kRows;
    const unsigned grid = (unsigned)((n_tiles * (int64_t)m_tiles + 7) / 8 * 8);
    hipLaunchKernelGGL((w8_tiles_kernel<TYPE, S, false>), dim3(grid), dim3(S::kThreads), 0, stream, a, n_tiles, m_tiles);
}

template <int TYPE> void pick(Args a, hipStream_t stream) {
    a.part = nullptr;
    a.steps = 1 << 20;
    if (a.m <= 64) {
        const int mt = (a.m + 15) / 16;
        mt == 1 ? launch_rows<TYPE, 1, 1>(a, stream)
                : mt == 2 ? launch_rows<TYPE, 2, 2>(a, stream)
                          : mt == 3 ? launch_rows<TYPE, 3, 4>(a, stream) : launch_rows<TYPE, 4, 4>(a, stream);
    } else if ((int64_t)a.m * a.n >= 200 * 256 * 256) {
        launch_tiles<TYPE, Tile<4, 2, 2, 4, 128, 2>>(a, stream);
    } else {
        launch_tiles<TYPE, Tile<2, 1, 2, 4, 128, 2>>(a, stream);
    }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }

}  // namespace

extern "C" size_t w8_matmul_workspace_bytes(int32_t m, int32_t n, int32_t k) {
    (void)m, (void)n, (void)k;
    return 0;
}

extern "C" wino_status w8_matmul(const int8_t* x, int64_t x_stride, const float* x_scales, const int8_t* w, const float* w_scales,
                                 const void* bias, void* y, int64_t y_stride, int32_t m, int32_t n, int32_t k,
                                 wino_float_type type, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (type != WINO_BF16 && type != WINO_FP16) return WINO_EINVAL;
    if (m < 0 || n < 0 || k < 0 || k % 16 != 0) return WINO_EINVAL;
    if (m == 0 || n == 0) return WINO_OK;
    if (!y || !x_scales || !w_scales || (k > 0 && (!x || !w))) return WINO_EINVAL;
    if (m > 1 && (x_stride < k || y_stride < n)) return WINO_EINVAL;
    if (m > 1 << 20 || n > 1 << 24 || k >= 1 << 17) return WINO_EUNSUPPORTED;
    if (!aligned16(x) || !aligned16(w) || !aligned16(workspace) || !aligned4(x_scales) || !aligned4(w_scales) ||
        ((uintptr_t)y & 1) || ((uintptr_t)bias & 1) || (k > 0 && m > 1 && (x_stride & 15)))
        return WINO_EUNSUPPORTED;
    if (!launch_holds((int64_t)((m + 127) / 128) * ((n + 127) / 128))) return WINO_EUNSUPPORTED;
    Args a = {};
    a.x = x, a.w = w, a.x_scales = x_scales, a.w_scales = w_scales, a.bias = bias, a.y = y;
    a.x_stride = x_stride, a.y_stride = y_stride, a.m = m, a.n = n, a.k = k, a.part = (int32_t*)workspace;
    type == WINO_BF16 ? pick<WINO_BF16>(a, stream) : pick<WINO_FP16>(a, stream);
    return hipGetLastError() == hipSuccess ? WINO_OK : WINO_EHIP;
}
