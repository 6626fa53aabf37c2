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

// Parts of k in whole stages of BK.
int share_out(Args& a, int parts, int bk) {
    const int stages = (a.k + bk - 1) / bk;
    a.steps = (stages + parts - 1) / parts;
    parts = a.steps > 0 ? (stages + a.steps - 1) / a.steps : 1;
    if (parts <= 1) a.part = nullptr;
    return parts;
}
template <int TYPE, int NT, int V> void launch_rows(const Args& a, hipStream_t stream) {
    const dim3 grid((unsigned)((a.n + 16 * NT - 1) / (16 * NT)), (unsigned)((a.m + 15) / 16));
    hipLaunchKernelGGL((w8_rows_kernel<TYPE, NT, V, false>), grid, dim3(64 * V), 0, stream, a);
}
template <int TYPE, class S, bool FAR = false> void launch_tiles(Args a, int parts, hipStream_t stream) {
    parts = share_out(a, parts, S::BK);
    const int n_tiles = (a.n + S::kOuts - 1) / S::kOuts, m_tiles = (a.m + S::kRows - 1) / S::kRows;
    const dim3 grid(workgroups<S>(a, (int64_t)n_tiles * m_tiles), (unsigned)parts);
    hipLaunchKernelGGL((w8_tiles_kernel<TYPE, S, false, FAR>), grid, dim3(S::kThreads), 0, stream, a, n_tiles, m_tiles);
    launch_tail<TYPE, S, false>(a, n_tiles, m_tiles, stream);
    if (parts > 1)
        hipLaunchKernelGGL((w8_join_kernel<TYPE>), dim3((unsigned)(((int64_t)a.m * a.n + 255) / 256)), dim3(256), 0, stream, a, parts);
}

// Which kernel takes a call and in how many parts of k: the shortest estimate.  Parts are joined by a second launch, which
// pays where few outputs have long sums (8 rows by 764 x 15824: 9.3 us in 8 parts, 12.7 whole; 515 rows by 1024 x 16384 24
// in 2, 32 whole); each is 1024 of k at least, and their sums 16 MiB at most.
// The kernels for few rows are looked at for up to 256 of them, sixteen a workgroup (of 36 calls of 33 to 64 rows, 84 of 65 to
// 128 and 40 of 129 to 256 17, 38 and 15 take them, and on average a call is 12, 10 and 11% shorter than with tiles for all).
constexpr int kMostFew = 256;
struct Cut {
    Kernel kernel;
    int parts;
};
Cut cut(int64_t m, int64_t n, int64_t k) {
    Cut best{kTile256x256, 1};
    double least = 0;
    for (int i = 0; i < kKernels; ++i) {
        if (i >= kRows16 && m > kMostFew) break;
        const Form& f = kForms[i];
        const int64_t tiles = (n + f.outs - 1) / f.outs * ((m + f.rows - 1) / f.rows);
        if (!launch_holds(tiles)) continue;
        for (const int parts : {1, 2, 4, 8, 16}) {
            if (parts > 1 && (i >= kRows16 || k < 1024 * parts || parts * m * n > 1 << 22)) break;
            if (f.pair == 0 && tiles * parts > 256) break;
            const double join = parts > 1 ? 1.95 + 0.17 * parts + 1.3e-6 * (double)(parts * m * n) : 0;
            double t = estimate((Kernel)i, tiles * parts, k / parts, n * k, m) + join;
            if (i == kTile256x256 && parts == 1) t -= std::max(tail_gain(tiles, k), 0.0);
            if (least == 0 || t < least) least = t, best = Cut{(Kernel)i, parts};
        }
    }
    return best;
}

bool beyond(int64_t m, int64_t n, int64_t k) {
    return m > 1 << 20 || n > 1 << 24 || k >= 1 << 17 || !launch_holds((m + 127) / 128 * ((n + 127) / 128));
}

size_t part_bytes(const Cut& c, int64_t m, int64_t n) { return c.parts > 1 ? (size_t)(c.parts * m * n) * sizeof(int32_t) : 0; }
bool cuts_tail(const Cut& c, int64_t m, int64_t n, int64_t k) {
    return c.kernel == kTile256x256 && c.parts == 1 && tail_gain((m + 255) / 256 * ((n + 255) / 256), k) > 0;
}

// Rows of x too far apart for the offsets of a kernel of tiles: Tile64x128 takes them, which has some for that.
bool far_rows(const Cut& c, int64_t m, int64_t x_stride, int64_t k) {
    return c.kernel < kRows16 && far(std::min<int64_t>(kForms[c.kernel].rows, m), x_stride, k);
}

template <int TYPE> void pick(Args a, const Cut& c, size_t bytes, hipStream_t stream) {
    if (far_rows(c, a.m, a.x_stride, a.k)) {
        a.part = nullptr;
        return launch_tiles<TYPE, Tile64x128, true>(a, 1, stream);
    }
    const int parts = a.part && bytes >= part_bytes(c, a.m, a.n) ? c.parts : 1;
    if (cuts_tail(c, a.m, a.n, a.k) && bytes >= kTailBytes) a.tail = a.part;
    switch (c.kernel) {
        case kTile256x256: return launch_tiles<TYPE, Tile256x256>(a, parts, stream);
        case kTile128x256: return launch_tiles<TYPE, Tile128x256>(a, parts, stream);
        case kTile128x128: return launch_tiles<TYPE, Tile128x128>(a, parts, stream);
        case kPair128x128: return launch_tiles<TYPE, Pair128x128>(a, parts, stream);
        case kTile64x128: return launch_tiles<TYPE, Tile64x128>(a, parts, stream);
        case kTile64x64: return launch_tiles<TYPE, Tile64x64>(a, parts, stream);
        case kTile32x32: return launch_tiles<TYPE, Tile32x32>(a, parts, stream);
        case kShared64x128: return launch_tiles<TYPE, Shared64x128>(a, parts, stream);
        case kShared64x64: return launch_tiles<TYPE, Shared64x64>(a, parts, stream);
        case kShared64x32: return launch_tiles<TYPE, Shared64x32>(a, parts, stream);
        case kRows16: return launch_rows<TYPE, 1, 16>(a, stream);
        case kRows16Few: return launch_rows<TYPE, 1, 8>(a, stream);
        default: return launch_rows<TYPE, 2, 4>(a, stream);
    }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }

}  // namespace

extern "C" size_t w8_matmul_workspace_bytes(int32_t m, int32_t n, int32_t k) {
    if (m < 1 || n < 1 || k < 1 || beyond(m, n, k)) return 0;
    const Cut c = cut(m, n, k);
    return cuts_tail(c, m, n, k) ? kTailBytes : part_bytes(c, m, n);
}

extern "C" wino_status w8_matmul(const int8_t* x, int64_t x_stride, const float* x_scales, const int8_t* w, const float* w_scales,
                                 const void* bias, void* y, int64_t y_stride, int32_t m, int32_t n, int32_t k,
                                 wino_float_type type, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (type != WINO_BF16 && type != WINO_FP16) return WINO_EINVAL;
    if (m < 0 || n < 0 || k < 0 || k % 16 != 0) return WINO_EINVAL;
    if (m == 0 || n == 0) return WINO_OK;
    if (!y || !x_scales || !w_scales || (k > 0 && (!x || !w))) return WINO_EINVAL;
    if (m > 1 && (x_stride < k || y_stride < n)) return WINO_EINVAL;
    if (beyond(m, n, k)) return WINO_EUNSUPPORTED;
    if (!aligned16(x) || !aligned16(w) || !aligned16(workspace) || !aligned4(x_scales) || !aligned4(w_scales) ||
        ((uintptr_t)y & 1) || ((uintptr_t)bias & 1) || (k > 0 && m > 1 && (x_stride & 15)))
        return WINO_EUNSUPPORTED;
    const Cut c = cut(m, n, k);
    if (far_rows(c, m, x_stride, k) && !launch_holds((int64_t)((m + 127) / 128) * ((n + 63) / 64))) return WINO_EUNSUPPORTED;
    Args a = {};
    a.x = x, a.w = w, a.x_scales = x_scales, a.w_scales = w_scales, a.bias = bias, a.y = y;
    a.x_stride = x_stride, a.y_stride = y_stride, a.m = m, a.n = n, a.k = k, a.part = (int32_t*)workspace;
    type == WINO_BF16 ? pick<WINO_BF16>(a, c, workspace_bytes, stream) : pick<WINO_FP16>(a, c, workspace_bytes, stream);
    return hipGetLastError() == hipSuccess ? WINO_OK : WINO_EHIP;
}
