// w8_experts_matmul: each route's row of 8-bit codes times its expert's 8-bit weights, routes in the order of their
// experts; optionally the weighted sum of a token's routes.
#include <algorithm>

#include "w8_rows.h"
#include "w8_tiles.h"

namespace {
using namespace w8;

// out[t] = sum_j weights[t][j] products[t top + j], in the order of j; routes without an expert add nothing.  Memory bounds
// it: four columns a thread (2000 tokens, two routes each, 4096 outputs: 15 us for 27 with one, 5.5 TB/s of products that are
// in the last-level cache).
template <int TYPE> __global__ __launch_bounds__(256) void w8_combine_kernel(Args a, const int32_t* chosen, const float* weights, int top) {
    typedef typename Half<TYPE>::type T;
    typedef __attribute__((ext_vector_type(4), aligned(4))) float Row;      // rows may begin at any number
    typedef __attribute__((ext_vector_type(4), aligned(2))) T Out;
    int col = ((int)blockIdx.y * 256 + (int)threadIdx.x) * 4;
    const int64_t token = blockIdx.x;
    if (col >= a.n) return;
    col = max(min(col, a.n - 4), 0);        // the last four: two threads may have the same ones, and the same results
    const bool whole = a.n >= 4;
    // eight rows of products are asked for together, and those of routes without an expert dropped (one token with eight
    // routes, 2048 outputs: 3.2 us, one row after the other 4.5)
    f32x4 sum = {};
    for (int j0 = 0; j0 < top; j0 += 8) {
        f32x4 p[8] = {};
        float weight[8] = {};
        int expert[8] = {};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (j0 + j >= top) break;
            const int64_t route = token * top + j0 + j;
            const float* from = a.products + route * a.n + col;
            expert[j] = chosen[route];
            weight[j] = weights[route];
            if (whole)
                p[j] = *(const Row*)from;
            else
                for (int e = 0; e < a.n; ++e) p[j][e] = from[e];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (j0 + j < top && (uint32_t)expert[j] < (uint32_t)a.experts) sum[e] = __builtin_fmaf(weight[j], p[j][e], sum[e]);
    }
    T* to = (T*)a.y + token * a.y_stride + col;
    if (whole)
        *(Out*)to = Out{(T)sum[0], (T)sum[1], (T)sum[2], (T)sum[3]};
    else
        for (int e = 0; e < a.n; ++e) to[e] = (T)sum[e];
}

template <int TYPE, int NT, int V> void launch_rows(const Args& a, hipStream_t stream) {
    // Few routes: workgroups for as many experts as can have one, which then look for it (0.1 us), where that saves many: one
    // token to 8 of 256, 1024 x 2048: 6.5 us, with workgroups for all experts 10.7.
    const int n_tiles = (a.n + 16 * NT - 1) / (16 * NT);
    const bool few = 2 * a.routes <= a.experts && (a.experts - a.routes) * n_tiles >= 512;
    const dim3 grid((unsigned)n_tiles, (unsigned)(few ? a.routes : a.experts));
    hipLaunchKernelGGL((w8_rows_kernel<TYPE, NT, V, true>), grid, dim3(64 * V), 0, stream, a);
}
template <int TYPE, class S, bool FAR = false> void launch_tiles(const Args& a, hipStream_t stream) {
    const int n_tiles = (a.n + S::kOuts - 1) / S::kOuts;
    // whole tiles of the rows, and one more for each expert's last
    const int m_tiles = a.routes / S::kRows + std::min(a.experts, a.routes);
    const dim3 grid(workgroups<S>(a, (int64_t)n_tiles * m_tiles));
    hipLaunchKernelGGL((w8_tiles_kernel<TYPE, S, true, FAR>), grid, dim3(S::kThreads), 0, stream, a, n_tiles, m_tiles);
    launch_tail<TYPE, S, true>(a, n_tiles, m_tiles, stream);
}

// The shortest estimate for routes that are spread evenly: the host does not know how they are.  Uneven ones mostly take less, as
// fewer experts are read (us; even, and as uneven as can be): 1000 tokens to one of 64 74, 16; 128 to 8 of 64 74, 16.  They take more
// where tiles need another round: 512 to 2 of 8 16, 25; 4096 to 8 of 64 with a tenth of the routes on one 259 for 243.  An expert
// with r rows on average has r / rows tiles and half a one more, or one.  Measured (us): 4096 tokens to 8 of 64 experts, n 2816, k 2048:
// 256 x 256 249, two 128 x 128 297, 128 x 256 337; 2000 to 2 of 8, 4096 x 8192: 187 with the last tiles in parts and 220
// without, 210, 218; 256 to 6 of 64: 102, 87, 91, 64 x 64 79; 32 to 6 of 64: rows of 32 outputs 60, 64 x 64 67; one to 2 of 8,
// 1024 x 2048: rows of 16 outputs 4.5.
Kernel choose(int64_t routes, int64_t experts, int64_t n, int64_t k, bool tail) {
    const int64_t used = std::min(routes, experts);
    const double each = (double)routes / (double)used;
    Kernel best = kTile256x256;
    double least = 0;
    for (int i = 0; i < kKernels; ++i) {
        const Form& f = kForms[i];
        if (i >= kRows16 && each > 16) break;
        if (i < kRows16 && !launch_holds((routes / f.rows + used) * ((n + f.outs - 1) / f.outs))) continue;
        const double tiles = each > f.rows ? each / f.rows + 0.5 : 1;
        const int64_t all = (int64_t)(tiles * (double)(used * ((n + f.outs - 1) / f.outs)));
        // uneven routes have more tiles than that, and one more than 256 would cost these a second round
        if (f.pair == 0 && all > 200) continue;
        double t = estimate((Kernel)i, all, k, used * n * k, (int64_t)std::min(each, 16.0));
        // tiles whose last ones are cut in parts of k take a part of the last round, and their join 20 us
        if (i == kTile256x256 && tail)
            t = std::min(t, std::max((f.start + f.step * (1 + f.full) * (double)k / 1024) * ((double)all / 256 + 0.1) + 20,
                                     (double)(used * n * k) / 5.2e6));
        if (least == 0 || t < least) least = t, best = (Kernel)i;
    }
    return best;
}

template <int TYPE> void pick(const Args& a, int64_t x_rows, hipStream_t stream) {
    const Kernel kernel = choose(a.routes, a.experts, a.n, a.k, a.tail != nullptr);
    if (kernel < kRows16 && far(x_rows, a.x_stride, a.k)) return launch_tiles<TYPE, Tile64x128, true>(a, stream);
    switch (kernel) {
        case kTile256x256: return launch_tiles<TYPE, Tile256x256>(a, stream);
        case kTile128x256: return launch_tiles<TYPE, Tile128x256>(a, stream);
        case kTile128x128: return launch_tiles<TYPE, Tile128x128>(a, stream);
        case kPair128x128: return launch_tiles<TYPE, Pair128x128>(a, stream);
        case kTile64x128: return launch_tiles<TYPE, Tile64x128>(a, stream);
        case kTile64x64: return launch_tiles<TYPE, Tile64x64>(a, stream);
        case kTile32x32: return launch_tiles<TYPE, Tile32x32>(a, stream);
        case kShared64x128: return launch_tiles<TYPE, Shared64x128>(a, stream);
        case kShared64x64: return launch_tiles<TYPE, Shared64x64>(a, stream);
        case kShared64x32: return launch_tiles<TYPE, Shared64x32>(a, stream);
        case kRows16: return launch_rows<TYPE, 1, 16>(a, stream);
        case kRows16Few: return launch_rows<TYPE, 1, 8>(a, stream);
        default: return launch_rows<TYPE, 2, 4>(a, stream);
    }
}

template <int TYPE> void combine(const Args& a, const int32_t* chosen, const float* weights, int top, hipStream_t stream) {
    const dim3 grid((unsigned)(a.routes / top), (unsigned)((a.n + 1023) / 1024));
    hipLaunchKernelGGL((w8_combine_kernel<TYPE>), grid, dim3(256), 0, stream, a, chosen, weights, top);
}

size_t product_bytes(int64_t routes, int64_t n) { return ((size_t)routes * n * sizeof(float) + 15) / 16 * 16; }
// Results for which tiles of 256 x 256, the last ones cut in parts of k, may be the fastest.
bool many(int64_t routes, int64_t n) { return routes * n >= 1 << 22; }

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }

}  // namespace

extern "C" size_t w8_experts_matmul_workspace_bytes(int32_t routes, int32_t n, int32_t combine) {
    if (routes < 1 || n < 1) return 0;
    return (combine ? product_bytes(routes, n) : 0) + (many(routes, n) ? kTailBytes : 0);
}

extern "C" wino_status w8_experts_matmul(const int8_t* x, int64_t x_stride, const float* x_scales, int32_t x_rows, const int8_t* w,
                                         const float* w_scales, const int32_t* order, const int32_t* ends, int32_t routes,
                                         int32_t experts, const int32_t* chosen, const float* weights, int32_t top, void* y,
                                         int64_t y_stride, int32_t n, int32_t k, wino_float_type type, void* workspace,
                                         size_t workspace_bytes, hipStream_t stream) {
    if (type != WINO_BF16 && type != WINO_FP16) return WINO_EINVAL;
    if (x_rows < 0 || routes < 0 || experts < 1 || n < 0 || k < 0 || k % 16 != 0) return WINO_EINVAL;
    if ((weights != nullptr) != (chosen != nullptr) || (weights && (top < 1 || routes % top != 0))) return WINO_EINVAL;
    if (routes == 0 || n == 0) return WINO_OK;
    if (x_rows < 1 || routes % x_rows != 0) return WINO_EINVAL;
    if (!y || !x_scales || !w_scales || !order || !ends || (k > 0 && (!x || !w))) return WINO_EINVAL;
    const int32_t y_rows = weights ? routes / top : routes;
    if ((x_rows > 1 && x_stride < k) || (y_rows > 1 && y_stride < n)) return WINO_EINVAL;
    if (routes > 1 << 22 || experts > 1024 || n > 1 << 20 || k >= 1 << 17) return WINO_EUNSUPPORTED;
    if (!aligned16(x) || !aligned16(w) || !aligned16(workspace) || !aligned4(x_scales) || !aligned4(w_scales) || !aligned4(order) ||
        !aligned4(ends) || !aligned4(chosen) || !aligned4(weights) || ((uintptr_t)y & 1) || (k > 0 && x_rows > 1 && (x_stride & 15)))
        return WINO_EUNSUPPORTED;
    if (!launch_holds((int64_t)(routes / 128 + experts) * ((n + 127) / 128)) || !launch_holds((int64_t)((n + 15) / 16) * experts) ||
        (far(x_rows, x_stride, k) && !launch_holds((int64_t)(routes / 128 + experts) * ((n + 63) / 64))) ||
        (weights && !launch_holds((int64_t)y_rows * ((n + 255) / 256))))
        return WINO_EUNSUPPORTED;
    Args a = {};
    a.x = x, a.w = w, a.x_scales = x_scales, a.w_scales = w_scales, a.y = y, a.x_stride = x_stride, a.y_stride = y_stride;
    a.n = n, a.k = k, a.order = order, a.ends = ends, a.experts = experts, a.routes = routes;
    a.share = winof4::make_fastdiv((uint32_t)(routes / x_rows));
    const size_t products = weights ? product_bytes(routes, n) : 0;
    if (weights) {
        if (!workspace || workspace_bytes < (size_t)routes * n * sizeof(float)) return WINO_EINVAL;
        a.products = (float*)workspace;
    }
    // Shorter sums gain less than the join of their parts takes: 3000 tokens to 4 of 16, 2048 x 4096, 121 us without parts and
    // 124 with them.
    if (many(routes, n) && k > 4096 && workspace && workspace_bytes >= products + kTailBytes) a.tail = (int32_t*)((char*)workspace + products);
    type == WINO_BF16 ? pick<WINO_BF16>(a, x_rows, stream) : pick<WINO_FP16>(a, x_rows, stream);
    if (weights) {
        if (hipGetLastError() != hipSuccess) return WINO_EHIP;      // asking for an error clears it
        type == WINO_BF16 ? combine<WINO_BF16>(a, chosen, weights, top, stream) : combine<WINO_FP16>(a, chosen, weights, top, stream);
    }
    return hipGetLastError() == hipSuccess ? WINO_OK : WINO_EHIP;
}
