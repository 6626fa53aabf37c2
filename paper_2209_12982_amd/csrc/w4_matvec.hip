// y = x W^T + b for a few rows x, with W in the 4-bit format (mx4.h).
//
// The bytes of W bound it: 17/32 of a byte a weight, each read once.  A wave
// takes 16 rows of W (times R) and 128 of k a step: a lane loads 16 bytes of one
// row, a whole group with its scale, so that a row's four lanes read one cache
// line; a 4 x 4 exchange between the quarters of the wave then turns the groups
// around, so that x is read in whole lines as well.  The converter makes two
// codes an instruction into 16-bit numbers, exactly, and the matrix cores
// multiply them with x, whose up to 16 rows cost as much as one; a sum is
// fp32 throughout.  With x in fp16 the weights become fp16 too, as long as a
// wave's scales allow it (most sets do); else the wave begins again with x split
// into two bf16 numbers, which costs a second product.  The waves of a workgroup
// share out k and are joined in LDS, workgroups that share out k are joined
// by a second kernel, both in a fixed order.
//
// Measured (bf16): 16384 x 4096, 35.7 MB: 10.2 us for one row of x (3.5 TB/s,
// of 4.9 that a large copy reaches), 17.6 us for 16, where the reads of x from
// the L2 count as much as those of W.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

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
    int32_t steps;          // of 128 of k, for each part
    float* part;            // [parts][m][n], or null
};

// R tiles of 16 rows of W, N tiles of 16 rows of x, V waves that share out k, D
// steps of codes on their way.  X: x lies in LDS; else its pieces come with the
// codes.  blockIdx.z takes `steps` steps of k; where there are several, their
// sums go to a.part and w4_matvec_join adds them up.
template <int TYPE, int R, int N, int V, int D, bool X>
__global__ __launch_bounds__(64 * V) void w4_matvec_kernel(MatvecArgs a) {
    typedef typename Half<TYPE>::type T;
    typedef T T8 __attribute__((ext_vector_type(8)));
    __shared__ float join[V][R * 16][N * 16 + 1];
    extern __shared__ __attribute__((aligned(16))) uint8_t x_lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int row0 = blockIdx.x * (16 * R), tok0 = blockIdx.y * (16 * N);
    const int groups = a.k / kGroup;
    const int begin = blockIdx.z * a.steps * 4, end = min(groups, begin + a.steps * 4);

    const uint8_t* codes[R];
    const uint8_t* scales[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int64_t row = min(row0 + 16 * i + r, a.n - 1);    // rows past the end are computed and not stored
        codes[i] = a.codes + (row * groups + g) * 16;
        scales[i] = a.scales + row * groups;
    }
    // x of this lane: row r of each tile (the last one again past the end), eighth g of a group
    const T* x[N];
    const uint8_t* xl[N];
    const int x_row = (end - begin) * kGroup * 2 + 16;          // bytes of a row in LDS: 16 rows in 16 columns of the banks
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int tok = min(16 * j + r, a.m - 1 - tok0);
        x[j] = (const T*)a.x + (int64_t)(tok0 + tok) * a.x_stride + 8 * g;
        xl[j] = x_lds + tok * x_row - begin * kGroup * 2 + 16 * g;
    }

    // A step's four groups.  Codes arrive with group g in quarter g of the wave, which reads whole cache lines; the
    // products take group e with its eighths spread over the quarters, which reads x in whole lines too.
    struct Step {
        u32x4 w[R];
        uint32_t s[R];
        T8 x[X ? 1 : N][4];
    };
    auto load = [&](int first, Step& t) {
        if (first + 4 <= end) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                t.w[i] = *(const u32x4*)(codes[i] + (int64_t)first * 16);
                __builtin_memcpy(&t.s[i], scales[i] + first, 4);
            }
            if constexpr (!X) {
#pragma unroll
                for (int j = 0; j < N; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) t.x[j][e] = *(const T8*)(x[j] + (first + e) * kGroup);
            }
        } else if (first < end) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                t.w[i] = first + g < end ? *(const u32x4*)(codes[i] + (int64_t)first * 16) : u32x4{0, 0, 0, 0};
                t.s[i] = 0x7f7f7f7f;
                for (int e = 0; e < 3; ++e)
                    if (first + e < end) t.s[i] = (t.s[i] & ~(255u << (8 * e))) | (uint32_t)scales[i][first + e] << (8 * e);
            }
            if constexpr (!X) {
#pragma unroll
                for (int j = 0; j < N; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        t.x[j][e] = first + e < end ? *(const T8*)(x[j] + (first + e) * kGroup) : T8{};
            }
        }
    };

    f32x4 acc[R][N];                                            // lane: rows 4 g + e of W, row r of x
    uint32_t most = 0x007f007f, least = 0x007f007f;             // of the scales, two at a time
    // `split`: x in fp16 as two bf16 numbers (8 + 3 bits, exact).  Else the products are fp16 ones, which hold W
    // exactly as long as its scales lie between 2^-23 and 2^13.
    auto compute = [&](int first, const Step& t, auto split) {
        constexpr bool kSplit = decltype(split)::value, kF16 = TYPE == WINO_FP16 && !kSplit;
        constexpr int kParts = kSplit ? 2 : 1;
        uint32_t w[R][4];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const auto s02 = __builtin_amdgcn_permlane32_swap(t.w[i][0], t.w[i][2], false, false);
            const auto s13 = __builtin_amdgcn_permlane32_swap(t.w[i][1], t.w[i][3], false, false);
            const auto s01 = __builtin_amdgcn_permlane16_swap(s02[0], s13[0], false, false);
            const auto s23 = __builtin_amdgcn_permlane16_swap(s02[1], s13[1], false, false);
            w[i][0] = s01[0], w[i][1] = s01[1], w[i][2] = s23[0], w[i][3] = s23[1];
            if constexpr (kF16) {
                typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
                const u16x2 even = __builtin_bit_cast(u16x2, t.s[i] & 0x00ff00ffu);
                const u16x2 odd = __builtin_bit_cast(u16x2, (t.s[i] >> 8) & 0x00ff00ffu);
                most = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(
                           __builtin_bit_cast(u16x2, most), __builtin_elementwise_max(even, odd)));
                least = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(
                            __builtin_bit_cast(u16x2, least), __builtin_elementwise_min(even, odd)));
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            T8 v[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                if constexpr (X)
                    v[j] = first + e < end ? *(const T8*)(xl[j] + (first + e) * (kGroup * 2)) : T8{};
                else
                    v[j] = t.x[j][e];
            }
            bf16x8 b[kParts][N];
            if constexpr (!kF16) {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    if constexpr (TYPE == WINO_BF16) {
                        b[0][j] = v[j];
                    } else {
#pragma unroll
                        for (int d = 0; d < 8; ++d) {
                            const float f = (float)v[j][d];
                            const __bf16 hi = (__bf16)f;
                            b[0][j][d] = hi;
                            b[kParts - 1][j][d] = (__bf16)(f - (float)hi);
                        }
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const float s = scale_bits((t.s[i] >> (8 * e)) & 255u);
                if constexpr (kF16) {
                    const f16x8 u = decode8_f16(w[i][e], s);
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(u, v[j], acc[i][j], 0, 0, 0);
                } else {
                    const bf16x8 u = decode8(w[i][e], s);
#pragma unroll
                    for (int p = 0; p < kParts; ++p)
#pragma unroll
                        for (int j = 0; j < N; ++j)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(u, b[p][j], acc[i][j], 0, 0, 0);
                }
            }
        }
    };
    // the wave's steps: every V-th
    const int mine = max(0, (end - begin - wave * 4 + 4 * V - 1) / (4 * V));
    auto at = [&](int i) { return begin + (wave + V * i) * 4; };
    auto sweep = [&](Step (&t)[D], auto split) {
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int i = 0; i < mine; i += D) {
#pragma unroll
            for (int d = 0; d < D; ++d) {
                if (i + d < mine) {
                    compute(at(i + d), t[d], split);
                    if (i + d + D < mine) load(at(i + d + D), t[d]);
                }
            }
        }
    };
    Step t[D];
#pragma unroll
    for (int d = 0; d < D; ++d)
        if (d < mine) load(at(d), t[d]);
    if constexpr (X) {
        const int pieces = (end - begin) * 4, rows = min(16 * N, a.m - tok0);
        for (int i = threadIdx.x; i < pieces * rows; i += 64 * V) {
            const int tok = i / pieces, p = i - tok * pieces;
            *(T8*)(x_lds + tok * x_row + p * 16) =
                *(const T8*)((const T*)a.x + (int64_t)(tok0 + tok) * a.x_stride + begin * kGroup + p * 8);
        }
        __syncthreads();
    }
    sweep(t, std::false_type{});
    if constexpr (TYPE == WINO_FP16) {
        const uint32_t hi = max(most & 0xffffu, most >> 16), lo = min(least & 0xffffu, least >> 16);
        if (__any(hi > 140u || lo < 104u)) {
#pragma unroll
            for (int d = 0; d < D; ++d)
                if (d < mine) load(at(d), t[d]);
            sweep(t, std::true_type{});
        }
    }
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) join[wave][16 * i + 4 * g + e][16 * j + r] = acc[i][j][e];
    __syncthreads();
    for (int o = threadIdx.x; o < R * N * 256; o += 64 * V) {
        const int row = o % (R * 16), tok = o / (R * 16);
        if (row0 + row >= a.n || tok0 + tok >= a.m) continue;
        float sum = join[0][row][tok];
#pragma unroll
        for (int w = 1; w < V; ++w) sum += join[w][row][tok];
        if (a.part) {
            a.part[((int64_t)blockIdx.z * a.m + tok0 + tok) * a.n + row0 + row] = sum;
        } else {
            if (a.bias) sum += (float)((const T*)a.bias)[row0 + row];
            ((T*)a.y)[(int64_t)(tok0 + tok) * a.y_stride + row0 + row] = (T)sum;
        }
    }
}

// Adds up the parts of k, in their order.
template <int TYPE> __global__ __launch_bounds__(256) void w4_matvec_join(MatvecArgs a, int splits) {
    typedef typename Half<TYPE>::type T;
    const int row = blockIdx.x * 256 + threadIdx.x, tok = blockIdx.y;
    if (row >= a.n) return;
    const float* p = a.part + (int64_t)tok * a.n + row;
    float sum = p[0];
    for (int s = 1; s < splits; ++s) sum += p[(int64_t)s * a.m * a.n];
    if (a.bias) sum += (float)((const T*)a.bias)[row];
    ((T*)a.y)[(int64_t)tok * a.y_stride + row] = (T)sum;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

template <int TYPE, int R, int N, int V, int D, bool X> void launch(MatvecArgs a, int splits, hipStream_t stream) {
    const int steps = (a.k + 127) / 128;
    a.steps = (steps + splits - 1) / splits;
    splits = a.steps > 0 ? (steps + a.steps - 1) / a.steps : 1;
    if (splits <= 1) a.part = nullptr;
    const dim3 grid((unsigned)((a.n + 16 * R - 1) / (16 * R)), (unsigned)((a.m + 16 * N - 1) / (16 * N)), (unsigned)splits);
    const size_t lds = X ? (size_t)std::min(a.m, 16 * N) * (std::min(a.k, a.steps * 128) * 2 + 16) : 0;
    hipLaunchKernelGGL((w4_matvec_kernel<TYPE, R, N, V, D, X>), grid, dim3(64 * V), lds, stream, a);
    if (splits > 1)
        hipLaunchKernelGGL((w4_matvec_join<TYPE>), dim3((unsigned)((a.n + 255) / 256), (unsigned)a.m), dim3(256), 0, stream,
                           a, splits);
}

// How a call is cut: 16 rows of W a workgroup (times `r`), k in `splits` parts, x in LDS or beside the codes.
struct Cut {
    int r, splits;
    bool x;
    int waves = 8;
};

// Few workgroups read x few times, many keep the device busy; a second launch, for the join, costs 3 us.  Measured (us,
// bf16, rows of x / n / k; r and parts):
//   x in LDS                    1/4096/4096: r1 4.7 (8 waves 5.1)   4/16384/4096: r2 13.0, r1 14.4   1/16384/4096: r2 11.3
//   x beside the codes          8/4096/4096: r1 6.5, r4 in 4 8.0    8/8192/8192: r2 15.3, r4 in 2 16.5
//                               16/16384/4096: r4 14.8, r2 17.6     16/2048/8192: r2 in 4 9.2, r4 in 8 9.9
//                               16/4096/16384: r4 in 4 18.4, r2 in 2 19.9, r1 24   1/1024/16384: r2 in 8 7.9, r1 10.9
//   more than 16 rows           32/4096/1024: r2 5.2, r4 6.4        32/2048/4096: r2 in 4 8.6, r4 in 4 9.8
//                               32/8192/8192: r4 in 2 22.2, r2 25.4 64/16384/4096: r4 28, r2 42
Cut cut(int64_t m, int64_t n, int64_t k) {
    // as many parts as make a workgroup for each of 256 compute units, no more, with 1024 of k in each at least
    auto parts = [&](int r) {
        const int64_t groups = (n + 16 * r - 1) / (16 * r);
        return (int)std::max<int64_t>(1, std::min<int64_t>(256 / groups, k / 1024));
    };
    if (m > 16) {
        const int r = n <= 2048 || (k < 2048 && n <= 8192) ? 2 : 4;
        return Cut{r, parts(r), false};
    }
    const bool fits = m * (2 * k + 16) <= 40960;
    if (n <= 2048 && k >= 12288) return Cut{2, parts(2), false};
    if (fits) return Cut{n <= 8192 ? 1 : 2, 1, true, n <= 4096 ? 16 : 8};
    if (n <= 4096 && k >= 8192) {
        const int r = m > 8 && n > 2048 ? 4 : 2;
        return Cut{r, parts(r), false};
    }
    return Cut{n <= 4096 ? 1 : (n <= 8192 ? 2 : 4), 1, false};
}

template <int TYPE> void pick(const MatvecArgs& a, bool room, hipStream_t stream) {
    const Cut c = cut(a.m, a.n, a.k);
    const int s = room ? c.splits : 1;
    if (a.m > 32)
        c.r == 2 ? launch<TYPE, 2, 4, 8, 1, false>(a, s, stream) : launch<TYPE, 4, 4, 8, 1, false>(a, s, stream);
    else if (a.m > 16)
        c.r == 2 ? launch<TYPE, 2, 2, 8, 2, false>(a, s, stream) : launch<TYPE, 4, 2, 8, 2, false>(a, s, stream);
    else if (c.x)
        c.waves == 16 ? launch<TYPE, 1, 1, 16, 2, true>(a, 1, stream)
                      : (c.r == 1 ? launch<TYPE, 1, 1, 8, 2, true>(a, 1, stream) : launch<TYPE, 2, 1, 8, 2, true>(a, 1, stream));
    else if (c.r == 1)
        launch<TYPE, 1, 1, 8, 2, false>(a, s, stream);
    else if (c.r == 2)
        launch<TYPE, 2, 1, 8, 2, false>(a, s, stream);
    else
        launch<TYPE, 4, 1, 8, 2, false>(a, s, stream);
}

}  // namespace

extern "C" size_t w4_matvec_workspace_bytes(int32_t m, int32_t n, int32_t k) {
    if (m < 1 || n < 1 || k < 1) return 0;
    const int splits = cut(m, n, k).splits;
    return splits > 1 ? (size_t)splits * m * n * sizeof(float) : 0;
}

extern "C" wino_status w4_matvec(const void* x, int64_t x_stride, const uint8_t* codes, const uint8_t* scales,
                                 const void* bias, void* y, int64_t y_stride, int32_t m, int32_t n, int32_t k,
                                 wino_float_type type, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (type != WINO_BF16 && type != WINO_FP16) return WINO_EINVAL;
    if (m < 0 || n < 0 || k < 0 || k % kGroup != 0) return WINO_EINVAL;
    if (m == 0 || n == 0) return WINO_OK;
    if (!y || (k > 0 && (!x || !codes || !scales))) return WINO_EINVAL;
    if (m > 1 && (x_stride < k || y_stride < n)) return WINO_EINVAL;
    if (m > 65535 || n > (1 << 24) || k > (1 << 20)) return WINO_EUNSUPPORTED;
    if (!aligned16(x) || !aligned16(codes) || !aligned16(workspace) || (k > 0 && m > 1 && (x_stride & 7))) return WINO_EUNSUPPORTED;
    MatvecArgs a = {x, codes, scales, bias, y, x_stride, y_stride, m, n, k, 0, (float*)workspace};
    const bool room = workspace && workspace_bytes >= w4_matvec_workspace_bytes(m, n, k);
    if (type == WINO_BF16)
        pick<WINO_BF16>(a, room, stream);
    else
        pick<WINO_FP16>(a, room, stream);
    return hipGetLastError() == hipSuccess ? WINO_OK : WINO_EHIP;
}
