// Rows of 16-bit numbers to 8-bit codes with a scale each: a = max|x| of the
// row, scale = a / 127, code = R(127 x / a), R(v) = floor(v + 1/2), exactly.
//
// The quotient comes from one multiplication by 127 / a in fp32, off by less
// than 2^-22 of itself.  x and a have at most 11 significant bits, so that a
// quotient of at least 1/4 that is not itself half-way between two codes is
// 2^-20 of itself or more away from that (numerators 254 X - (2c + 1) A 2^d
// are whole, A 2^d is at most 2^20 quotients).  Raised by 2^-21 of its
// magnitude, it is on the right side of every such half, and a quotient that
// is a half is no less than it: R takes halves up.
//
// Memory bounds it: 2 bytes read and 1 written a value.  A workgroup takes a
// row and holds it in registers between the maximum and the codes.  2048 rows
// of 16384: 22.4 us, 4.5 TB/s.  Short rows leave threads without work: 32768
// rows of 2816 49 us, 5.6 TB/s in part from the last-level cache; of 1408 37,
// 3.7 TB/s; of 768 25, 2.9 TB/s.
#include <hip/hip_runtime.h>

#include "mx4.h"
#include "winof4.h"

namespace {
using namespace mx4;

struct QuantizeArgs {
    const void* x;
    int8_t* codes;
    float* scales;
    int64_t x_stride;
    int32_t k;
};

// The larger of two pairs of magnitudes (bits of 16-bit numbers without their signs).
__device__ inline uint32_t max_pair(uint32_t a, uint32_t b) {
    typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

template <int TYPE> __device__ inline float value(uint32_t bits) {
    if (TYPE == WINO_BF16) return __builtin_bit_cast(float, bits << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}

// THREADS threads take a row, UNITS times 16 values each; UNITS 0: any number, read twice.
template <int TYPE, int THREADS, int UNITS>
__global__ __launch_bounds__(THREADS) void w8_quantize_kernel(QuantizeArgs a) {
    constexpr int kUnits = UNITS > 0 ? UNITS : 1;
    const int64_t row = blockIdx.x;
    const uint16_t* x = (const uint16_t*)a.x + row * a.x_stride;
    int8_t* codes = a.codes + row * a.k;
    const int units = a.k / 16;
    u32x4 v[kUnits][2];
    uint32_t top = 0;
    auto load = [&](int u, u32x4 (&to)[2]) {
        to[0] = *(const u32x4*)(x + 16 * (int64_t)u);
        to[1] = *(const u32x4*)(x + 16 * (int64_t)u + 8);
    };
    auto raise = [&](const u32x4 (&from)[2]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max_pair(top, from[e / 4][e % 4] & 0x7fff7fffu);
    };
    if constexpr (UNITS > 0) {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int u = threadIdx.x + i * THREADS;
            v[i][0] = v[i][1] = u32x4{0u, 0u, 0u, 0u};
            if (u < units) load(u, v[i]);
        }
#pragma unroll
        for (int i = 0; i < kUnits; ++i) raise(v[i]);
    } else {
        for (int u = threadIdx.x; u < units; u += THREADS) {
            load(u, v[0]);
            raise(v[0]);
        }
    }
    uint32_t most = max(top & 0xffffu, top >> 16);
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, s));
    if constexpr (THREADS > 64) {
        __shared__ uint32_t waves[THREADS / 64];
        if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) most = max(most, waves[w]);
    }
    const bool finite = most < (TYPE == WINO_BF16 ? 0x7f80u : 0x7c00u);
    const float amax = value<TYPE>(most);
    if (threadIdx.x == 0) a.scales[row] = finite ? amax / 127.f : __builtin_nanf("");
    // 127 / amax passes fp32 for the smallest bf16 numbers: those are raised by 2^64 first
    const float lift = amax < 0x1p-64f ? 0x1p64f : 1.f;
    const float inv = finite && most ? 127.f / (amax * lift) : 0.f;
    auto code = [&](uint32_t bits) {
        const float q = finite ? value<TYPE>(bits) * lift * inv : 0.f;
        return (uint32_t)(int32_t)__builtin_floorf(__builtin_fmaf(__builtin_fabsf(q), 0x1p-21f, q) + 0.5f) & 0xffu;
    };
    auto store = [&](int u, const u32x4 (&from)[2]) {
        u32x4 out;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t lo = from[e / 2][e % 2 * 2], hi = from[e / 2][e % 2 * 2 + 1];
            out[e] = code(lo & 0xffffu) | code(lo >> 16) << 8 | code(hi & 0xffffu) << 16 | code(hi >> 16) << 24;
        }
        *(u32x4*)(codes + 16 * (int64_t)u) = out;
    };
    if constexpr (UNITS > 0) {
#pragma unroll
        for (int i = 0; i < kUnits; ++i)
            if (const int u = threadIdx.x + i * THREADS; u < units) store(u, v[i]);
    } else {
        for (int u = threadIdx.x; u < units; u += THREADS) {
            load(u, v[0]);
            store(u, v[0]);
        }
    }
}

template <int TYPE> void launch(const QuantizeArgs& a, int32_t m, hipStream_t stream) {
    const dim3 grid((unsigned)m);
    if (a.k <= 4096)
        hipLaunchKernelGGL((w8_quantize_kernel<TYPE, 256, 1>), grid, dim3(256), 0, stream, a);
    else if (a.k <= 16384)
        hipLaunchKernelGGL((w8_quantize_kernel<TYPE, 256, 4>), grid, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL((w8_quantize_kernel<TYPE, 256, 0>), grid, dim3(256), 0, stream, a);
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace

extern "C" wino_status w8_quantize(const void* x, int64_t x_stride, int8_t* codes, float* scales, int32_t m, int32_t k,
                                   wino_float_type type, hipStream_t stream) {
    if (type != WINO_BF16 && type != WINO_FP16) return WINO_EINVAL;
    if (m < 0 || k < 0 || k % 16 != 0) return WINO_EINVAL;
    if (m == 0) return WINO_OK;
    if (!scales || (k > 0 && (!x || !codes))) return WINO_EINVAL;
    if (m > 1 && x_stride < k) return WINO_EINVAL;
    if (m >= 1 << 24) return WINO_EUNSUPPORTED;             // a launch counts its threads in 32 bits
    if (!aligned16(x) || !aligned16(codes) || ((uintptr_t)scales & 3) || (k > 0 && m > 1 && (x_stride & 7))) return WINO_EUNSUPPORTED;
    const QuantizeArgs a = {x, codes, scales, x_stride, k};
    type == WINO_BF16 ? launch<WINO_BF16>(a, m, stream) : launch<WINO_FP16>(a, m, stream);
    return hipGetLastError() == hipSuccess ? WINO_OK : WINO_EHIP;
}
