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
// Measured over three sets of weights, which the last-level cache holds in part:
// 16384 x 4096, 35.7 MB: 9.9 us for one row of x (3.6 TB/s; a copy of 2 GiB
// reaches 4.8, one of 256 MiB 5.4), and 10.9 over 16 sets, 571 MB; 4096 x 16384
// for 16 rows, in parts: 15.9, and 18.0 over 16 sets.
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

// One step (128 of k, four groups) of R tiles of 16 rows of W: lane (r, g) holds group g of row r, so that a row's four
// lanes read one piece of memory.
template <int R> struct Step {
    u32x4 w[R];
    uint32_t s[R];          // the four scales of the row
};

template <int R> struct Rows {
    const uint8_t* codes[R];
    const uint8_t* scales[R];
    // rows past the end are computed and not stored
    __device__ Rows(const MatvecArgs& a, int row0, int r, int g) {
        const int groups = a.k / kGroup;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t row = min(row0 + 16 * i + r, a.n - 1);
            codes[i] = a.codes + (row * groups + g) * 16;
            scales[i] = a.scales + row * groups;
        }
    }
    // groups first .. first + 3; zeros past the end
    __device__ void load(int first, int end, int g, Step<R>& t) const {
        if (first + 4 <= end) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                t.w[i] = *(const u32x4*)(codes[i] + (int64_t)first * 16);
                __builtin_memcpy(&t.s[i], scales[i] + first, 4);
            }
        } else if (first < end) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                t.w[i] = first + g < end ? *(const u32x4*)(codes[i] + (int64_t)first * 16) : u32x4{0, 0, 0, 0};
                t.s[i] = 0x7f7f7f7f;
                for (int e = 0; e < 3; ++e)
                    if (first + e < end) t.s[i] = (t.s[i] & ~(255u << (8 * e))) | (uint32_t)scales[i][first + e] << (8 * e);
            }
        }
    }
};

// The same without a branch, for k of a step at least: what lies past the end is read from before it, and not used.
template <int R> __device__ inline void load_within(const Rows<R>& rows, int first, int groups, int g, Step<R>& t) {
    const int from = min(first, groups - 4), shift = 8 * min(first - from, 3), back = min(first + g, groups - 1) - g;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        t.w[i] = *(const u32x4*)(rows.codes[i] + (int64_t)back * 16);
        __builtin_memcpy(&t.s[i], rows.scales[i] + from, 4);
        t.s[i] = t.s[i] >> shift | (~(0xffffffffu >> shift) & 0x7f7f7f7fu);
    }
}

// The products take group e of a step with its eighths spread over the quarters of the wave: a 4 x 4 exchange.
__device__ inline void turn(const u32x4& w, uint32_t (&out)[4]) {
    const auto s02 = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
    const auto s13 = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    const auto s01 = __builtin_amdgcn_permlane16_swap(s02[0], s13[0], false, false);
    const auto s23 = __builtin_amdgcn_permlane16_swap(s02[1], s13[1], false, false);
    out[0] = s01[0], out[1] = s01[1], out[2] = s23[0], out[3] = s23[1];
}

// Smallest and largest scale byte, two at a time.
struct Range {
    uint32_t most = 0x007f007f, least = 0x007f007f;
    __device__ void add(uint32_t s) {
        typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
        const u16x2 even = __builtin_bit_cast(u16x2, s & 0x00ff00ffu), odd = __builtin_bit_cast(u16x2, (s >> 8) & 0x00ff00ffu);
        most = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, most),
                                                                      __builtin_elementwise_max(even, odd)));
        least = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u16x2, least),
                                                                       __builtin_elementwise_min(even, odd)));
    }
    // scales from 2^-23 to 2^13: fp16 holds the weights exactly
    __device__ bool fits_fp16() const {
        return max(most & 0xffffu, most >> 16) <= 140u && min(least & 0xffffu, least >> 16) >= 104u;
    }
};

// acc += W x for one group: word w[i] and scale s[i] of R rows, v of N tiles of x.  SPLIT: x in fp16 as two bf16
// numbers (8 + 3 bits, exact); else the products of fp16 are fp16 ones.
template <int TYPE, bool SPLIT, int R, int N, typename T8>
__device__ inline void multiply(const uint32_t (&w)[R], const float (&s)[R], const T8 (&v)[N], f32x4 (&acc)[R][N]) {
    if constexpr (TYPE == WINO_FP16 && !SPLIT) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const f16x8 u = decode8_f16(w[i], s[i]);
#pragma unroll
            for (int j = 0; j < N; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(u, v[j], acc[i][j], 0, 0, 0);
        }
    } else {
        constexpr int kParts = SPLIT ? 2 : 1;
        bf16x8 b[kParts][N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if constexpr (!SPLIT) {
                b[0][j] = v[j];
            } else {
#pragma unroll
                for (int d = 0; d < 8; ++d) {
                    const float f = (float)v[j][d];
                    const __bf16 hi = (__bf16)f;
                    b[0][j][d] = hi;
                    const float rest = f - (float)hi;           // infinity less itself: no rest
                    b[1][j][d] = (__bf16)(rest == rest ? rest : 0.f);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const bf16x8 u = decode8(w[i], s[i]);
#pragma unroll
            for (int p = 0; p < kParts; ++p)
#pragma unroll
                for (int j = 0; j < N; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(u, b[p][j], acc[i][j], 0, 0, 0);
        }
    }
}

// A sum of row `row` of W and row `tok` of x: stored, or left for w4_matvec_join.
template <typename T> __device__ inline void store(const MatvecArgs& a, int row, int tok, float sum) {
    if (row >= a.n || tok >= a.m) return;
    if (a.part) {
        a.part[((int64_t)blockIdx.z * a.m + tok) * a.n + row] = sum;
    } else {
        if (a.bias) sum += (float)((const T*)a.bias)[row];
        ((T*)a.y)[(int64_t)tok * a.y_stride + row] = (T)sum;
    }
}

// 16 rows of x.  R tiles of 16 rows of W, V waves that share out k, two steps of codes on their way.  X: x lies in
// LDS; else its pieces come with the codes.  blockIdx.z takes `steps` steps of k; where there are several, their sums
// go to a.part and w4_matvec_join adds them up.
template <int TYPE, int R, int V, bool X> __global__ __launch_bounds__(64 * V) void w4_matvec_kernel(MatvecArgs a) {
    typedef typename Half<TYPE>::type T;
    typedef T T8 __attribute__((ext_vector_type(8)));
    constexpr int D = 2;
    __shared__ float join[V][R * 16][17];
    extern __shared__ __attribute__((aligned(16))) uint8_t x_lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int row0 = blockIdx.x * (16 * R), tok0 = blockIdx.y * 16, toks = min(16, a.m - tok0);
    const int begin = blockIdx.z * a.steps * 4, end = min(a.k / kGroup, begin + a.steps * 4);
    const Rows<R> rows(a, row0, r, g);
    // x of this lane: row r (the last one again past the end), eighth g of a group
    const int x_row = (end - begin) * kGroup * 2 + 16;          // bytes of a row in LDS: 16 rows in 16 columns of the banks
    const int tok = min(r, toks - 1);
    const T* x = (const T*)a.x + (int64_t)(tok0 + tok) * a.x_stride + 8 * g;
    const uint8_t* xl = x_lds + tok * x_row - begin * kGroup * 2 + 16 * g;

    struct Both {
        Step<R> w;
        T8 x[4];
    };
    auto load = [&](int first, Both& t) {
        rows.load(first, end, g, t.w);
        if constexpr (!X) {
            if (first + 4 <= end) {
#pragma unroll
                for (int e = 0; e < 4; ++e) t.x[e] = *(const T8*)(x + (first + e) * kGroup);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) t.x[e] = first + e < end ? *(const T8*)(x + (first + e) * kGroup) : T8{};
            }
        }
    };
    f32x4 acc[R][1];                                            // lane: rows 4 g + e of W, row r of x
    Range range;
    auto compute = [&](int first, const Both& t, auto split) {
        uint32_t w[R][4];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            turn(t.w.w[i], w[i]);
            if constexpr (TYPE == WINO_FP16) range.add(t.w.s[i]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            T8 v[1];
            if constexpr (X)
                v[0] = first + e < end ? *(const T8*)(xl + (first + e) * (kGroup * 2)) : T8{};
            else
                v[0] = t.x[e];
            uint32_t we[R];
            float s[R];
#pragma unroll
            for (int i = 0; i < R; ++i) we[i] = w[i][e], s[i] = scale_bits((t.w.s[i] >> (8 * e)) & 255u);
            multiply<TYPE, decltype(split)::value, R, 1>(we, s, v, acc);
        }
    };
    // the wave's steps: every V-th
    const int mine = max(0, (end - begin - wave * 4 + 4 * V - 1) / (4 * V));
    auto at = [&](int i) { return begin + (wave + V * i) * 4; };
    Both t[D];
    auto start = [&]() {
#pragma unroll
        for (int d = 0; d < D; ++d)
            if (d < mine) load(at(d), t[d]);
    };
    auto sweep = [&](auto split) {
#pragma unroll
        for (int i = 0; i < R; ++i) acc[i][0] = f32x4{0.f, 0.f, 0.f, 0.f};
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
    start();
    if constexpr (X) {
        const int pieces = (end - begin) * 4;
        for (int i = threadIdx.x; i < pieces * toks; i += 64 * V) {
            const int tok = i / pieces, p = i - tok * pieces;
            *(T8*)(x_lds + tok * x_row + p * 16) =
                *(const T8*)((const T*)a.x + (int64_t)(tok0 + tok) * a.x_stride + begin * kGroup + p * 8);
        }
        __syncthreads();
    }
    sweep(std::false_type{});
    if constexpr (TYPE == WINO_FP16) {
        if (__any(!range.fits_fp16())) {
            start();
            sweep(std::true_type{});
        }
    }
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) join[wave][16 * i + 4 * g + e][r] = acc[i][0][e];
    __syncthreads();
    for (int o = threadIdx.x; o < R * 256; o += 64 * V) {
        const int row = o % (R * 16), tok = o / (R * 16);
        float sum = join[0][row][tok];
#pragma unroll
        for (int w = 1; w < V; ++w) sum += join[w][row][tok];
        store<T>(a, row0 + row, tok0 + tok, sum);
    }
}

// More rows of x, or more of W, in tiles of N times 16 of x.  Eight waves: two with R tiles of 16 rows of W each, times
// four that share out k.  x goes through LDS, 512 of k at a time, the next ones on their way while these are multiplied:
// both halves of the waves read it there, which halves what the L2 has to deliver, and rows are copied a KiB at a time.
// Two steps of codes are on their way.  64 rows by 16384 x 4096: 20.4 us, 1.7 TB/s of weights; a workgroup takes 1.6 us
// for 512 of k, whose products and LDS reads take half of that and whose barrier keeps the waves in step.
template <int TYPE, int R, int N> __global__ __launch_bounds__(512) void w4_matmul_kernel(MatvecArgs a) {
    typedef typename Half<TYPE>::type T;
    typedef T T8 __attribute__((ext_vector_type(8)));
    constexpr int D = 2, kShare = 4, kRow = kShare * 256;       // steps of codes; waves along k; bytes of a row of x in LDS
    constexpr int kBuf = 16 * N * kRow, kCopies = 2 * N;        // pieces of 16 bytes that a thread copies
    constexpr int kJoin = kShare * 32 * R * (16 * N + 1) * 4;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * kBuf > kJoin ? 2 * kBuf : kJoin];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4, share = wave % kShare, upper = wave / kShare;
    const int row0 = blockIdx.x * (32 * R), tok0 = blockIdx.y * (16 * N);
    const int groups = a.k / kGroup, begin = blockIdx.z * a.steps * 4, end = min(groups, begin + a.steps * 4);
    const Rows<R> rows(a, row0 + 16 * R * upper, r, g);
    const int chunks = (end - begin + 4 * kShare - 1) / (4 * kShare);
    auto at = [&](int c) { return begin + (c * kShare + share) * 4; };

    // A wave copies row `wave` + 8 x of the tile, a lane one piece of it.  Piece p of row t lies at p ^ (t % 16), so that
    // reading one piece of 16 rows takes all banks once.  Past the ends it copies the last row and piece again.
    T8 piece[kCopies];
    auto fetch = [&](int c) {
        const int first = begin + c * (4 * kShare);
#pragma unroll
        for (int x = 0; x < kCopies; ++x) {
            const int t = wave + 8 * x, tok = min(tok0 + t, a.m - 1), p = min(lane ^ (t & 15), (end - first) * 4 - 1);
            piece[x] = *(const T8*)((const T*)a.x + (int64_t)tok * a.x_stride + first * kGroup + p * 8);
        }
    };
    auto put = [&](int buf) {
#pragma unroll
        for (int x = 0; x < kCopies; ++x) *(T8*)(lds + buf * kBuf + (wave + 8 * x) * kRow + lane * 16) = piece[x];
    };
    f32x4 acc[R][N];
    Range range;
    auto compute = [&](int first, int buf, const Step<R>& t, auto split) {
        uint32_t w[R][4];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            turn(t.w[i], w[i]);
            if constexpr (TYPE == WINO_FP16) range.add(t.s[i]);
        }
        const uint8_t* x = lds + buf * kBuf + r * kRow;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (first + e >= end) break;
            T8 v[N];
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = *(const T8*)(x + 16 * j * kRow + ((share * 16 + e * 4 + g) ^ r) * 16);
            uint32_t we[R];
            float s[R];
#pragma unroll
            for (int i = 0; i < R; ++i) we[i] = w[i][e], s[i] = scale_bits((t.s[i] >> (8 * e)) & 255u);
            multiply<TYPE, decltype(split)::value, R, N>(we, s, v, acc);
        }
    };
    auto sweep = [&](auto split) {
        Step<R> t[D];
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int d = 0; d < D; ++d)
            if (d < chunks) load_within(rows, at(d), groups, g, t[d]);
        fetch(0);
        put(0);
        // chunk c, whose codes are in t[d], and what is asked for meanwhile
        auto turn_to = [&](int c, int d, bool next, bool codes) {
            __syncthreads();                                    // the chunk is there, and nobody reads the other one any more
            if (next) fetch(c + 1);
            compute(at(c), c & 1, t[d], split);
            if (codes) load_within(rows, at(c + D), groups, g, t[d]);
            if (next) put((c + 1) & 1);
        };
        // Loads behind conditions make the products wait for all that may have been asked for, so there are none but at
        // the end.
        int c = 0;
        for (; c + 2 * D <= chunks; c += D) {
#pragma unroll
            for (int d = 0; d < D; ++d) turn_to(c + d, d, true, true);
        }
#pragma unroll
        for (int d = 0; d < 2 * D - 1; ++d)
            if (c + d < chunks) turn_to(c + d, d % D, c + d + 1 < chunks, d < D - 1 && c + d + D < chunks);
        __syncthreads();
    };
    sweep(std::false_type{});
    if constexpr (TYPE == WINO_FP16)
        if (__syncthreads_or(!range.fits_fp16())) sweep(std::true_type{});
    float(*join)[32 * R][16 * N + 1] = (float(*)[32 * R][16 * N + 1])lds;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) join[share][16 * (R * upper + i) + 4 * g + e][16 * j + r] = acc[i][j][e];
    __syncthreads();
    for (int o = threadIdx.x; o < R * N * 512; o += 512) {
        const int row = o % (32 * R), tok = o / (32 * R);
        float sum = join[0][row][tok];
#pragma unroll
        for (int w = 1; w < kShare; ++w) sum += join[w][row][tok];
        store<T>(a, row0 + row, tok0 + tok, sum);
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

// Parts of k in whole steps.
int share_out(MatvecArgs& a, int splits) {
    const int steps = (a.k + 127) / 128;
    a.steps = (steps + splits - 1) / splits;
    splits = a.steps > 0 ? (steps + a.steps - 1) / a.steps : 1;
    if (splits <= 1) a.part = nullptr;
    return splits;
}
template <int TYPE> void join(const MatvecArgs& a, int splits, hipStream_t stream) {
    if (splits > 1)
        hipLaunchKernelGGL((w4_matvec_join<TYPE>), dim3((unsigned)((a.n + 255) / 256), (unsigned)a.m), dim3(256), 0, stream,
                           a, splits);
}
template <int TYPE, int R, int V, bool X> void launch(MatvecArgs a, int splits, hipStream_t stream) {
    splits = share_out(a, splits);
    const size_t lds = X ? (size_t)std::min(a.m, 16) * (std::min(a.k, a.steps * 128) * 2 + 16) : 0;
    const dim3 grid((unsigned)((a.n + 16 * R - 1) / (16 * R)), (unsigned)((a.m + 15) / 16), (unsigned)splits);
    hipLaunchKernelGGL((w4_matvec_kernel<TYPE, R, V, X>), grid, dim3(64 * V), lds, stream, a);
    join<TYPE>(a, splits, stream);
}
template <int TYPE, int R, int N> void launch_wide(MatvecArgs a, int splits, hipStream_t stream) {
    splits = share_out(a, splits);
    const dim3 grid((unsigned)((a.n + 32 * R - 1) / (32 * R)), (unsigned)((a.m + 16 * N - 1) / (16 * N)), (unsigned)splits);
    hipLaunchKernelGGL((w4_matmul_kernel<TYPE, R, N>), grid, dim3(512), 0, stream, a);
    join<TYPE>(a, splits, stream);
}

// Which kernel takes a call and how it is cut: tiles of 16 rows of W (times two waves where `wide`), k in `splits` parts,
// x in LDS or beside the codes.
struct Cut {
    bool wide;
    int r, splits;
    bool x = false;
    int waves = 8;
};

// A kernel that does not hold x in LDS whole, and what it takes (us, measured): `step` for 1024 of k and `start` beside
// it, for as many workgroups as there are compute units (256) or fewer; `pair` times that for twice as many, side by side.
struct Form {
    bool wide;
    int r;
    double step, start, pair;
    // k in `splits` parts: whole rounds of the device, and the join, a second launch
    double time(int64_t m, int64_t n, int64_t k, int splits) const {
        const int64_t rows = (wide ? 32 : 16) * r, x_tiles = wide ? (m + 63) / 64 : 1;
        const int64_t groups = (n + rows - 1) / rows * x_tiles * splits, rest = groups % 512;
        const double rounds = pair * (double)(groups / 512) + (rest == 0 ? 0 : (rest <= 256 ? 1 : pair));
        const double join = splits > 1 ? 2.2 + 0.21 * splits + 3.8e-6 * (double)(splits * m * n) : 0;
        return (start + step * (double)k / (1024 * splits)) * rounds + join;
    }
};

// x in LDS while it fits and there is little of it beside W: one row of 4096 x 4096 4.7 us (beside the codes 5.3), four
// 5.2 (5.9); with 16 waves for few outputs (eight: 5.2 and 5.8).  64 rows by 2048 x 1248: 4.3 (wide 6.8).  Else what is
// estimated to be the shortest: over 737 sizes of 1 to 64 rows, 512 to 32768 outputs and k of 1024 to 16384 (bf16) that is
// 1% longer than the shortest measured one on average, 20% at most.  With parts only while a workgroup for each compute unit
// holds them all it was 6% on average and 50% at most, beside whole rounds.  Some of them (us; w: wide, n: beside the codes,
// tiles of W, parts):
//   16 rows, k 16384   4096 outputs w1 in 4 17.8, w2 in 4 17.8, w1 30.4     4160 w1 in 3 22.0, w1 in 4 22.6, n2 31.3, w1 30.9
//                      5120 w1 in 3 22.6, w2 in 3 22.3, n2 31.8             8256 w2 in 3 33.8, w2 46.1
//   8 rows             4096 x 4096 n1 6.6, w1 in 2 7.8                      8192 x 8192 n2 14.9, w1 in 2 15.9
//   32 rows            4096 x 4096 w1 in 2 9.5, w2 in 4 9.9                 8192 x 8192 w1 20.5, w2 in 2 19.1 (taken: w1)
//   64 rows            16384 x 4096 w2 20.1, w1 29.3
//   2048 rows          4096 x 16384 whole 430, in 4 parts 534 and 128 MB of sums
Cut cut(int64_t m, int64_t n, int64_t k) {
    const bool fits = std::min<int64_t>(m, 16) * (2 * k + 16) <= 40960;
    const bool little = (m <= 16 || n <= 4096) && (m <= 4 || n <= 8192) && !(n <= 2048 && k >= 12288);
    if (fits && (little || k < 128)) return Cut{false, n <= 8192 ? 1 : 2, 1, true, n <= 4096 ? 16 : 8};
    const double rows = 1 + 0.062 * (double)m;              // beside the codes, each row of x is read by each wave
    const Form one[] = {{false, 1, 0.64 * rows, 0.23, 2}, {false, 2, 0.93 * rows, 0.23, 2}, {true, 1, 1.64, 0.15, 1.52}, {true, 2, 3.2, 0.15, 1.52}};
    const Form two[] = {{true, 1, 2.03, 0.3, 1.6}, {true, 2, 3.25, 0.3, 1.6}};
    const Form four[] = {{true, 1, 3.3, 0.1, 1.8}, {true, 2, 4.69, 0.1, 1.8}};
    const Form* forms = m <= 16 ? one : (m <= 32 ? two : four);
    Cut best{};
    double least = 0;
    for (int f = 0; f < (m <= 16 ? 4 : 2); ++f)
        for (const int splits : {1, 2, 3, 4, 6, 8}) {
            // 1024 of k in a part at least, and 4 MiB of sums at most
            if (splits > 1 && (k < 1024 * splits || splits * m * n > 1 << 20)) break;
            const double t = forms[f].time(m, n, k, splits);
            if (least == 0 || t < least) least = t, best = Cut{forms[f].wide, forms[f].r, splits};
        }
    return best;
}

bool beyond(int32_t m, int32_t n, int32_t k) { return m > 65535 || n > (1 << 24) || k > (1 << 20); }

size_t part_bytes(const Cut& c, int64_t m, int64_t n) { return c.splits > 1 ? (size_t)(c.splits * m * n) * sizeof(float) : 0; }

template <int TYPE> void pick(const MatvecArgs& a, size_t bytes, hipStream_t stream) {
    const Cut c = cut(a.m, a.n, a.k);
    const int s = a.part && bytes >= part_bytes(c, a.m, a.n) ? c.splits : 1;
    if (c.wide && a.m > 32)
        c.r == 1 ? launch_wide<TYPE, 1, 4>(a, s, stream) : launch_wide<TYPE, 2, 4>(a, s, stream);
    else if (c.wide && a.m > 16)
        c.r == 1 ? launch_wide<TYPE, 1, 2>(a, s, stream) : launch_wide<TYPE, 2, 2>(a, s, stream);
    else if (c.wide)
        c.r == 1 ? launch_wide<TYPE, 1, 1>(a, s, stream) : launch_wide<TYPE, 2, 1>(a, s, stream);
    else if (c.x)
        c.waves == 16 ? launch<TYPE, 1, 16, true>(a, 1, stream)
                      : (c.r == 1 ? launch<TYPE, 1, 8, true>(a, 1, stream) : launch<TYPE, 2, 8, true>(a, 1, stream));
    else
        c.r == 1 ? launch<TYPE, 1, 8, false>(a, s, stream) : launch<TYPE, 2, 8, false>(a, s, stream);
}

}  // namespace

extern "C" size_t w4_matvec_workspace_bytes(int32_t m, int32_t n, int32_t k) {
    if (m < 1 || n < 1 || k < 1 || beyond(m, n, k)) return 0;
    return part_bytes(cut(m, n, k), m, n);
}

extern "C" wino_status w4_matvec(const void* x, int64_t x_stride, const uint8_t* codes, const uint8_t* scales,
                                 const void* bias, void* y, int64_t y_stride, int32_t m, int32_t n, int32_t k,
                                 wino_float_type type, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (type != WINO_BF16 && type != WINO_FP16) return WINO_EINVAL;
    if (m < 0 || n < 0 || k < 0 || k % kGroup != 0) return WINO_EINVAL;
    if (m == 0 || n == 0) return WINO_OK;
    if (!y || (k > 0 && (!x || !codes || !scales))) return WINO_EINVAL;
    if (m > 1 && (x_stride < k || y_stride < n)) return WINO_EINVAL;
    if (beyond(m, n, k)) return WINO_EUNSUPPORTED;
    if (!aligned16(x) || !aligned16(codes) || !aligned16(workspace) || (k > 0 && m > 1 && (x_stride & 7))) return WINO_EUNSUPPORTED;
    MatvecArgs a = {x, codes, scales, bias, y, x_stride, y_stride, m, n, k, 0, (float*)workspace};
    if (type == WINO_BF16)
        pick<WINO_BF16>(a, workspace_bytes, stream);
    else
        pick<WINO_FP16>(a, workspace_bytes, stream);
    return hipGetLastError() == hipSuccess ? WINO_OK : WINO_EHIP;
}
