// Many rows times 8-bit weights: tiles of outputs, operands through LDS.
//
// The matrix cores bound it.  Weights are the first operand of mfma 32x32x32 (the form that reaches their full rate), x the
// second; a wave has WN x WM blocks of 32 x 32.  Stages of BK bytes of k are copied from memory straight to LDS, STAGES - 1
// ahead; the copies fill LDS densely, so the 16-byte pieces of a row are exchanged (swap) such that sixteen rows' reads of
// the same piece fall into the sixteen columns of the 256-byte banks.  Within 32 rows of weights the copy puts row
// 16 h + 4 q + e where operand row 8 q + 4 h + e is read: a lane's sixteen sums are then neighbouring outputs of one row.
#pragma once
#include "w8_device.h"

namespace w8 {

template <int WN_, int WM_, int GN_, int GM_, int BK_, int STAGES_> struct Tile {
    static constexpr int WN = WN_, WM = WM_, GN = GN_, GM = GM_, BK = BK_, STAGES = STAGES_;
    static constexpr int kWaves = GN * GM, kThreads = 64 * kWaves;
    static constexpr int kOuts = 32 * WN * GN, kRows = 32 * WM * GM;        // of a workgroup
    static constexpr int kRowPieces = BK / 16;
    static constexpr int kPiecesW = kOuts * kRowPieces / kThreads, kPiecesX = kRows * kRowPieces / kThreads;    // of a thread
    static constexpr int kBytesW = kOuts * BK, kBytes = kBytesW + kRows * BK;
    static_assert(kOuts * kRowPieces % kThreads == 0 && kRows * kRowPieces % kThreads == 0, "whole copies");
    static __device__ int swap(int row) { return BK == 128 ? (row >> 1) & 7 : (row >> 2) & 3; }
};

// The tile of the experts' rows that is the index-th: its expert, and where its rows begin and end in the order.
template <int ROWS> __device__ inline bool find(const Args& a, int index, int& expert, int& begin, int& end) {
    const int lane = threadIdx.x & 63;
    for (int e0 = 0; e0 < a.experts; e0 += 64) {
        int b = 0, e = 0;
        if (e0 + lane < a.experts) rows_of(a, e0 + lane, b, e);
        const int count = (e - b + ROWS - 1) / ROWS;
        int upto = count;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const int other = __shfl_up(upto, s);
            if (lane >= s) upto += other;
        }
        const uint64_t here = __ballot(index < upto);
        if (here) {
            const int l = __builtin_ctzll(here);
            expert = e0 + l;
            begin = __shfl(b, l) + (index - (__shfl(upto, l) - __shfl(count, l))) * ROWS;
            end = __shfl(e, l);
            return true;
        }
        index -= __shfl(upto, 63);
    }
    return false;
}

template <int TYPE, class S, bool EXPERTS>
__global__ __launch_bounds__(S::kThreads) void w8_tiles_kernel(Args a, int n_tiles, int m_tiles) {
    typedef typename Half<TYPE>::type T;
    typedef __attribute__((ext_vector_type(2))) T T2;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[S::STAGES][S::kBytes];
    __shared__ float w_scale[S::kOuts], bias[S::kOuts], x_scale[S::kRows];
    __shared__ int out_row[S::kRows];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 31, half = lane >> 5;

    int m0, m1, n0, expert = 0;
    if (EXPERTS) {
        n0 = (int)(blockIdx.x % n_tiles) * S::kOuts;
        if (!find<S::kRows>(a, blockIdx.x / n_tiles, expert, m0, m1)) return;
        expert = __builtin_amdgcn_readfirstlane(expert);
        m0 = __builtin_amdgcn_readfirstlane(m0);
        m1 = __builtin_amdgcn_readfirstlane(m1);
    } else {
        // workgroup i runs on XCD i % 8: each gets neighbouring tiles, eight rows of them at a time
        const int tiles = n_tiles * m_tiles, each = (tiles + 7) / 8;
        const int t = (int)(blockIdx.x % 8) * each + (int)(blockIdx.x / 8);
        if ((int)(blockIdx.x / 8) >= each || t >= tiles) return;
        const int set = 8 * n_tiles, g = t / set, high = min(8, m_tiles - 8 * g), in = t - g * set;
        m0 = (8 * g + in % high) * S::kRows;
        n0 = in / high * S::kOuts;
        m1 = a.m;
    }
    const int all = (a.k + S::BK - 1) / S::BK;
    const int first = EXPERTS ? 0 : (int)blockIdx.y * a.steps, last = EXPERTS ? all : min(first + a.steps, all);

    for (int o = threadIdx.x; o < S::kOuts; o += S::kThreads) {
        const int col = min(n0 + o, a.n - 1);
        w_scale[o] = a.w_scales[(int64_t)expert * a.n + col];
        bias[o] = !EXPERTS && a.bias ? (float)((const T*)a.bias)[col] : 0.f;
    }
    for (int o = threadIdx.x; o < S::kRows; o += S::kThreads) {
        const int at = min(m0 + o, m1 - 1), route = EXPERTS ? a.order[at] : at;
        x_scale[o] = a.x_scales[EXPERTS ? x_row(a, route) : route];
        out_row[o] = m0 + o < m1 && (!EXPERTS || (uint32_t)route < (uint32_t)a.routes) ? route : -1;
    }

    const int8_t *from_w[S::kPiecesW], *from_x[S::kPiecesX];
    auto place = [&](int p, int& row, int& piece) {
        row = p / S::kRowPieces;
        piece = (p % S::kRowPieces) ^ S::swap(row);
    };
#pragma unroll
    for (int i = 0; i < S::kPiecesW; ++i) {
        int row, piece;
        place((i * S::kWaves + wave) * 64 + lane, row, piece);
        const int w_row = (row & ~31) | (row >> 2 & 1) << 4 | (row >> 3 & 3) << 2 | (row & 3);
        from_w[i] = a.w + ((int64_t)expert * a.n + min(n0 + w_row, a.n - 1)) * a.k + (int64_t)first * S::BK + 16 * piece;
    }
#pragma unroll
    for (int i = 0; i < S::kPiecesX; ++i) {
        int row, piece;
        place((i * S::kWaves + wave) * 64 + lane, row, piece);
        const int at = min(m0 + row, m1 - 1);
        from_x[i] = a.x + (EXPERTS ? x_row(a, a.order[at]) : at) * a.x_stride + (int64_t)first * S::BK + 16 * piece;
    }
    typedef __attribute__((address_space(3))) uint8_t* lds_ptr;
    const lds_ptr to = (lds_ptr)&lds[0][0] + wave * 1024;
    auto copy = [&](int s, int buf) {
        const bool cut = (s + 1) * S::BK > a.k;              // the end of k lies inside this stage
#pragma unroll
        for (int i = 0; i < S::kPiecesW + S::kPiecesX; ++i) {
            const bool is_w = i < S::kPiecesW;
            const int j = is_w ? i : i - S::kPiecesW;
            const int8_t*& from = is_w ? from_w[j] : from_x[j];
            const int8_t* src = from;
            if (cut) {
                int row, piece;
                place((j * S::kWaves + wave) * 64 + lane, row, piece);
                if (s * S::BK + 16 * piece >= a.k) src = (const int8_t*)kZeros;
            }
            winof4::lds_copy16(src, to + buf * S::kBytes + (is_w ? 0 : S::kBytesW) + j * (1024 * S::kWaves));
            from += S::BK;
        }
    };

    i32x16 acc[S::WN][S::WM];
#pragma unroll
    for (int i = 0; i < S::WN; ++i)
#pragma unroll
        for (int j = 0; j < S::WM; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;

    const int wn = wave % S::GN, wm = wave / S::GN;
    constexpr int kPieces = S::kPiecesW + S::kPiecesX;
#pragma unroll
    for (int s = 0; s < S::STAGES - 1; ++s)
        if (first + s < last) copy(first + s, s);
    int buf = 0, next = S::STAGES - 1;
    for (int s = first; s < last; ++s) {
        // this stage has arrived once no more than the later ones are on their way
        if (s + S::STAGES - 2 < last)
            WINO_WAIT_VM_LDS((S::STAGES - 2) * kPieces);
        else
            WINO_WAIT_VM_LDS(0);
        winof4::ring_barrier();                             // all waves' copies, and nobody reads the buffer that is filled next
        if (s + S::STAGES - 1 < last) copy(s + S::STAGES - 1, next);
        const uint8_t* lw = lds[buf] + (32 * S::WN * wn + c) * S::BK;
        const uint8_t* lx = lds[buf] + S::kBytesW + (32 * S::WM * wm + c) * S::BK;
#pragma unroll
        for (int t = 0; t < S::BK / 32; ++t) {
            const int at = ((2 * t + half) ^ S::swap(c)) * 16;
            i32x4 w[S::WN], x[S::WM];
#pragma unroll
            for (int i = 0; i < S::WN; ++i) w[i] = *(const i32x4*)(lw + i * (32 * S::BK) + at);
#pragma unroll
            for (int j = 0; j < S::WM; ++j) x[j] = *(const i32x4*)(lx + j * (32 * S::BK) + at);
#pragma unroll
            for (int i = 0; i < S::WN; ++i)
#pragma unroll
                for (int j = 0; j < S::WM; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[i], x[j], acc[i][j], 0, 0, 0);
        }
        buf = buf + 1 == S::STAGES ? 0 : buf + 1;
        next = next + 1 == S::STAGES ? 0 : next + 1;
    }
    __syncthreads();                                        // the scales, where there was no stage

#pragma unroll
    for (int j = 0; j < S::WM; ++j) {
        const int at = 32 * (S::WM * wm + j) + c, row = out_row[at];
        if (row < 0) continue;
        const float xs = x_scale[at];
#pragma unroll
        for (int i = 0; i < S::WN; ++i) {
            const int o = 32 * (S::WN * wn + i) + 16 * half, col = n0 + o;
            if (!EXPERTS && a.part) {
                int32_t* to = a.part + ((int64_t)blockIdx.y * a.m + row) * a.n + col;
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (col + e < a.n) to[e] = acc[i][j][e];
                continue;
            }
            float y[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = finish(acc[i][j][e], xs, w_scale[o + e], bias[o + e]);
            if (EXPERTS && a.products) {
                float* to = a.products + (int64_t)row * a.n + col;
                if (col + 16 <= a.n && (a.n & 3) == 0) {
#pragma unroll
                    for (int e = 0; e < 16; e += 4) *(f32x4*)(to + e) = f32x4{y[e], y[e + 1], y[e + 2], y[e + 3]};
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (col + e < a.n) to[e] = y[e];
                }
                continue;
            }
            T* to = (T*)a.y + row * a.y_stride + col;
            if (col + 16 <= a.n && ((uintptr_t)to & 15) == 0) {
                u32x4 out[2];
#pragma unroll
                for (int e = 0; e < 8; ++e) out[e / 4][e % 4] = __builtin_bit_cast(uint32_t, T2{(T)y[2 * e], (T)y[2 * e + 1]});
                *(u32x4*)to = out[0];
                *(u32x4*)(to + 8) = out[1];
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (col + e < a.n) to[e] = (T)y[e];
            }
        }
    }
}

}  // namespace w8
