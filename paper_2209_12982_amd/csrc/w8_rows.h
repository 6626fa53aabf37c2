// Few rows times 8-bit weights, sixteen at a time: each time every byte of the weights is read once and used by one wave.  More
// dense rows are more workgroups, which share the weights in the caches; an expert's rows have one workgroup, sixteen after
// sixteen.  A workgroup has 16 NT outputs; its V waves share out k in steps of 128 bytes, and their sums meet in LDS.
//
// Rows of the weights are rows of the first operand of mfma 16x16x64, rows of x columns of the second.  Which part of k
// stands where in an operand is free as long as both agree: a lane reads 32 neighbouring bytes of its row, the first 16 for
// one product and the rest for the next, so that the two loads of a wave take whole lines of 128 bytes.
//
// Memory bounds it.  One row by 4096 x 4096: 4.7 to 5.7 us, 3.0 to 3.6 TB/s with the start and end of the launch; 32
// tokens to 6 of 64 experts, 2816 x 2048: 60 us, 5.8 TB/s for the experts that some token has.
#pragma once
#include "w8_device.h"

namespace w8 {

// The rows that workgroup `set` of a dense product takes: each row falls to one.
struct Span {
    int begin, end;
};
constexpr Span rows_of_set(int set, int rows, int m) { return {set * rows, m - set * rows < rows ? m : set * rows + rows}; }

// The expert that is number `which` of those that have rows, or false.
__device__ inline bool expert_with_rows(const Args& a, int which, int& expert, int& begin, int& end) {
    const int lane = threadIdx.x & 63;
    for (int e0 = 0; e0 < a.experts; e0 += 64) {
        int b = 0, e = 0;
        if (e0 + lane < a.experts) rows_of(a, e0 + lane, b, e);
        const uint64_t some = __ballot(b < e);
        const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(some >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)some, 0));
        const uint64_t here = __ballot(b < e && before == which);
        if (here) {
            const int l = __builtin_ctzll(here);
            expert = e0 + l;
            begin = __builtin_amdgcn_readlane(b, l);
            end = __builtin_amdgcn_readlane(e, l);
            return true;
        }
        which -= __builtin_popcountll(some);
    }
    return false;
}

template <int TYPE, int NT, int V, bool EXPERTS>
__global__ __launch_bounds__(64 * V) void w8_rows_kernel(Args a) {
    typedef typename Half<TYPE>::type T;
    constexpr int kRows = 16, kOuts = 16 * NT, kAhead = 2;  // steps whose loads are on their way together
    __shared__ int sums[kRows][kOuts + 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, quarter = lane >> 4;
    const int n0 = blockIdx.x * kOuts;
    int begin, end, expert = 0;
    if (EXPERTS) {
        expert = blockIdx.y;
        if ((int)gridDim.y < a.experts) {
            if (!expert_with_rows(a, blockIdx.y, expert, begin, end)) return;
        } else {
            rows_of(a, expert, begin, end);
        }
    } else {
        const Span own = rows_of_set(blockIdx.y, kRows, a.m);
        begin = own.begin, end = own.end;
    }
    const int8_t* w[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i)
        w[i] = a.w + ((int64_t)expert * a.n + min(n0 + 16 * i + r, a.n - 1)) * a.k + 32 * quarter;
    const int last = (a.k + 127) / 128;
    for (int m0 = begin; m0 < end; m0 += kRows) {               // once, where they are no expert's
        const int own = min(m0 + r, end - 1);
        const int8_t* x = a.x + (EXPERTS ? x_row(a, a.order[own]) : own) * a.x_stride + 32 * quarter;
        for (int o = threadIdx.x; o < kRows * kOuts; o += 64 * V) sums[o / kOuts][o % kOuts] = 0;
        // what a thread's results need beside their sums is asked for before the loop, not behind it
        constexpr int kMine = (kRows * kOuts + 64 * V - 1) / (64 * V);
        int row[kMine];
        float xs[kMine], ws[kMine], bias[kMine];
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int o = threadIdx.x + 64 * V * i, at = m0 + o / kOuts, c = n0 + o % kOuts;
            row[i] = -1;
            if (o >= kRows * kOuts || at >= end || c >= a.n) continue;
            row[i] = EXPERTS ? a.order[at] : at;
            xs[i] = a.x_scales[EXPERTS ? x_row(a, row[i]) : at];
            ws[i] = a.w_scales[(int64_t)expert * a.n + c];
            bias[i] = !EXPERTS && a.bias ? (float)((const T*)a.bias)[c] : 0.f;
            if (EXPERTS && row[i] >= a.routes) row[i] = -1;
        }
        i32x4 acc[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) acc[i] = i32x4{0, 0, 0, 0};
        for (int s0 = wave; s0 < last; s0 += V * kAhead) {
            i32x4 wv[kAhead][NT][2], xv[kAhead][2];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int64_t at = (int64_t)(s0 + u * V) * 128;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const bool there = s0 + u * V < last && at + 32 * quarter + 16 * h < a.k;   // k is a multiple of 16
                    const int64_t off = at + 16 * h;
#pragma unroll
                    for (int i = 0; i < NT; ++i) wv[u][i][h] = *(const i32x4*)(there ? w[i] + off : (const int8_t*)kZeros);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const bool there = s0 + u * V < last && at + 32 * quarter + 16 * h < a.k;
                    xv[u][h] = *(const i32x4*)(there ? x + at + 16 * h : (const int8_t*)kZeros);
                }
            }
            // All at once, the halves of a line one after the other: left to itself the compiler asks for the last ones between the
            // products (one row by 3321 x 7408, eight waves: 6.3 us for 7.7), and with the halves apart 16 rows have lines twice
            // (9.6 us for 8.7).
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < NT; ++i) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[u][i][h], xv[u][h], acc[i], 0, 0, 0);
        }
        __syncthreads();                                    // the zeros are there
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) atomicAdd(&sums[r][16 * i + 4 * quarter + e], acc[i][e]);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            if (row[i] < 0) continue;
            const int o = threadIdx.x + 64 * V * i, c = n0 + o % kOuts;
            const float y = finish(sums[o / kOuts][o % kOuts], xs[i], ws[i], bias[i]);
            if (EXPERTS && a.products)
                a.products[(int64_t)row[i] * a.n + c] = y;
            else
                ((T*)a.y)[row[i] * a.y_stride + c] = (T)y;
        }
        __syncthreads();                                    // before the sums are cleared again
    }
}

}  // namespace w8
