// Causal attention over whole prompts: packed sequences of different lengths,
// grouped heads, keys and values in 16 bits: o = sum_t softmax_t(scale q.k_t) v_t.
//
// The matrix cores bound it.  A workgroup takes 128 queries of one head, a wave
// 32 of them, and walks over the keys 64 at a time with a running maximum and
// sum.  Scores come out transposed (keys x queries), so a lane keeps one
// query's statistics, half of its keys in the lane 32 further on, and its
// probabilities are already the second operand of the second product: the
// order of keys inside a product is free, and V, read across keys by the
// transposing LDS read, takes the order that the scores have.
#include <hip/hip_runtime.h>

#include "mx4.h"
#include "wino_device.h"
#include "winof4.h"

namespace {
using namespace mx4;

constexpr int kRows = 128, kKeys = 64;
constexpr float kNever = -__builtin_inff();

struct PromptArgs {
    const void *q, *k, *v;
    void* out;
    const int32_t *cu_q, *cu_k;
    int64_t q_stride, k_stride, v_stride;
    int32_t seqs, total_q, total_k, heads, kv_heads, causal;
    float scale_log2;       // |scale| * log2(e), 1 for a scale of 0: probabilities are powers of two
    uint32_t q_and, q_xor;  // the scale's sign, or its being 0, put into pairs of query elements
};

// A tile of K or V in LDS: 64 dense rows whose 16-byte pieces are exchanged inside a row, because copies from memory
// straight to LDS fill it from one end to the other.  The banks are 256 bytes wide.
template <int DIM> struct Shape {
    static constexpr int kRow = DIM * 2, kPiecesRow = kRow / 16;
    static constexpr int kTile = kKeys * kRow;
    // Wide heads: two waves share 32 queries, each with half the dimensions of the result.  Both work out the scores,
    // half again as many products in all, but the registers of one wave do not hold the whole result.
    static constexpr int kShare = DIM > 128 ? 2 : 1, kWaves = 4 * kShare, kOut = DIM / 32 / kShare;
    static constexpr int kPieces = kKeys * kPiecesRow / (64 * kWaves);  // of a tile, for a thread
    // K is read 16 rows at a time, the same piece of each: they have to stand in 16 different columns.  Of a row's
    // pieces, 2^kBits in a row can be exchanged.
    static constexpr int kBits = DIM == 96 ? 2 : (DIM == 64 || DIM == 192 ? 3 : 4);
    static __device__ int swap_k(int row) { return (row >> (4 - kBits)) & ((1 << kBits) - 1); }
    // V is read four rows at a time, 64 bytes of each: four different quarters of the banks.
    static __device__ int swap_v(int row) {
        return DIM == 96 ? 0 : (DIM == 64 || DIM == 192 ? (row >> 1 & 1) << 2 : (row & 3) << 2);
    }
};

// 16 bytes a lane from base + off to LDS at dst + 16 lane, which is on its way until vmcnt says otherwise; in assembly
// for the reason that lds_copy16 gives.
__device__ inline void copy16(const void* base, uint32_t off, uint32_t dst) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "{m0}"(dst) : "memory");
}

template <int TYPE> struct Mfma;
template <> struct Mfma<WINO_BF16> {
    typedef bf16x8 T8;
    typedef bf16x2 T2;
    static __device__ float pair_sum(T2 p, float c) {
        return __builtin_amdgcn_fdot2_f32_bf16(p, T2{(__bf16)1.f, (__bf16)1.f}, c, false);
    }
    static __device__ f32x16 mul(T8 a, T8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mfma<WINO_FP16> {
    typedef f16x8 T8;
    typedef f16x2 T2;
    static __device__ float pair_sum(T2 p, float c) {
        return __builtin_amdgcn_fdot2(p, T2{(_Float16)1.f, (_Float16)1.f}, c, false);
    }
    static __device__ f32x16 mul(T8 a, T8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

// The sequence and the tile of its queries that workgroup `index` takes, or false past the last.  Offsets are cut
// to the tensor.
struct Work {
    int q0, nq, k0, nk, tile;
};
__device__ inline bool find(const PromptArgs& a, int index, Work& w) {
    const int lane = threadIdx.x & 63;
    for (int s0 = 0; s0 < a.seqs; s0 += 64) {
        const int s = s0 + lane;
        int from = 0, n = 0;
        if (s < a.seqs) {
            from = max(a.cu_q[s], 0);
            n = max(min(a.cu_q[s + 1], a.total_q) - from, 0);
        }
        const int count = (n + kRows - 1) / kRows;
        int before = count;                                 // tiles of this and the sequences before, in the 64
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(before, o);
            if (lane >= o) before += x;
        }
        const int all = __shfl(before, 63);
        if (index < all) {
            const uint64_t past = __ballot(index < before);
            const int l = __builtin_ctzll(past);
            w.q0 = __shfl(from, l);
            w.nq = __shfl(n, l);
            w.tile = index - __shfl(before - count, l);
            w.k0 = max(min(a.cu_k[s0 + l], a.total_k), 0);
            w.nk = max(min(a.cu_k[s0 + l + 1], a.total_k) - w.k0, 0);
            return true;
        }
        index -= all;
    }
    return false;
}

template <int TYPE, int DIM>
__global__ __launch_bounds__(64 * Shape<DIM>::kWaves, 2) void prompt_attention_kernel(PromptArgs a) {
    typedef typename Half<TYPE>::type T;
    typedef Mfma<TYPE> M;
    typedef typename M::T8 T8;
    typedef typename M::T2 T2;
    typedef Shape<DIM> S;
    // probabilities are held 2^6 higher in fp16, whose small numbers end at 2^-24
    constexpr float kLift = TYPE == WINO_FP16 ? 6.f : 0.f;
    constexpr int kAhead = DIM <= 128 ? DIM / 8 : 8;    // pieces of K read before they are multiplied
    __shared__ __attribute__((aligned(256))) uint8_t lds[2][2 * S::kTile];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 31, half = lane >> 5, d0 = wave / 4 * (S::kOut * 32);      // d0: the wave's first dimension

    // workgroups that follow each other run on different XCDs: the heads that share a K and V are kv_heads apart, and
    // late tiles, which see the most keys, come first
    const int turn = blockIdx.x % a.heads;
    const int group = a.heads / a.kv_heads, kvh = turn % a.kv_heads, h = kvh * group + turn / a.kv_heads;
    const int tiles = gridDim.x / a.heads;
    Work w;
    if (!find(a, tiles - 1 - (int)(blockIdx.x / a.heads), w)) return;
    w.q0 = __builtin_amdgcn_readfirstlane(w.q0), w.nq = __builtin_amdgcn_readfirstlane(w.nq);
    w.k0 = __builtin_amdgcn_readfirstlane(w.k0), w.nk = __builtin_amdgcn_readfirstlane(w.nk);
    w.tile = __builtin_amdgcn_readfirstlane(w.tile);

    const int i0 = w.tile * kRows;                          // first query of the workgroup, in its sequence
    const int shift = a.causal ? w.nk - w.nq + 1 : w.nk;    // query i sees shift + i keys (all, where not causal)
    auto sees = [&](int i) { return max(0, a.causal ? min(shift + i, w.nk) : w.nk); };
    const int every = sees(i0);                             // keys that all rows of the workgroup see
    const int end = sees(min(i0 + kRows, w.nq) - 1);        // keys that some row sees
    const int iw = i0 + 32 * (wave % 4);
    const int wave_every = sees(iw), wave_end = iw < w.nq ? sees(min(iw + 32, w.nq) - 1) : 0;
    const int i = iw + c;                                   // this lane's query
    const int row_end = i < w.nq ? sees(i) : 0;

    T8 q[DIM / 16];
    {
        const T* p = (const T*)a.q + (int64_t)(w.q0 + min(i, w.nq - 1)) * a.q_stride + (int64_t)h * DIM + 8 * half;
#pragma unroll
        for (int s = 0; s < DIM / 16; ++s) {
            const u32x4 x = *(const u32x4*)(p + 16 * s);
            q[s] = __builtin_bit_cast(T8, (x & a.q_and) ^ a.q_xor);
        }
    }
    f32x16 o[S::kOut];                                      // lane: dimensions d0 + 32 n + 8 (e / 4) + 4 half + e % 4 of query c
#pragma unroll
    for (int n = 0; n < S::kOut; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[n][e] = 0.f;
    float ref = kNever, sum = 0.f;                          // ref: the power of two that o and sum are held against

    const T* kbase = (const T*)a.k + (int64_t)w.k0 * a.k_stride + (int64_t)kvh * DIM;
    const T* vbase = (const T*)a.v + (int64_t)w.k0 * a.v_stride + (int64_t)kvh * DIM;
    // pieces of a tile that this thread copies: where they come from
    uint32_t off_k[S::kPieces], off_v[S::kPieces];
    auto offsets = [&](int rows) {
#pragma unroll
        for (int x = 0; x < S::kPieces; ++x) {
            const int piece = threadIdx.x + 64 * S::kWaves * x, row = piece / S::kPiecesRow, at = piece % S::kPiecesRow;
            const int from = min(row, rows - 1);            // rows past the end: the last one again
            off_k[x] = (uint32_t)(from * (int)a.k_stride + (at ^ S::swap_k(row)) * 8) * 2u;
            off_v[x] = (uint32_t)(from * (int)a.v_stride + (at ^ S::swap_v(row)) * 8) * 2u;
        }
    };
    auto copy = [&](int t0, int buf) {
        if (t0 + kKeys > w.nk) offsets(w.nk - t0);
        const T* k = kbase + (int64_t)t0 * a.k_stride;
        const T* v = vbase + (int64_t)t0 * a.v_stride;
        const uint32_t dst = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds[buf] + wave * 1024;
#pragma unroll
        for (int x = 0; x < S::kPieces; ++x) {
            copy16(k, off_k[x], dst + x * (1024 * S::kWaves));
            copy16(v, off_v[x], dst + x * (1024 * S::kWaves) + S::kTile);
        }
    };
    offsets(kKeys);
    if (end > 0) copy(0, 0);
    int buf = 0;
    for (int t0 = 0; t0 < end; t0 += kKeys, buf ^= 1) {
        const uint8_t* lk = lds[buf];
        uint8_t* lv = lds[buf] + S::kTile;
        WINO_WAIT_VM_LDS(0);
        winof4::ring_barrier();                                     // the tile is there, and nobody reads the other one any more
        if (t0 + kKeys < end) copy(t0 + kKeys, buf ^ 1);    // on its way while this one is computed
        // A value that is not finite would spoil the rows that do not see its key too (0 times it is NaN): in tiles that
        // some row sees in part it leaves the product, and is added to the rows that see it.  Rows of V past the end go
        // as well.
        bool spoilt = false;
        if (t0 + kKeys > every) {
            constexpr uint32_t kExp = TYPE == WINO_BF16 ? 0x7f80u : 0x7c00u;
#pragma unroll
            for (int x = 0; x < S::kPieces; ++x) {
                const int piece = threadIdx.x + 64 * S::kWaves * x;
                u32x4 v = *(u32x4*)(lv + 16 * piece);
                const bool past = t0 + piece / S::kPiecesRow >= w.nk;
                bool bad = past;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t u = v[e];
                    const bool lo = past || (u & kExp) == kExp, hi = past || ((u >> 16) & kExp) == kExp;
                    bad = bad || lo || hi;
                    v[e] = (lo ? 0u : u & 0xffffu) | (hi ? 0u : u & 0xffff0000u);
                }
                if (bad) *(u32x4*)(lv + 16 * piece) = v;
                spoilt = spoilt || (bad && !past);
            }
            spoilt = __syncthreads_or(spoilt);
        }
        if (t0 >= wave_end) continue;
        // Addresses of a wave's pieces differ by exchanged bits.  Wide heads have no registers to keep them all: there
        // they are made anew from the row in each tile.
        int ck = c, lane_v = lane;
        if constexpr (DIM > 128) asm("" : "+v"(ck), "+v"(lane_v));

        f32x16 z[2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) z[b][e] = 0.f;
#pragma unroll
        for (int f0 = 0; f0 < DIM / 8; f0 += kAhead) {
            T8 k[kAhead];
#pragma unroll
            for (int f = 0; f < kAhead; ++f) {
                const int row = (f0 + f) / (DIM / 16) * 32 + ck, s = (f0 + f) % (DIM / 16);
                k[f] = *(const T8*)(lk + row * S::kRow + (((2 * s + half) ^ S::swap_k(row)) * 16));
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int f = 0; f < kAhead; ++f) {
                const int b = (f0 + f) / (DIM / 16);
                z[b] = M::mul(k[f], q[(f0 + f) % (DIM / 16)], z[b]);
            }
        }
        // the first half of V is read while the scores are turned into probabilities
        const int l = lane_v & 15, vrow = 4 * half + (l >> 2), piece = 2 * ((lane_v >> 4) & 1) + ((l & 3) >> 1);
        auto read_v = [&](int b, int s, T8 (&v)[S::kOut]) {
#pragma unroll
            for (int n = 0; n < S::kOut; ++n) {
                // lane l of 16 gives the address of four dimensions of key l / 4 and gets dimension l of four keys;
                // rows 8 apart exchange their pieces alike
                typedef __attribute__((ext_vector_type(4))) short s4;
                typedef __attribute__((address_space(3))) s4* lds4;
                const uint8_t* f = lv + (32 * b + 16 * s + vrow) * S::kRow + ((d0 / 8 + 4 * n + piece) ^ S::swap_v(vrow)) * 16 + (l & 1) * 8;
                const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)f));
                const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(f + 8 * S::kRow)));
                v[n] = __builtin_bit_cast(T8, u32x4{x[0], x[1], y[0], y[1]});
            }
        };
        T8 v[2][S::kOut];
        read_v(0, 0, v[0]);
        read_v(0, 1, v[1]);
        __builtin_amdgcn_sched_barrier(0);
        if (t0 + kKeys > wave_every) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (t0 + 32 * b + 8 * (e / 4) + 4 * half + e % 4 >= row_end) z[b][e] = kNever;
        }
        float top = max3(z[0][0], z[0][1], z[0][2]), top1 = max3(z[1][0], z[1][1], z[1][2]);
#pragma unroll
        for (int e = 3; e < 15; e += 2) {
            top = max3(z[0][e], z[0][e + 1], top);
            top1 = max3(z[1][e], z[1][e + 1], top1);
        }
        top = max3(top, z[0][15], top1);
        {
            const f32x2 x = swap_rows<2>(max3(top, top, z[1][15]));
            top = max3(x[0], x[1], x[1]) * a.scale_log2;
        }
        // o and sum move to a new reference only where the maximum has outgrown the old one by 2^8
        if (__any(top > ref + 8.f)) {
            const float to = __builtin_fmaxf(ref, top);
            const float alpha = to == kNever ? 1.f : __builtin_amdgcn_exp2f(ref - to);
            ref = to;
            sum *= alpha;
#pragma unroll
            for (int n = 0; n < S::kOut; ++n) o[n] *= alpha;
        }
        const float base = ref == kNever ? 0.f : kLift - ref;
        uint32_t p[2][8];
        float sum1 = 0.f;                                   // of the rounded probabilities: they are the weights
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const T2 x = {(T)__builtin_amdgcn_exp2f(__builtin_fmaf(z[b][e], a.scale_log2, base)),
                              (T)__builtin_amdgcn_exp2f(__builtin_fmaf(z[b][e + 1], a.scale_log2, base))};
                if (b == 0)
                    sum = M::pair_sum(x, sum);
                else
                    sum1 = M::pair_sum(x, sum1);
                p[b][e / 2] = __builtin_bit_cast(uint32_t, x);
            }
        sum += sum1;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const T8 pp = __builtin_bit_cast(T8, u32x4{p[b][4 * s], p[b][4 * s + 1], p[b][4 * s + 2], p[b][4 * s + 3]});
                if (b == 1) read_v(b, s, v[s]);
#pragma unroll
                for (int n = 0; n < S::kOut; ++n) o[n] = M::mul(v[s][n], pp, o[n]);
            }
        if (spoilt) {
            for (int t = t0; t < min(t0 + kKeys, row_end); ++t) {
                const T* v = vbase + (int64_t)t * a.v_stride + d0 + 4 * half;
#pragma unroll
                for (int n = 0; n < S::kOut; ++n) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float x = (float)v[32 * n + 8 * (e / 4) + e % 4];
                        if (!(__builtin_fabsf(x) < __builtin_inff())) o[n][e] += x;
                    }
                    __builtin_amdgcn_sched_barrier(0);      // a rare path: few registers rather than speed
                }
            }
        }
    }
    {
        const f32x2 x = swap_rows<2>(sum);
        sum = x[0] + x[1];
    }
    if (i < w.nq) {
        typedef T T4 __attribute__((ext_vector_type(4)));
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        T* out = (T*)a.out + ((int64_t)(w.q0 + i) * a.heads + h) * DIM + d0 + 4 * half;
#pragma unroll
        for (int n = 0; n < S::kOut; ++n)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *(T4*)(out + 32 * n + 2 * e) =
                    sum == 0.f ? T4{} : T4{(T)(o[n][e] * inv), (T)(o[n][e + 1] * inv), (T)(o[n][e + 2] * inv), (T)(o[n][e + 3] * inv)};
    }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

template <int TYPE, int DIM> void launch(dim3 grid, hipStream_t stream, const PromptArgs& a) {
    hipLaunchKernelGGL((prompt_attention_kernel<TYPE, DIM>), grid, dim3(64 * Shape<DIM>::kWaves), 0, stream, a);
}
template <int TYPE> void launch_dim(int dim, dim3 grid, hipStream_t stream, const PromptArgs& a) {
    switch (dim) {
        case 64: return launch<TYPE, 64>(grid, stream, a);
        case 96: return launch<TYPE, 96>(grid, stream, a);
        case 128: return launch<TYPE, 128>(grid, stream, a);
        case 192: return launch<TYPE, 192>(grid, stream, a);
        default: return launch<TYPE, 256>(grid, stream, a);
    }
}

}  // namespace

extern "C" wino_status prompt_attention(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                        const void* v, int64_t v_stride, const int32_t* cu_q, const int32_t* cu_k,
                                        int32_t seqs, int32_t total_q, int32_t total_k, int32_t max_q, int32_t heads,
                                        int32_t kv_heads, int32_t head_dim, float scale, int32_t causal, void* out,
                                        wino_float_type type, hipStream_t stream) {
    if (type != WINO_BF16 && type != WINO_FP16) return WINO_EINVAL;
    if (seqs < 0 || total_q < 0 || total_k < 0 || max_q < 0 || heads < 1 || kv_heads < 1 || head_dim < 1) return WINO_EINVAL;
    if (heads % kv_heads || (causal != 0 && causal != 1) || !(scale == scale) || scale - scale != 0.f) return WINO_EINVAL;
    if (head_dim != 64 && head_dim != 96 && head_dim != 128 && head_dim != 192 && head_dim != 256)
        return WINO_EUNSUPPORTED;
    if (seqs > 65536 || heads > 65536 || total_q > 0x7fffffff - 4096 || total_k > 0x7fffffff - 4096) return WINO_EUNSUPPORTED;
    if (total_q == 0 || seqs == 0) return WINO_OK;
    if (!q || !out || (total_k > 0 && (!k || !v)) || !cu_q || !cu_k) return WINO_EINVAL;
    const int64_t dim = head_dim;
    if ((total_q > 1 && q_stride < heads * dim) || (total_k > 1 && (k_stride < kv_heads * dim || v_stride < kv_heads * dim)))
        return WINO_EINVAL;
    if (total_k > 1 && (k_stride > 1 << 24 || v_stride > 1 << 24)) return WINO_EUNSUPPORTED;
    if ((total_q > 1 && (q_stride & 7)) || (total_k > 1 && ((k_stride | v_stride) & 7)) ||
        !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out))
        return WINO_EUNSUPPORTED;
    // whole tiles, and one started by each sequence
    const int64_t blocks = ((int64_t)total_q / kRows + seqs) * heads;
    if (blocks > 0x7fffffffll) return WINO_EUNSUPPORTED;
    PromptArgs a = {q, k, v, out, cu_q, cu_k, q_stride, k_stride, v_stride, seqs, total_q, total_k,
                    heads, kv_heads, causal, 0.f, scale == 0.f ? 0u : 0xffffffffu, scale < 0.f ? 0x80008000u : 0u};
    a.scale_log2 = scale == 0.f ? 1.f : __builtin_fabsf(scale) * 1.44269504088896340736f;
    if (a.scale_log2 - a.scale_log2 != 0.f) return WINO_EUNSUPPORTED;       // past fp32's range
    if (type == WINO_BF16)
        launch_dim<WINO_BF16>(head_dim, dim3((unsigned)blocks), stream, a);
    else
        launch_dim<WINO_FP16>(head_dim, dim3((unsigned)blocks), stream, a);
    return hipGetLastError() == hipSuccess ? WINO_OK : WINO_EHIP;
}
