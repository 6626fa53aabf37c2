// Causal attention over whole prompts: packed sequences of different lengths,
// grouped heads, keys and values in 16 bits: o = sum_t softmax_t(scale q.k_t) v_t.
//
// The matrix cores bound it.  The heads that share K and V are rows of the same
// tile, one query's heads next to each other: a tile of 128 rows then spans few
// queries, whose masks differ little, and short sequences fill it.  A workgroup
// takes such a tile, a wave 32 rows of it, and walks over the keys 64 at a time
// with a running maximum and sum.  Scores come out transposed (keys x rows), so
// a lane keeps one row's statistics, half of its keys in the lane 32 further
// on, and its probabilities are already the second operand of the second
// product: the order of keys inside a product is free, and V, read across keys
// by the transposing LDS read, takes the order that the scores have.
//
// Where there are too few tiles for the device, teams of waves share out the
// keys of one tile and are joined in LDS at the end.
//
// Precision: probabilities are rounded to the type of q, k and v for the second
// product (fp16 ones held 2^6 higher, clear of its smallest numbers), and their
// sum is that of the rounded ones, so that the weights of a row add up to 1.
//
// One sequence of 16384 tokens, 16 heads of 128 on 4: 1010 to 1030 us on most
// devices, 1.07 to 1.09 PFLOP/s (a large library product of the same type: 1.25 to
// 1.38); the matrix cores work 57% of the cycles, at the clock that this load leaves
// (1.6 to 1.8 GHz).  Twelve packed ones of up to 2048, 32 heads on 8: 143 to 150 us,
// 0.74 to 0.78 PFLOP/s, 40%: their workgroups walk over eight tiles on average, and
// begin and end in between.  Both once the clock has settled: the first hundred
// calls of a burst take 1035 to 1050 and 167 us on average.
// Heads of 256: four sequences of 4096, 16 heads on 4, 659 us, 0.84 PFLOP/s.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "mx4.h"
#include "wino_device.h"
#include "winof4.h"

namespace {
using namespace mx4;

constexpr float kNever = -__builtin_inff();

struct PromptArgs {
    const void *q, *k, *v;
    void* out;
    const int32_t *cu_q, *cu_k;
    int64_t q_stride, k_stride, v_stride;
    int32_t seqs, total_q, total_k, heads, kv_heads, group, causal;
    winof4::FastDiv by_group;
    float scale_log2;       // |scale| * log2(e), 1 for a scale of 0: probabilities are powers of two
    uint32_t q_and, q_xor;  // the scale's sign, or its being 0, put into pairs of query elements
};

// A workgroup: TEAMS teams that share out the keys, each with ROWS / 32 row blocks, a wave (or two) each, and KEYS keys
// at a time.
//
// A tile of K or V in LDS is dense rows whose 16-byte pieces are exchanged inside a row, because copies from memory
// straight to LDS fill it from one end to the other.  The banks are 256 bytes wide.
template <int DIM, int ROWS, int TEAMS, int KEYS> struct Shape {
    static constexpr int kRow = DIM * 2, kPiecesRow = kRow / 16;
    static constexpr int kTile = KEYS * kRow;
    // Wide heads: two waves share 32 rows, each with half the dimensions of the result, because the registers of one wave
    // do not hold the whole.  Where a tile has two blocks of 32 keys (kSplit), each works out the probabilities of one
    // and they exchange them in LDS; else both work out all scores, half again as many products.
    static constexpr int kShare = DIM > 128 ? 2 : 1, kOut = DIM / 32 / kShare;
    static constexpr bool kSplit = kShare == 2 && KEYS == 64;
    static constexpr int kBlocks = ROWS / 32, kTeam = kBlocks * kShare, kWaves = kTeam * TEAMS;
    static constexpr int kPieces = KEYS * kPiecesRow / (64 * kTeam);    // of a tile, for a thread
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

// The sequence and the tile of its rows that workgroup `index` takes, or false where it has none.  Those that see the most
// keys come first, so that the device is full to the end: among each 64 sequences the longest one's tiles, from its end
// to its beginning, then the next one's.  Offsets are cut to the tensor.
//
// The 64 sequences from 64 g on begin at workgroup first(g): whole tiles of the rows before them, and one for each
// sequence before them, which is room for their last tiles.  So nobody counts the tiles of other sequences, and the work
// grows with the number of sequences, not its square (4096 of 64 tokens, 16 heads of 128 on 4: 0.97 ms; with all counted
// by each workgroup 23.2).
struct Work {
    int q0, nq, k0, nk, tile;
};
template <int ROWS> __device__ inline bool find(const PromptArgs& a, int index, Work& w) {
    const int lane = threadIdx.x & 63;
    int s0 = 0;
    if (a.seqs > 64) {
        const int sets = (a.seqs + 63) / 64;
        auto first = [&](int g) { return g == 0 ? 0 : min(max(a.cu_q[64 * g], 0), a.total_q) * a.group / ROWS + 64 * g; };
        // the last set that begins at index or before it: of every step-th one, then of those that follow it
        const int step = (sets + 63) / 64;                  // 16 at most
        auto last = [&](int from, int apart, int lanes) {
            const int g = from + lane * apart;
            const uint64_t begun = __ballot(lane < lanes && g < sets && first(min(g, sets - 1)) <= index);
            return from + (63 - __builtin_clzll(begun | 1)) * apart;
        };
        int g = last(0, step, 64);
        if (step > 1) g = last(g, 1, step);
        s0 = 64 * g;
        index -= first(g);
    }
    const int s = s0 + lane;
    int from = 0, n = 0, k0 = 0, k1 = 0;
    if (s < a.seqs) {
        from = max(a.cu_q[s], 0);
        n = max(max(min(a.cu_q[s + 1], a.total_q), 0) - from, 0);
        k0 = max(min(a.cu_k[s], a.total_k), 0);
        k1 = max(min(a.cu_k[s + 1], a.total_k), 0);
    }
    const int count = (n * a.group + ROWS - 1) / ROWS;
    // the 64 sequences by their keys, the longest first: tiles before this lane's, and all of them
    const int keys = k1 - k0;
    int before = 0, all = 0;
    for (int j = 0; j < min(64, a.seqs - s0); ++j) {
        const int other = __builtin_amdgcn_readlane(keys, j), tiles = __builtin_amdgcn_readlane(count, j);
        before += other > keys || (other == keys && j < lane) ? tiles : 0;
        all += tiles;
    }
    if (index < 0 || index >= all) return false;
    const int l = __builtin_ctzll(__ballot(index >= before && index < before + count));
    w.q0 = __shfl(from, l);
    w.nq = __shfl(n, l);
    w.tile = __shfl(before + count, l) - 1 - index;
    w.k0 = __shfl(k0, l);
    w.nk = max(__shfl(keys, l), 0);
    return true;
}

template <int TYPE, int DIM, int ROWS, int TEAMS, int KEYS>
__global__ __launch_bounds__((64 * Shape<DIM, ROWS, TEAMS, KEYS>::kWaves), 2) void prompt_attention_kernel(PromptArgs a) {
    typedef typename Half<TYPE>::type T;
    typedef Mfma<TYPE> M;
    typedef typename M::T8 T8;
    typedef typename M::T2 T2;
    typedef Shape<DIM, ROWS, TEAMS, KEYS> S;
    constexpr int kB = KEYS / 32, kMine = S::kSplit ? 1 : kB;   // 32-key blocks of a tile, and those whose scores a wave takes
    // probabilities are held 2^6 higher in fp16, whose small numbers end at 2^-24
    constexpr float kLift = TYPE == WINO_FP16 ? 6.f : 0.f;
    constexpr int kAhead = DIM <= 128 ? kB * DIM / 16 : (DIM == 192 ? 12 : 8);
    static_assert(kMine * DIM / 16 % kAhead == 0, "whole groups");  // pieces of K read before they are multiplied
    __shared__ __attribute__((aligned(256))) uint8_t lds[TEAMS][2][2 * S::kTile];
    constexpr int kXWaves = S::kSplit ? S::kWaves : 1;      // what the waves of a pair exchange, and who has outgrown ref
    __shared__ u32x4 p_lds[kXWaves][2][64];
    __shared__ float top_lds[kXWaves][64];
    __shared__ uint32_t grown[kXWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 31, half = lane >> 5;
    const int team = wave / S::kTeam, mate = wave % S::kTeam, d0 = mate / S::kBlocks * (S::kOut * 32);   // d0: first dimension
    // kSplit: the block of keys that is this wave's, and the wave that has the other one (TEAMS is 1)
    const int mine = S::kSplit ? mate / S::kBlocks : 0, partner = S::kSplit ? wave ^ S::kBlocks : 0;
    auto meet = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // what was written to LDS; the next tile stays on its way
        winof4::ring_barrier();
    };

    // Workgroups that follow each other run on different XCDs: a K and V stays with one or two of them.
    const int kvh = blockIdx.x % a.kv_heads;
    Work w;
    if (!find<ROWS>(a, blockIdx.x / a.kv_heads, w)) return;
    w.q0 = __builtin_amdgcn_readfirstlane(w.q0), w.nq = __builtin_amdgcn_readfirstlane(w.nq);
    w.k0 = __builtin_amdgcn_readfirstlane(w.k0), w.nk = __builtin_amdgcn_readfirstlane(w.nk);
    w.tile = __builtin_amdgcn_readfirstlane(w.tile);

    // row r is query r / group, head r % group of the heads at kvh
    const int rows = w.nq * a.group, r0 = w.tile * ROWS, rw = r0 + 32 * (mate % S::kBlocks);
    const int shift = a.causal ? w.nk - w.nq + 1 : w.nk;    // query i sees shift + i keys (all, where not causal)
    auto sees = [&](int row) {
        const int i = (int)winof4::fast_div((uint32_t)row, a.by_group);
        return max(0, a.causal ? min(shift + i, w.nk) : w.nk);
    };
    const int every = sees(r0);                             // keys that all rows of the workgroup see
    const int end = sees(min(r0 + ROWS, rows) - 1);         // keys that some row sees
    const int wave_every = sees(rw), wave_end = rw < rows ? sees(min(rw + 32, rows) - 1) : 0;
    const bool real = rw + c < rows;
    const int row = real ? rw + c : rows - 1;               // this lane's row
    const int i = (int)winof4::fast_div((uint32_t)row, a.by_group), h = kvh * a.group + row - i * a.group;
    const int row_end = real ? sees(row) : 0;

    T8 q[DIM / 16];
    {
        const T* p = (const T*)a.q + (int64_t)(w.q0 + i) * a.q_stride + (int64_t)h * DIM + 8 * half;
#pragma unroll
        for (int s = 0; s < DIM / 16; ++s) {
            const u32x4 x = *(const u32x4*)(p + 16 * s);
            q[s] = __builtin_bit_cast(T8, (x & a.q_and) ^ a.q_xor);
        }
    }
    f32x16 o[S::kOut];                                      // lane: dimensions d0 + 32 n + 8 (e / 4) + 4 half + e % 4 of its row
#pragma unroll
    for (int n = 0; n < S::kOut; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[n][e] = 0.f;
    float ref = kNever, sum = 0.f;                          // ref: the power of two that o and sum are held against

    const T* kbase = (const T*)a.k + (int64_t)w.k0 * a.k_stride + (int64_t)kvh * DIM;
    const T* vbase = (const T*)a.v + (int64_t)w.k0 * a.v_stride + (int64_t)kvh * DIM;
    // pieces of a tile that this thread copies: where they come from
    const int member = threadIdx.x - team * (64 * S::kTeam);
    uint32_t off_k[S::kPieces], off_v[S::kPieces];
    auto offsets = [&](int keys) {
#pragma unroll
        for (int x = 0; x < S::kPieces; ++x) {
            const int piece = member + 64 * S::kTeam * x, key = piece / S::kPiecesRow, at = piece % S::kPiecesRow;
            const int from = min(key, keys - 1);            // rows past the end: the last one again
            off_k[x] = (uint32_t)(from * (int)a.k_stride + (at ^ S::swap_k(key)) * 8) * 2u;
            off_v[x] = (uint32_t)(from * (int)a.v_stride + (at ^ S::swap_v(key)) * 8) * 2u;
        }
    };
    auto copy = [&](int t0, int buf) {
        if (t0 >= end) return;
        if (t0 + KEYS > w.nk) offsets(w.nk - t0);
        const T* k = kbase + (int64_t)t0 * a.k_stride;
        const T* v = vbase + (int64_t)t0 * a.v_stride;
        const uint32_t dst = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds[team][buf] + mate * 1024;
#pragma unroll
        for (int x = 0; x < S::kPieces; ++x) {
            copy16(k, off_k[x], dst + x * (1024 * S::kTeam));
            copy16(v, off_v[x], dst + x * (1024 * S::kTeam) + S::kTile);
        }
    };
    offsets(KEYS);
    copy(team * KEYS, 0);
    int buf = 0;
    for (int step = 0; step < end; step += TEAMS * KEYS, buf ^= 1) {
        const int t0 = step + team * KEYS;                  // the team's tile
        const uint8_t* lk = lds[team][buf];
        uint8_t* lv = lds[team][buf] + S::kTile;
        WINO_WAIT_VM_LDS(0);
        winof4::ring_barrier();                             // the tile is there, and nobody reads the other one any more
        copy(t0 + TEAMS * KEYS, buf ^ 1);                   // on its way while this one is computed
        // A value that is not finite would spoil the rows that do not see its key too (0 times it is NaN): in tiles that
        // some row sees in part it leaves the product, and is added to the rows that see it.  Rows of V past the end go
        // as well.
        bool spoilt = false;
        if (step + TEAMS * KEYS > every) {
            constexpr uint32_t kExp = TYPE == WINO_BF16 ? 0x7f80u : 0x7c00u;
            if (t0 < end) {
#pragma unroll
                for (int x = 0; x < S::kPieces; ++x) {
                    const int piece = member + 64 * S::kTeam * x;
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
            }
            spoilt = __syncthreads_or(spoilt);
        }
        const bool busy = t0 < wave_end;                    // both waves of a pair alike
        if (!S::kSplit && !busy) continue;
        // Addresses of a wave's pieces differ by exchanged bits.  Wide heads have no registers to keep them all: there
        // they are made anew from the row in each tile.
        int ck = c, lane_v = lane;
        if constexpr (DIM > 128) asm("" : "+v"(ck), "+v"(lane_v));

        f32x16 z[kMine];
#pragma unroll
        for (int b = 0; b < kMine; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) z[b][e] = 0.f;
        if (busy) {
#pragma unroll
            for (int f0 = 0; f0 < kMine * DIM / 16; f0 += kAhead) {
                T8 k[kAhead];
#pragma unroll
                for (int f = 0; f < kAhead; ++f) {
                    const int key = (mine + (f0 + f) / (DIM / 16)) * 32 + ck, s = (f0 + f) % (DIM / 16);
                    k[f] = *(const T8*)(lk + key * S::kRow + (((2 * s + half) ^ S::swap_k(key)) * 16));
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int f = 0; f < kAhead; ++f) {
                    const int b = (f0 + f) / (DIM / 16);
                    z[b] = M::mul(k[f], q[(f0 + f) % (DIM / 16)], z[b]);
                }
            }
        }
        // the first half of V is read while the scores are turned into probabilities
        const int l = lane_v & 15, vkey = 4 * half + (l >> 2), piece = 2 * ((lane_v >> 4) & 1) + ((l & 3) >> 1);
        auto read_v = [&](int b, int s, T8 (&v)[S::kOut]) {
#pragma unroll
            for (int n = 0; n < S::kOut; ++n) {
                // lane l of 16 gives the address of four dimensions of key l / 4 and gets dimension l of four keys;
                // rows 8 apart exchange their pieces alike
                typedef __attribute__((ext_vector_type(4))) short s4;
                typedef __attribute__((address_space(3))) s4* lds4;
                const uint8_t* f = lv + (32 * b + 16 * s + vkey) * S::kRow + ((d0 / 8 + 4 * n + piece) ^ S::swap_v(vkey)) * 16 + (l & 1) * 8;
                const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)f));
                const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(f + 8 * S::kRow)));
                v[n] = __builtin_bit_cast(T8, u32x4{x[0], x[1], y[0], y[1]});
            }
        };
        T8 v[2][S::kOut];
        read_v(mine, 0, v[0]);
        read_v(mine, 1, v[1]);
        __builtin_amdgcn_sched_barrier(0);
        if (t0 + KEYS > wave_every) {
#pragma unroll
            for (int b = 0; b < kMine; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (t0 + 32 * (mine + b) + 8 * (e / 4) + 4 * half + e % 4 >= row_end) z[b][e] = kNever;
        }
        float part[kMine];
#pragma unroll
        for (int b = 0; b < kMine; ++b) {
            part[b] = max3(z[b][0], z[b][1], z[b][2]);
#pragma unroll
            for (int e = 3; e < 15; e += 2) part[b] = max3(z[b][e], z[b][e + 1], part[b]);
            part[b] = max3(part[b], z[b][15], part[0]);
        }
        float top;
        {
            const f32x2 x = swap_rows<2>(part[kMine - 1]);
            top = max3(x[0], x[1], x[1]) * a.scale_log2;
        }
        // o and sum move to a new reference only where the maximum has outgrown the old one by 2^8
        auto outgrow = [&](float by) {
            const float to = __builtin_fmaxf(ref, by);
            const float alpha = to == kNever ? 1.f : __builtin_amdgcn_exp2f(ref - to);
            ref = to;
            sum *= alpha;
#pragma unroll
            for (int n = 0; n < S::kOut; ++n) o[n] *= alpha;
        };
        uint32_t p[kB][8];                                  // kSplit: this wave's block first
        float add[kMine];                                   // the rounded probabilities: they are the weights
        auto weigh = [&]() {
            const float base = ref == kNever ? 0.f : kLift - ref;
#pragma unroll
            for (int b = 0; b < kMine; ++b) {
                add[b] = 0.f;
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const T2 x = {(T)__builtin_amdgcn_exp2f(__builtin_fmaf(z[b][e], a.scale_log2, base)),
                                  (T)__builtin_amdgcn_exp2f(__builtin_fmaf(z[b][e + 1], a.scale_log2, base))};
                    add[b] = M::pair_sum(x, add[b]);
                    p[b][e / 2] = __builtin_bit_cast(uint32_t, x);
                }
            }
        };
        if constexpr (!S::kSplit) {
            if (__any(top > ref + 8.f)) outgrow(top);
            weigh();
        } else {
            // Both waves of a pair hold the same reference.  Hardly ever has a maximum outgrown it: the probabilities are
            // worked out and handed over as if none had, and again where one has.
            auto hand_over = [&]() {
                weigh();
#pragma unroll
                for (int x = 0; x < 2; ++x) p_lds[wave][x][lane] = u32x4{p[0][4 * x], p[0][4 * x + 1], p[0][4 * x + 2], p[0][4 * x + 3]};
            };
            const bool grows = busy && __any(top > ref + 8.f);
            if (busy && !grows) hand_over();
            if (lane == 0) grown[wave] = grows;
            meet();
            if (__any(lane < S::kWaves && grown[lane % kXWaves] != 0)) {
                top_lds[wave][lane] = top;
                meet();
                if (busy) {
                    outgrow(__builtin_fmaxf(top, top_lds[partner][lane]));
                    hand_over();
                }
                meet();
            }
            if (!busy) continue;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const u32x4 y = p_lds[partner][x][lane];
#pragma unroll
                for (int k = 0; k < 4; ++k) p[kB - 1][4 * x + k] = y[k];
            }
        }
#pragma unroll
        for (int b = 0; b < kMine; ++b) sum += add[b];
#pragma unroll
        for (int b = 0; b < kB; ++b)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const T8 pp = __builtin_bit_cast(T8, u32x4{p[b][4 * s], p[b][4 * s + 1], p[b][4 * s + 2], p[b][4 * s + 3]});
                if (b > 0) read_v(S::kSplit ? 1 - mine : b, s, v[s]);
#pragma unroll
                for (int n = 0; n < S::kOut; ++n) o[n] = M::mul(v[s][n], pp, o[n]);
            }
        if (spoilt) {
            for (int t = t0; t < min(t0 + KEYS, row_end); ++t) {
                const T* x = vbase + (int64_t)t * a.v_stride + d0 + 4 * half;
#pragma unroll
                for (int n = 0; n < S::kOut; ++n) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float y = (float)x[32 * n + 8 * (e / 4) + e % 4];
                        if (!(__builtin_fabsf(y) < __builtin_inff())) o[n][e] += y;
                    }
                    __builtin_amdgcn_sched_barrier(0);      // a rare path: few registers rather than speed
                }
            }
        }
    }
    // the upper half of the teams hands over to the lower half, until one is left
#pragma unroll
    for (int left = TEAMS / 2; left > 0; left /= 2) {
        if (end <= left * KEYS) continue;                   // that half had no keys
        float* at = (float*)lds + ((team % left) * S::kTeam + mate) * (S::kOut * 16 + 2) * 64 + lane;
        __syncthreads();
        if (team >= left && team < 2 * left) {
#pragma unroll
            for (int n = 0; n < S::kOut; ++n)
#pragma unroll
                for (int e = 0; e < 16; ++e) at[(n * 16 + e) * 64] = o[n][e];
            at[S::kOut * 16 * 64] = ref;
            at[(S::kOut * 16 + 1) * 64] = sum;
        }
        __syncthreads();
        if (team < left) {
            const float other = at[S::kOut * 16 * 64], to = __builtin_fmaxf(ref, other), base = to == kNever ? 0.f : to;
            const float mine = __builtin_amdgcn_exp2f(ref - base), theirs = __builtin_amdgcn_exp2f(other - base);
            ref = to;
            sum = sum * mine + at[(S::kOut * 16 + 1) * 64] * theirs;
#pragma unroll
            for (int n = 0; n < S::kOut; ++n)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[n][e] = o[n][e] * mine + at[(n * 16 + e) * 64] * theirs;
        }
    }
    {
        const f32x2 x = swap_rows<2>(sum);
        sum = x[0] + x[1];
    }
    if constexpr (S::kSplit) {                              // the other wave's keys
        __syncthreads();
        top_lds[wave][lane] = sum;
        __syncthreads();
        const float other = top_lds[partner][lane];
        sum = mine == 0 ? sum + other : other + sum;
    }
    if (team == 0) {
        // the halves of the wave exchange four dimensions of sixteen, so that a lane stores eight neighbours
        // a row that sees keys has a sum, or scores that are all minus infinity and is not a number (0 times infinity)
        const float inv = 1.f / sum;
        T* out = (T*)a.out + ((int64_t)(w.q0 + i) * a.heads + h) * DIM + d0 + 8 * half;
#pragma unroll
        for (int n = 0; n < S::kOut; ++n)
#pragma unroll
            for (int e = 0; e < 16; e += 8) {
                uint32_t y[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const T2 x = {(T)(o[n][e + 2 * k] * inv), (T)(o[n][e + 2 * k + 1] * inv)};
                    y[k] = row_end == 0 ? 0u : __builtin_bit_cast(uint32_t, x);
                }
                const auto s02 = __builtin_amdgcn_permlane32_swap(y[0], y[2], false, false);
                const auto s13 = __builtin_amdgcn_permlane32_swap(y[1], y[3], false, false);
                if (real) *(u32x4*)(out + 32 * n + 2 * e) = u32x4{s02[0], s13[0], s02[1], s13[1]};
            }
    }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Workgroups for tiles of `rows` rows: whole tiles, and one started by each sequence.
int64_t tiles(const PromptArgs& a, int rows) { return ((int64_t)a.total_q * a.group / rows + a.seqs) * a.kv_heads; }

template <int TYPE, int DIM, int ROWS, int TEAMS, int KEYS> wino_status launch(const PromptArgs& a, hipStream_t stream) {
    const int64_t blocks = tiles(a, ROWS);
    constexpr int kThreads = 64 * Shape<DIM, ROWS, TEAMS, KEYS>::kWaves;
    if (blocks * kThreads > 0xffffffffll) return WINO_EUNSUPPORTED;         // of a launch
    hipLaunchKernelGGL((prompt_attention_kernel<TYPE, DIM, ROWS, TEAMS, KEYS>), dim3((unsigned)blocks), dim3(kThreads), 0,
                       stream, a);
    return hipGetLastError() == hipSuccess ? WINO_OK : WINO_EHIP;
}
// Tiles of 128 rows by one team once they fill the device twice over (more than once for wide heads, whose workgroups
// take a whole compute unit); before that 64 rows by two teams, and by four where the keys are many and the tiles very few.  Heads of
// 128, causal, us for one team of 128 / two of 64 / four of 64:
//   1 x 256, 16 heads (32 tiles) 11.8 / 9.8 / 11.2      1 x 512 on 4096 keys, 8 heads (32) 80 / 53 / 44
//   1 x 1024, 16 heads (128) 26.0 / 19.4 / 19.0         1 x 2048, 16 heads (256) 45 / 35 / 38
//   4 x 512, 32 heads (512) 25.6 / 27.3 / 42.9          8 x 512, 32 heads (1024) 41 / 49 / 84
// and of 256 for one / two: 1 x 1700, 16 heads (216) 67 / 56, 1 x 2048 (256) 80 / 72, 1 x 2500 (316) 94 / 108.
template <int TYPE, int DIM> wino_status pick(const PromptArgs& a, int max_q, hipStream_t stream) {
    // tiles of 128 rows that have something to do, by the longest sequence's length
    const int64_t busy = std::min(tiles(a, 128), (((int64_t)max_q * a.group + 127) / 128) * a.seqs * a.kv_heads);
    if (busy >= (DIM > 128 ? 257 : 512)) return launch<TYPE, DIM, 128, 1, 64>(a, stream);
    if constexpr (DIM <= 128)
        if (busy <= 128 && a.total_k / a.seqs >= 1024) return launch<TYPE, DIM, 64, 4, 32>(a, stream);
    return launch<TYPE, DIM, 64, 2, 32>(a, stream);
}
template <int TYPE> wino_status launch_dim(int dim, const PromptArgs& a, int max_q, hipStream_t stream) {
    switch (dim) {
        case 64: return pick<TYPE, 64>(a, max_q, stream);
        case 96: return pick<TYPE, 96>(a, max_q, stream);
        case 128: return pick<TYPE, 128>(a, max_q, stream);
        case 192: return pick<TYPE, 192>(a, max_q, stream);
        default: return pick<TYPE, 256>(a, max_q, stream);
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
    if ((int64_t)total_q * (heads / kv_heads) > 0x7fffffff - 4096) return WINO_EUNSUPPORTED;     // rows are counted in 32 bits
    if (total_q == 0 || seqs == 0) return WINO_OK;
    if (!q || !out || (total_k > 0 && (!k || !v)) || !cu_q || !cu_k) return WINO_EINVAL;
    const int64_t dim = head_dim;
    if ((total_q > 1 && q_stride < heads * dim) || (total_k > 1 && (k_stride < kv_heads * dim || v_stride < kv_heads * dim)))
        return WINO_EINVAL;
    if (total_k > 1 && (k_stride > 1 << 24 || v_stride > 1 << 24)) return WINO_EUNSUPPORTED;
    if ((total_q > 1 && (q_stride & 7)) || (total_k > 1 && ((k_stride | v_stride) & 7)) ||
        !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out))
        return WINO_EUNSUPPORTED;
    PromptArgs a = {q, k, v, out, cu_q, cu_k, q_stride, k_stride, v_stride, seqs, total_q, total_k,
                    heads, kv_heads, heads / kv_heads, causal, winof4::make_fastdiv((uint32_t)(heads / kv_heads)), 0.f,
                    scale == 0.f ? 0u : 0xffffffffu, scale < 0.f ? 0x80008000u : 0u};
    a.scale_log2 = scale == 0.f ? 1.f : __builtin_fabsf(scale) * 1.44269504088896340736f;
    if (a.scale_log2 - a.scale_log2 != 0.f) return WINO_EUNSUPPORTED;       // past fp32's range
    return type == WINO_BF16 ? launch_dim<WINO_BF16>(head_dim, a, max_q, stream)
                             : launch_dim<WINO_FP16>(head_dim, a, max_q, stream);
}
