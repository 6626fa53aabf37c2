// Attention over the paged 4-bit cache (mx4.h) for one or a few query tokens
// of each sequence: o = sum_t softmax_t(scale q.k_t) v_t.
//
// The bytes of the cache bound it, so one pass reads each once, for up to 16
// query rows (the heads that share a cache head, times the query tokens) at a
// time.  A wave takes 16-token tiles: K codes go from global memory straight to
// the registers of the matrix cores' first operand (a lane holds a quarter of
// one token's head: consecutive bytes, one or two scales), two codes an
// instruction, exact in bf16.  Scores come out transposed (tokens x rows), so
// a lane keeps one row's statistics and its probabilities are already where
// the second product wants them; that product's V must be read across tokens,
// which LDS does: V is written there token by token and read back transposed.
// The order of tokens inside a product is free, so V takes the order that the
// scores have.  Each wave has its own part of LDS and its own running maximum
// and sum; the waves, and the parts of a split sequence, are joined at the end.
//
// Precision: queries in fp16 and all probabilities are split into two bf16
// numbers (16 bits), the matrix cores have time for both; the products are
// then exact in fp32.
//
// 32 heads of 128 on 8, bf16: two sequences of 131072 tokens, 157 MB of cache,
// take 39.5 us, 35 of them this kernel (4.5 TB/s, of 4.8 that a copy of 2 GiB
// reaches); 64 sequences of 1 to 4096 tokens, 81 MB, 22 us (3.7 TB/s) and 4.6 for
// the join: their many short units cost a wait for the first codes each.  In fp16
// the two take 50.6 us, and the 64 with the append 37.2 instead of 31.0: queries
// take twice the registers and score products, and 14 registers are spilled under
// the limit of three workgroups a compute unit.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "mx4.h"
#include "wino_device.h"
#include "winof4.h"

namespace {
using namespace mx4;
using winof4::FastDiv;

constexpr int kBlock = 256;                 // tokens that the work is shared out in
constexpr int kGroups = 768;                // workgroups that fit on the device at once (heads up to 128)
constexpr float kNever = -__builtin_inff();

struct DecodeArgs {
    const void* q;
    void* out;
    const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    const int32_t *table, *lens;
    float* part;            // [2 * workgroups][16][dim] sums of parts, then [2 * workgroups][16][2] their references and
                            // totals, then [batch * units] where a unit's parts are; null: a workgroup takes a whole unit
    int64_t q_stride, pages;
    int32_t q_len, heads, kv_heads, group, page, max_pages;
    int32_t tiles;          // 16-row tiles of a sequence's rows at one cache head
    int32_t batch;
    int32_t units;          // of a sequence: kv_heads * tiles
    int32_t groups;         // workgroups
    int32_t room;           // tokens that a table has room for
    FastDiv by_page, by_group, by_tiles, by_units, by_heads, by_q;
    float scale_log2;       // |scale| * log2(e), 1 for a scale of 0: probabilities are powers of two
    uint32_t q_and, q_xor;  // the scale's sign, or its being 0, put into pairs of query elements
};

__device__ inline int divide(int n, FastDiv f) { return (int)winof4::fast_div((uint32_t)n, f); }
// For what hardly ever passes 32 bits (n is not negative).
__device__ inline int64_t divide(int64_t n, int d) { return n >> 31 ? n / d : (int64_t)((uint32_t)n / (uint32_t)d); }

template <int DIM, int WAVES = 4> struct Shape {
    static constexpr int kSteps = DIM / 32;                 // products of 32 dimensions
    static constexpr int kTok = DIM <= 128 ? 64 : 32;       // tokens of a wave's step
    static constexpr int kTiles = kTok / 16;
    static constexpr int kRow = DIM * 2 + 32;               // bytes of a token's V in LDS: 8 rows cover all banks once
    static constexpr int kScales = DIM == 64 || DIM == 128 ? 1 : 2;   // scales in a lane's quarter
    static constexpr int kStage = 32 * kRow;                // a wave's V in LDS, 32 tokens at a time
    static constexpr int kJoin = 16 * (DIM + 4) * 4;        // a wave's results in LDS: sums, reference, total
    static constexpr int kLds = WAVES * (kStage > kJoin ? kStage : kJoin);
};

// One step's codes and scales: lane (t, g) has quarter g of token t of each tile.
template <int DIM> struct Codes {
    uint32_t w[Shape<DIM>::kTiles][Shape<DIM>::kSteps];
    uint32_t s[Shape<DIM>::kTiles][Shape<DIM>::kScales];
};

template <int DIM>
__device__ inline void load_codes(Codes<DIM>& c, const uint8_t* codes, const uint8_t* scales, const int64_t (&at)[Shape<DIM>::kTiles],
                                  int lane) {
    typedef Shape<DIM> S;
    const int t = lane & 15, g = lane >> 4;
    const int code_at = t * (DIM / 2) + g * (DIM / 8), first = g * (DIM / 4) / 32, scale_at = t * (DIM / 32) + first;
#pragma unroll
    for (int i = 0; i < S::kTiles; ++i) {
        const uint8_t* p = codes + at[i] * (DIM / 2) + code_at;
        if constexpr (S::kSteps % 4 == 0) {
#pragma unroll
            for (int j = 0; j < S::kSteps; j += 4) {
                const u32x4 x = *(const u32x4*)(p + 4 * j);
                c.w[i][j] = x[0], c.w[i][j + 1] = x[1], c.w[i][j + 2] = x[2], c.w[i][j + 3] = x[3];
            }
        } else if constexpr (S::kSteps % 2 == 0) {
#pragma unroll
            for (int j = 0; j < S::kSteps; j += 2) {
                const u32x2 x = *(const u32x2*)(p + 4 * j);
                c.w[i][j] = x[0], c.w[i][j + 1] = x[1];
            }
        } else {
#pragma unroll
            for (int j = 0; j < S::kSteps; ++j) c.w[i][j] = *(const uint32_t*)(p + 4 * j);
        }
        const uint8_t* s = scales + at[i] * (DIM / 32) + scale_at;
        c.s[i][0] = s[0];
        if constexpr (S::kScales == 2) c.s[i][1] = s[first + 1 < DIM / 32 ? 1 : 0];
    }
}

// Scale of the eight dimensions j of a lane's quarter.
template <int DIM> __device__ inline float piece_scale(const uint32_t (&s)[Shape<DIM>::kScales], int j, int g) {
    if constexpr (Shape<DIM>::kScales == 1) return scale_bits(s[0]);
    const int first = g * (DIM / 4) / 32, mine = (g * (DIM / 4) + 8 * j) / 32;
    return scale_bits(mine == first ? s[0] : s[Shape<DIM>::kScales - 1]);
}

// The work of a call is the blocks of 256 tokens of all units in a row: sequence by sequence, its units one after the
// other, the blocks of a unit in order.  Each workgroup takes an equal share of the row, so long and short sequences
// keep all of them busy alike; units that it holds whole go straight to the output, the two at its ends may be parts.
// What a unit costs beside its tokens (its queries, the wait for its first codes, the join of the waves) counts as a
// block too: block 0 of each unit holds no tokens.
__device__ inline int length(const DecodeArgs& a, int b) { return min(max(a.lens[b], 0), a.room); }
__device__ inline int blocks(int len) { return 1 + (len + kBlock - 1) / kBlock; }

struct Place {
    int64_t share, before;      // blocks of a workgroup; blocks of all units of the sequences before b
    int b;
};
// The share of workgroup w, and the sequence that it begins in (batch: it has none).
__device__ inline Place find(const DecodeArgs& a, int w) {
    const int lane = threadIdx.x & 63;
    int n = 0, upto = 0;                                    // blocks of this lane's sequence, and of the 64 up to it
    auto scan = [&](int b0) {
        n = b0 + lane < a.batch ? blocks(length(a, b0 + lane)) : 0;
        upto = n;
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(upto, o);
            if (lane >= o) upto += x;
        }
        return __shfl(upto, 63);
    };
    int64_t total = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64) total += scan(b0);
    Place p;
    p.share = divide(total * a.units + a.groups - 1, a.groups);
    p.b = a.batch;
    p.before = 0;
    const int64_t first = p.share * w;
    for (int b0 = 0; b0 < a.batch; b0 += 64) {
        const int all = a.batch > 64 ? scan(b0) : (int)total;
        const uint64_t past = __ballot(first < (p.before + upto) * a.units);
        if (past) {
            const int l = __builtin_ctzll(past);
            p.b = __builtin_amdgcn_readfirstlane(b0 + l);
            p.before += __builtin_amdgcn_readfirstlane(__shfl(upto - n, l));
            break;
        }
        p.before += all;
    }
    return p;
}

// Where the parts of a unit are: workgroups first .. last; the first one's is its second part where `second`.
struct Parts {
    int32_t first, last, second, pad;
};
__device__ inline float* part_ml(const DecodeArgs& a, int dim) { return a.part + (int64_t)2 * a.groups * 16 * dim; }
__device__ inline Parts* unit_parts(const DecodeArgs& a, int dim) { return (Parts*)(part_ml(a, dim) + (int64_t)2 * a.groups * 16 * 2); }

// WAVES: 4 where the work is shared out (three workgroups a compute unit), 8 where a workgroup takes one unit, which is
// short then.
template <int TYPE, int DIM, int WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES == 8 || DIM > 128 ? 2 : 3) void kv4_attention_kernel(DecodeArgs a) {
    typedef typename Half<TYPE>::type T;
    typedef Shape<DIM, WAVES> S;
    typedef T T8 __attribute__((ext_vector_type(8)));
    constexpr int kParts = TYPE == WINO_FP16 ? 2 : 1;       // bf16 numbers of a query element
    __shared__ __attribute__((aligned(16))) uint8_t lds[S::kLds];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;

    int b, unit, blk, len, left, share = 0;                 // left: blocks of the share still to do
    if (a.part) {
        const Place p = find(a, blockIdx.x);
        if (p.b >= a.batch) return;
        b = p.b;
        len = __builtin_amdgcn_readfirstlane(length(a, b));
        const int n = blocks(len);
        const int64_t in = p.share * blockIdx.x - p.before * a.units;
        unit = __builtin_amdgcn_readfirstlane((int)divide(in, n));
        blk = __builtin_amdgcn_readfirstlane((int)(in - (int64_t)unit * n));
        share = left = __builtin_amdgcn_readfirstlane((int)p.share);
    } else {
        b = divide((int)blockIdx.x, a.by_units);
        unit = (int)blockIdx.x - b * a.units;
        blk = 0;
        len = __builtin_amdgcn_readfirstlane(length(a, b));
        left = blocks(len);
    }
    bool opening = true;                                    // the first unit of the share
    for (;;) {
    const int n_blocks = blocks(len);
    const int take = min(left, n_blocks - blk);
    const bool is_part = take < n_blocks;
    if (a.part && blk == 0 && threadIdx.x == 0)
        unit_parts(a, DIM)[(int64_t)b * a.units + unit] =
            Parts{(int)blockIdx.x, (int)blockIdx.x + (n_blocks - take + share - 1) / share, opening ? 0 : 1, 0};
    const int kvh = divide(unit, a.by_tiles), tile = unit - kvh * a.tiles;
    const int first_end = len - a.q_len + 1;                // tokens that query 0 sees; every row sees those
    const int begin = max(blk - 1, 0) * kBlock;
    const int end = a.pages == 0 ? begin : min((int64_t)len, (int64_t)(blk + take - 1) * kBlock);
    // one step or less is one wave's work, and needs no join
    const bool alone = WAVES == 8 && end <= S::kTok;
    if (alone && wave > 0) return;

    // this lane's row: query i, head h
    const int row = tile * 16 + r;
    const int i = divide(row, a.by_group), h = kvh * a.group + row - i * a.group;
    const bool real = i < a.q_len;
    const int row_end = real ? (first_end + i < len ? first_end + i : len) : 0;

    // An infinite element makes all scores infinite, of one sign or another: not a number where any is seen.  It becomes a
    // NaN here (0 times it; the second part in fp16 is one), because scores that are all minus infinity would look like none.
    bf16x8 q[kParts][S::kSteps];
    {
        float none = 0.f;
        const T* p = (const T*)a.q + ((int64_t)b * a.q_len + (real ? i : 0)) * a.q_stride + (int64_t)(real ? h : 0) * DIM +
                     g * (DIM / 4);
#pragma unroll
        for (int j = 0; j < S::kSteps; ++j) {
            const T8 x = __builtin_bit_cast(T8, (*(const u32x4*)(p + 8 * j) & a.q_and) ^ a.q_xor);
            if constexpr (TYPE == WINO_BF16) {
                q[0][j] = x;
#pragma unroll
                for (int e = 0; e < 8; e += 2)
                    none = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{x[e], x[e + 1]}, bf16x2{(__bf16)0.f, (__bf16)0.f}, none, false);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const __bf16 hi = (__bf16)(float)x[e];
                    q[0][j][e] = hi;
                    q[kParts - 1][j][e] = (__bf16)((float)x[e] - (float)hi);
                }
            }
        }
        if constexpr (TYPE == WINO_BF16) q[0][0][0] = (__bf16)((float)q[0][0][0] + none);
    }

    f32x4 o[DIM / 16];                                      // lane: dimensions 16 n + 4 g + e of row r
#pragma unroll
    for (int n = 0; n < DIM / 16; ++n) o[n] = f32x4{0.f, 0.f, 0.f, 0.f};
    float ref = kNever, sum = 0.f;                          // ref: the power of two that o and sum are held against
    uint8_t* stage = lds + wave * S::kStage;

    // First slots of the tiles to come: lane l has tile l % kTiles of step `listed` + l / kTiles.  A tile whose tokens
    // are not there has a bit in `there` missing, and stands at slot 0.
    constexpr int kListed = 64 / S::kTiles;
    const int32_t* pages = a.table + (int64_t)b * a.max_pages;
    const int w0 = begin + wave * S::kTok;                  // the wave's first token
    uint64_t slot = 0, there = 0;
    auto list = [&](int step) {
        const int t = w0 + (step + lane / S::kTiles) * (WAVES * S::kTok) + 16 * (lane % S::kTiles);
        int64_t id = -1;
        int pg = 0;
        if (t < end) {
            pg = divide(t, a.by_page);
            id = pages[pg];
        }
        const bool ok = id >= 0 && id < a.pages;
        slot = ok ? (id * a.kv_heads + kvh) * a.page + (t - pg * a.page) : 0;
        there = __ballot(ok);
    };
    auto place = [&](int step, int64_t (&at)[S::kTiles]) {
#pragma unroll
        for (int n = 0; n < S::kTiles; ++n) {
            const int l = step % kListed * S::kTiles + n;
            at[n] = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(slot >> 32), l) << 32 |
                              (uint32_t)__builtin_amdgcn_readlane((int)slot, l));
        }
    };
    auto tiles_there = [&](int step) { return (uint32_t)(there >> (step % kListed * S::kTiles)) & ((1u << S::kTiles) - 1); };

    int t0 = w0, step = 0;
    uint32_t have = 0;                                      // tiles of this step that are there
    Codes<DIM> kc, vc;
    if (t0 < end) {
        list(0);
        int64_t at[S::kTiles];
        place(0, at);
        have = tiles_there(0);
        load_codes<DIM>(kc, a.k_codes, a.k_scales, at, lane);
        load_codes<DIM>(vc, a.v_codes, a.v_scales, at, lane);
    }
    for (; t0 < end; t0 += WAVES * S::kTok) {
        const bool more = t0 + WAVES * S::kTok < end;
        // scores, transposed: lane has tokens 16 n + 4 g + e of row r
        f32x4 z[S::kTiles];
#pragma unroll
        for (int n = 0; n < S::kTiles; ++n) {
            z[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < S::kSteps; ++j) {
                const bf16x8 k = decode8(kc.w[n][j], piece_scale<DIM>(kc.s[n], j, g));
#pragma unroll
                for (int p = 0; p < kParts; ++p)
                    z[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[p][j], z[n], 0, 0, 0);
            }
        }
        // the next step's codes are on their way as soon as the registers of this one's are free
        int64_t at[S::kTiles];
        uint32_t have_next = 0;
        if (more) {
            ++step;
            if (step % kListed == 0) list(step);
            place(step, at);
            have_next = tiles_there(step);
            load_codes<DIM>(kc, a.k_codes, a.k_scales, at, lane);
        }
        // tokens that some row does not see
        if (t0 + S::kTok > (first_end < end ? first_end : end) || have != (1u << S::kTiles) - 1) {
#pragma unroll
            for (int n = 0; n < S::kTiles; ++n) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!((have >> n) & 1) || t0 + 16 * n + 4 * g + e >= row_end) z[n][e] = kNever;
                // what lies past the length was never written; its scale may say NaN
                const int t = (have >> n) & 1 ? t0 + 16 * n + r : end;
#pragma unroll
                for (int j = 0; j < S::kScales; ++j) {
                    // A value that is not finite would spoil the rows that do not see its token too (0 times it is
                    // NaN): it leaves the product, and the rows that see it are marked here.
                    uint64_t spoilt = __ballot(t < end && t >= first_end && vc.s[n][j] >= 253u);
                    if (t >= end || ((spoilt >> lane) & 1)) vc.s[n][j] = 0;
                    for (; spoilt; spoilt &= spoilt - 1) {
                        const int l = __builtin_ctzll(spoilt), quarter = l >> 4;
                        if (t0 + 16 * n + (l & 15) >= row_end) continue;
                        const int group = min(quarter * (DIM / 4) / 32 + j, DIM / 32 - 1);
#pragma unroll
                        for (int m = 0; m < DIM / 16; ++m)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int d = 16 * m + 4 * g + e;
                                if (d / (DIM / 4) == quarter && d / 32 == group) o[m][e] = __builtin_nanf("");
                            }
                    }
                }
            }
        }
        float top = kNever;
#pragma unroll
        for (int n = 0; n < S::kTiles; ++n) top = max3(max3(z[n][0], z[n][1], z[n][2]), z[n][3], top);
        top = max_rows(top) * a.scale_log2;
        // o and sum move to a new reference only where the maximum has outgrown the old one by 2^8
        if (__any(top > ref + 8.f)) {
            const float to = __builtin_fmaxf(ref, top);
            const float alpha = to == kNever ? 1.f : __builtin_amdgcn_exp2f(ref - to);
            ref = to;
            sum *= alpha;
#pragma unroll
            for (int n = 0; n < DIM / 16; ++n) o[n] *= alpha;
        }
        const float base = ref == kNever ? 0.f : -ref;
        uint32_t hi[S::kTiles][2], lo[S::kTiles][2];
#pragma unroll
        for (int n = 0; n < S::kTiles; ++n)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[n][e], a.scale_log2, base));
                const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[n][e + 1], a.scale_log2, base));
                sum += p0 + p1;
                const bf16x2 x = {(__bf16)p0, (__bf16)p1};
                const bf16x2 y = {(__bf16)(p0 - (float)x[0]), (__bf16)(p1 - (float)x[1])};
                hi[n][e / 2] = __builtin_bit_cast(uint32_t, x);
                lo[n][e / 2] = __builtin_bit_cast(uint32_t, y);
            }

        // 32 tokens at a time: V to LDS by tokens, back by dimensions
#pragma unroll
        for (int m = 0; m < S::kTiles / 2; ++m) {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int j = 0; j < S::kSteps; ++j)
                    *(bf16x8*)(stage + (16 * n + r) * S::kRow + g * (DIM / 2) + 16 * j) =
                        decode8(vc.w[2 * m + n][j], piece_scale<DIM>(vc.s[2 * m + n], j, g));
            if (m == S::kTiles / 2 - 1 && more) load_codes<DIM>(vc, a.v_codes, a.v_scales, at, lane);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            const u32x4 ph = {hi[2 * m][0], hi[2 * m][1], hi[2 * m + 1][0], hi[2 * m + 1][1]};
            const u32x4 pl = {lo[2 * m][0], lo[2 * m][1], lo[2 * m + 1][0], lo[2 * m + 1][1]};
            // lane l of 16 gives the address of four dimensions of token l / 4 and gets dimension l of four tokens
            const uint8_t* from = stage + (4 * g + (r >> 2)) * S::kRow + (r & 3) * 8;
#pragma unroll
            for (int n = 0; n < DIM / 16; n += 2) {         // two at a time: no product waits for the one before it
                typedef __attribute__((ext_vector_type(4))) short s4;
                typedef __attribute__((address_space(3))) s4* lds4;
                bf16x8 v[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint8_t* f = from + 32 * (n + k);
                    const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)f));
                    const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(f + 16 * S::kRow)));
                    v[k] = __builtin_bit_cast(bf16x8, u32x4{x[0], x[1], y[0], y[1]});
                }
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    o[n + k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[k], __builtin_bit_cast(bf16x8, ph), o[n + k], 0, 0, 0);
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    o[n + k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[k], __builtin_bit_cast(bf16x8, pl), o[n + k], 0, 0, 0);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        have = have_next;
    }
    sum = sum_rows(sum);
    if (alone) {
        typedef T T4 __attribute__((ext_vector_type(4)));
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        T* out = (T*)a.out + (((int64_t)b * a.q_len + i) * a.heads + h) * DIM + 4 * g;
#pragma unroll
        for (int n = 0; n < DIM / 16; ++n)
            if (real)
                *(T4*)(out + 16 * n) = sum == 0.f ? T4{} : T4{(T)(o[n][0] * inv), (T)(o[n][1] * inv), (T)(o[n][2] * inv), (T)(o[n][3] * inv)};
        return;
    }

    // join the waves: [wave][row][dim + 4]
    const int rows = min(16, a.q_len * a.group - tile * 16);
    constexpr int kRowJ = DIM + 4;
    __syncthreads();
    if (r < rows) {
        float* mine = (float*)lds + (wave * 16 + r) * kRowJ;
#pragma unroll
        for (int n = 0; n < DIM / 16; ++n) *(f32x4*)(mine + 16 * n + 4 * g) = o[n];
        if (g == 0) {
            mine[DIM] = ref;
            mine[DIM + 1] = sum;
        }
    }
    __syncthreads();
    for (int x = threadIdx.x; x < rows * (DIM / 4); x += 64 * WAVES) {
        const int rr = x / (DIM / 4), d = x % (DIM / 4) * 4;
        const float* w = (const float*)lds + rr * kRowJ;
        float m = kNever;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) m = __builtin_fmaxf(m, w[k * 16 * kRowJ + DIM]);
        const float base = m == kNever ? 0.f : m;
        float total = 0.f;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < WAVES; ++k) {
            const float f = __builtin_amdgcn_exp2f(w[k * 16 * kRowJ + DIM] - base);
            total += f * w[k * 16 * kRowJ + DIM + 1];
            acc += f * *(const f32x4*)(w + k * 16 * kRowJ + d);
        }
        if (is_part) {
            const int64_t p = ((int64_t)2 * blockIdx.x + (opening ? 0 : 1)) * 16 + rr;
            *(f32x4*)(a.part + p * DIM + d) = acc;
            if (d == 0) {
                float* ml = part_ml(a, DIM) + 2 * p;
                ml[0] = m, ml[1] = total;
            }
        } else {
            typedef T T4 __attribute__((ext_vector_type(4)));
            const int ro = tile * 16 + rr, io = divide(ro, a.by_group);
            const T4 y = total == 0.f ? T4{} : T4{(T)(acc[0] / total), (T)(acc[1] / total), (T)(acc[2] / total), (T)(acc[3] / total)};
            *(T4*)((T*)a.out + (((int64_t)b * a.q_len + io) * a.heads + kvh * a.group + ro - io * a.group) * DIM + d) = y;
        }
    }
    left -= take;
    if (left == 0) return;
    opening = false;
    blk = 0;                                                // the unit is done: the share goes on with the next one
    if (++unit == a.units) {
        unit = 0;
        if (++b == a.batch) return;
        len = __builtin_amdgcn_readfirstlane(length(a, b));
    }
    __syncthreads();
    }
}

// Joins the parts of units that several workgroups shared: one workgroup per query row and head; groups of DIM / 4
// threads take the parts in turn.
template <int TYPE, int DIM, int THREADS> __global__ __launch_bounds__(THREADS) void kv4_join_kernel(DecodeArgs a) {
    typedef typename Half<TYPE>::type T;
    typedef T T4 __attribute__((ext_vector_type(4)));
    constexpr int kCols = DIM / 4, kTeams = THREADS / kCols;
    __shared__ f32x4 acc_s[kTeams][kCols];
    __shared__ float m_s[kTeams], total_s[kTeams];
    const int token = divide((int)blockIdx.x, a.by_heads), h = (int)blockIdx.x - token * a.heads;
    const int b = divide(token, a.by_q), i = token - b * a.q_len, kvh = divide(h, a.by_group);
    const int row = i * a.group + h - kvh * a.group;
    const int unit = kvh * a.tiles + row / 16;
    const Parts p = unit_parts(a, DIM)[(int64_t)b * a.units + unit];
    const int w0 = p.first, w1 = p.last;
    if (w0 == w1) return;                                   // whole, and in the output already
    const int team = threadIdx.x / kCols, col = threadIdx.x % kCols;
    const float* ml = part_ml(a, DIM);
    float m = kNever, total = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (team < kTeams)
        for (int w = w0 + team; w <= w1; w += 4 * kTeams) {
            float mw[4], tw[4];
            f32x4 x[4];
            float to = m;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int v = w + k * kTeams <= w1 ? w + k * kTeams : w;
                const int64_t at = ((int64_t)2 * v + (v == w0 ? p.second : 0)) * 16 + row % 16;
                mw[k] = w + k * kTeams <= w1 ? ml[2 * at] : kNever, tw[k] = ml[2 * at + 1];
                x[k] = *(const f32x4*)(a.part + at * DIM + 4 * col);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) to = __builtin_fmaxf(to, mw[k]);
            const float base = to == kNever ? 0.f : to, f = __builtin_amdgcn_exp2f(m - base);
            total *= f;
            acc *= f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                // what stands in for a part that is not there is left out by its index: a part of minus infinity may be
                // one whose scores are all NaN, whose total says so (0 times NaN is NaN; a part that saw nothing adds 0)
                if (w + k * kTeams > w1) continue;
                const float fw = __builtin_amdgcn_exp2f(mw[k] - base);
                total += tw[k] * fw;
                acc += x[k] * fw;
            }
            m = to;
        }
    if (team < kTeams) {
        acc_s[team][col] = acc;
        if (col == 0) m_s[team] = m, total_s[team] = total;
    }
    __syncthreads();
    if (threadIdx.x >= kCols) return;
    float top = kNever;
#pragma unroll
    for (int t = 0; t < kTeams; ++t) top = __builtin_fmaxf(top, m_s[t]);
    const float base = top == kNever ? 0.f : top;
    total = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < kTeams; ++t) {
        const float f = __builtin_amdgcn_exp2f(m_s[t] - base);
        total += f * total_s[t];
        acc += f * acc_s[t][threadIdx.x];
    }
    const T4 y = total == 0.f ? T4{} : T4{(T)(acc[0] / total), (T)(acc[1] / total), (T)(acc[2] / total), (T)(acc[3] / total)};
    *(T4*)((T*)a.out + ((int64_t)token * a.heads + h) * DIM + 4 * threadIdx.x) = y;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

struct Cut {
    int64_t tiles, units, groups;
    bool split;
    size_t bytes;
};

// A call's workgroups.  Sequences are split where that spares a workgroup more than three blocks of tokens: the join
// is a launch of its own (777 tokens of two heads: 8.0 us in one launch, 10 in two).  The host knows no lengths, so it
// goes by what the table has room for: 500 tokens of 8 heads take 8.0 us with a table of their length and 10.9 with one for
// 131072, 64 such sequences 14.4 and 15.6.  A launch has less than 2^32 threads: the join's 256 a row set an end to splitting.
Cut cut(int64_t batch, int64_t q_len, int64_t heads, int64_t kv_heads, int dim, int64_t room) {
    Cut c;
    c.tiles = (q_len * (heads / kv_heads) + 15) / 16;
    c.units = kv_heads * c.tiles;
    const int64_t blocks = std::max<int64_t>(1, (room + kBlock - 1) / kBlock), all = batch * c.units * blocks;
    c.groups = std::min<int64_t>(all, dim <= 128 ? kGroups : kGroups * 2 / 3);
    c.split = blocks - (all + c.groups - 1) / c.groups > 3 && batch * q_len * heads < 1 << 24;
    c.bytes = c.split ? (size_t)(2 * c.groups * 16 * (dim + 2) * 4 + batch * c.units * sizeof(Parts)) : 0;
    return c;
}

template <int TYPE, int DIM> wino_status launch(const DecodeArgs& a, int64_t rows, hipStream_t stream) {
    const dim3 grid((unsigned)a.groups);
    if (!a.part) {
        hipLaunchKernelGGL((kv4_attention_kernel<TYPE, DIM, 8>), grid, dim3(512), 0, stream, a);
        return hipGetLastError() == hipSuccess ? WINO_OK : WINO_EHIP;
    }
    hipLaunchKernelGGL((kv4_attention_kernel<TYPE, DIM, 4>), grid, dim3(256), 0, stream, a);
    if (hipGetLastError() != hipSuccess) return WINO_EHIP;
    // few rows have many parts each (64 rows of 48: 39.7 us the call, with 256 threads 40.3), many rows few
    if (rows <= 256)
        hipLaunchKernelGGL((kv4_join_kernel<TYPE, DIM, 512>), dim3((unsigned)rows), dim3(512), 0, stream, a);
    else
        hipLaunchKernelGGL((kv4_join_kernel<TYPE, DIM, 256>), dim3((unsigned)rows), dim3(256), 0, stream, a);
    return hipGetLastError() == hipSuccess ? WINO_OK : WINO_EHIP;
}

template <int TYPE> wino_status launch_dim(int dim, const DecodeArgs& a, int64_t rows, hipStream_t stream) {
    switch (dim) {
        case 64: return launch<TYPE, 64>(a, rows, stream);
        case 96: return launch<TYPE, 96>(a, rows, stream);
        case 128: return launch<TYPE, 128>(a, rows, stream);
        case 192: return launch<TYPE, 192>(a, rows, stream);
        default: return launch<TYPE, 256>(a, rows, stream);
    }
}

}  // namespace

extern "C" size_t kv4_attention_workspace_bytes(int32_t batch, int32_t q_len, int32_t heads, int32_t kv_heads,
                                                int32_t head_dim, int32_t max_pages, int32_t page_size) {
    if (batch < 1 || q_len < 1 || heads < 1 || kv_heads < 1 || head_dim < 1 || max_pages < 1 || page_size < 1) return 0;
    if (heads % kv_heads || (int64_t)batch * q_len * heads > 0x7fffffffll) return 0;
    return cut(batch, q_len, heads, kv_heads, head_dim, (int64_t)max_pages * page_size).bytes;
}

extern "C" wino_status kv4_attention(const void* q, int64_t q_stride, const kv4_cache* cache,
                                     const int32_t* block_table, int32_t max_pages, const int32_t* lens, void* out,
                                     int32_t batch, int32_t q_len, int32_t heads, float scale, wino_float_type type,
                                     void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!cache || (type != WINO_BF16 && type != WINO_FP16)) return WINO_EINVAL;
    const kv4_cache& c = *cache;
    if (c.pages < 0 || c.kv_heads < 1 || c.page_size < 1 || c.head_dim < 1 || batch < 0 || q_len < 0 || heads < 1 ||
        max_pages < 0)
        return WINO_EINVAL;
    if (heads % c.kv_heads || !(scale == scale) || scale - scale != 0.f) return WINO_EINVAL;
    if (c.page_size % 16 || c.kv_heads > 4096 || heads > 65536 || c.pages > (int64_t)1 << 40 || c.page_size > 1 << 20)
        return WINO_EUNSUPPORTED;
    if (c.head_dim != 64 && c.head_dim != 96 && c.head_dim != 128 && c.head_dim != 192 && c.head_dim != 256)
        return WINO_EUNSUPPORTED;
    if (batch == 0 || q_len == 0) return WINO_OK;
    if (!q || !lens || !out || (max_pages > 0 && !block_table)) return WINO_EINVAL;
    if (c.pages > 0 && (!c.k_codes || !c.k_scales || !c.v_codes || !c.v_scales)) return WINO_EINVAL;
    const bool many = (int64_t)batch * q_len > 1;
    if (many && q_stride < (int64_t)heads * c.head_dim) return WINO_EINVAL;
    if ((many && (q_stride & 7)) || !aligned16(q) || !aligned16(out) || !aligned16(c.k_codes) || !aligned16(c.v_codes) ||
        !aligned16(workspace))
        return WINO_EUNSUPPORTED;
    const int64_t rows = (int64_t)batch * q_len * heads;
    if (rows > 0x7fffffffll) return WINO_EUNSUPPORTED;
    const int64_t room = std::min<int64_t>((int64_t)max_pages * c.page_size, 0x7fffffff - 65536);
    const Cut k = cut(batch, q_len, heads, c.kv_heads, c.head_dim, room);
    const bool split = k.split && workspace && workspace_bytes >= k.bytes;
    if (!split && batch * k.units >= 1 << 23) return WINO_EUNSUPPORTED;     // workgroups of 512 threads
    DecodeArgs a = {q, out, c.k_codes, c.k_scales, c.v_codes, c.v_scales, block_table, lens,
                    split ? (float*)workspace : nullptr, q_stride, c.pages, q_len, heads, c.kv_heads,
                    heads / c.kv_heads, c.page_size, max_pages, (int32_t)k.tiles, batch, (int32_t)k.units,
                    (int32_t)(split ? k.groups : batch * k.units), (int32_t)room,
                    winof4::make_fastdiv((uint32_t)c.page_size), winof4::make_fastdiv((uint32_t)(heads / c.kv_heads)),
                    winof4::make_fastdiv((uint32_t)k.tiles), winof4::make_fastdiv((uint32_t)k.units),
                    winof4::make_fastdiv((uint32_t)heads), winof4::make_fastdiv((uint32_t)q_len),
                    scale == 0.f ? 1.f : __builtin_fabsf(scale) * 1.44269504088896340736f, scale == 0.f ? 0u : 0xffffffffu,
                    scale < 0.f ? 0x80008000u : 0u};
    if (a.scale_log2 - a.scale_log2 != 0.f) return WINO_EUNSUPPORTED;       // past fp32's range
    return type == WINO_BF16 ? launch_dim<WINO_BF16>(c.head_dim, a, rows, stream)
                             : launch_dim<WINO_FP16>(c.head_dim, a, rows, stream);
}
