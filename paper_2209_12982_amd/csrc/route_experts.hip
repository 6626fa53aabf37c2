// Routing of tokens to experts: scores, the best experts of the best groups, their weights, and the routes in the order of
// their experts.
//
//   s = softmax(l) or 1 / (1 + exp(-l)) over a token's experts, c = s + bias
//   a group's value is the sum of its `group_best` (1 or 2) largest c; the `top_groups` groups of the largest values stay
//   chosen: the `top` largest c among their experts, the largest first; ties go to the lowest index, not-a-numbers count as
//   minus infinity;  weight = s (over the sum of the chosen s, where they are normalised) times `scale`
//
// Scores are held in 64 bits: which expert comes first hangs on differences that 32 bits do not hold, and the sizes are
// small.  A wave takes a token and holds its values, neighbouring experts in a lane; experts are taken one after the other, by
// the upper halves of their values as whole numbers, and the lower ones where those are equal.
//
// The order is a counting sort by expert, stable: counts for each block of tokens, their sums over the blocks, and then
// each route's place, three launches; a single block does all in one.  No atomics decide a place, so the order is the same
// each time.
//
// Instructions bound it: 16384 tokens to 8 of 256 experts by groups take 35 us, 27 of them here, 620 instructions a token
// on vector units that are busy half of the time (four waves a SIMD; eight, with fewer registers, take 36), 4.5 for the sums
// and 5.4 for the places.  Fewer tokens take the launches: 1000 to 6 of 60 11.9 us, without an order 3.9.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "mx4.h"
#include "wino_device.h"
#include "winof4.h"

namespace {
using namespace mx4;

constexpr int kMostExperts = 1024, kMostTop = 32, kMostGroups = 64;
constexpr int kTokens = 32;             // of a block at most
constexpr int kAlone = 32;              // that one block takes by itself at most
constexpr int kWaveRoutes = 128;        // that a wave places
constexpr int kFewBlocks = 16;          // whose counts each block adds up by itself: shorter than a launch between

struct RouteArgs {
    const void* logits;
    const float* bias;
    const int32_t* live;
    int32_t* chosen;
    float* weights;
    int64_t stride;
    int32_t tokens, experts, top, groups, size, top_groups, group_best, sigmoid, normalise;
    int32_t group_lanes;    // that a group has: the largest power of two, all groups in a wave
    float scale;
    winof4::FastDiv by_size;
    // the order, or null; counts: [experts][row_blocks], later what comes before a block; totals: [experts]
    int32_t *order, *ends, *counts, *totals;
    int32_t blocks, block_tokens, row_blocks;
};

template <int TYPE> __device__ inline float load(const void* p, int64_t at) {
    if (TYPE == WINO_BF16) return (float)((const __bf16*)p)[at];
    if (TYPE == WINO_FP16) return (float)((const _Float16*)p)[at];
    return ((const float*)p)[at];
}

// Order of doubles as whole numbers; every number is above 0.
__device__ inline uint64_t ordered(double v) {
    const u32x2 b = __builtin_bit_cast(u32x2, v + 0.0);             // -0 is 0
    const uint32_t sign = (uint32_t)((int)b[1] >> 31);
    return (uint64_t)(b[1] ^ (sign | 0x80000000u)) << 32 | (b[0] ^ sign);
}
// The largest of a wave, by moves inside the registers (a shuffle through LDS for each of six steps takes twice as long).
__device__ inline uint32_t wave_max(uint32_t v) {
#define STEP(ctrl, rows) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xf, false))
    STEP(0x111, 0xf);       // from 1, 2, 4 and 8 lanes before, inside rows of 16
    STEP(0x112, 0xf);
    STEP(0x114, 0xf);
    STEP(0x118, 0xf);
    STEP(0x142, 0xa);       // the last lane of a row to the next row
    STEP(0x143, 0xc);       // and of the first two rows to the others
#undef STEP
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
template <int CTRL, int ROWS> __device__ inline double moved(double v) {
    const u32x2 b = __builtin_bit_cast(u32x2, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b[0], CTRL, ROWS, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b[1], CTRL, ROWS, 0xf, false);
    return __builtin_bit_cast(double, u32x2{lo, hi});
}
__device__ inline double lane_value(double v, int lane) {
    const u32x2 b = __builtin_bit_cast(u32x2, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)b[0], lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)b[1], lane);
    return __builtin_bit_cast(double, u32x2{lo, hi});
}
// The sum over the first `lanes` lanes, the others have zeros: fewer steps for up to 4 or 16.
__device__ inline double wave_sum(double v, int lanes = 64) {
    v += moved<0x111, 0xf>(v);
    v += moved<0x112, 0xf>(v);
    if (lanes <= 4) return lane_value(v, 3);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    if (lanes <= 16) return lane_value(v, 15);
    v += moved<0x142, 0xa>(v);
    v += moved<0x143, 0xc>(v);
    return lane_value(v, 63);
}
// Order of floats as whole numbers above 0; 0 for what is not a number.
__device__ inline uint32_t ordered(float v) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    return v == v ? (b >> 31 ? ~b : b | 0x80000000u) : 0;
}
__device__ inline float unordered(uint32_t b) { return __builtin_bit_cast(float, b >> 31 ? b ^ 0x80000000u : ~b); }
// e^x to 2^-47 of itself: x = n ln 2 + r with |r| <= ln 2 / 2, and the series of e^r to r^11 (the rest is below r^12 / 12! =
// 6.3e-15).  Half the instructions of the library's function, whose last six bits no choice and no weight needs.  For |x| up to
// 800, where e^x is 0 or infinity, and a NaN.
__device__ inline double exponential(double x) {
    const double n = __builtin_rint(x * 1.4426950408889634);
    double r = __builtin_fma(n, -0.6931471805599453, x);
    r = __builtin_fma(n, -2.3190468138462996e-17, r);       // ln 2 - 0.6931471805599453
    double p = 1.0 / 39916800;
    p = __builtin_fma(p, r, 1.0 / 3628800);
    p = __builtin_fma(p, r, 1.0 / 362880);
    p = __builtin_fma(p, r, 1.0 / 40320);
    p = __builtin_fma(p, r, 1.0 / 5040);
    p = __builtin_fma(p, r, 1.0 / 720);
    p = __builtin_fma(p, r, 1.0 / 120);
    p = __builtin_fma(p, r, 1.0 / 24);
    p = __builtin_fma(p, r, 1.0 / 6);
    p = __builtin_fma(p, r, 0.5);
    p = __builtin_fma(p, r, 1.0);
    p = __builtin_fma(p, r, 1.0);
    return __builtin_ldexp(p, (int)n);
}

// 1 / d for d of 1 or more: two steps of Newton's make it exact and need no scaling (half the instructions of a division; what
// is below 2^-1022 may become 0).
__device__ inline double reciprocal(double d) {
    double r = __builtin_amdgcn_rcp(d);
    r = __builtin_fma(r, __builtin_fma(-d, r, 1.0), r);
    r = __builtin_fma(r, __builtin_fma(-d, r, 1.0), r);
    return __builtin_amdgcn_div_fixup(r, d, 1.0);           // infinity and NaN
}
// 1 / (1 + e^-z).
__device__ inline double sigmoid(float z) {
    const float x = z == z ? __builtin_amdgcn_fmed3f(-z, -800.f, 800.f) : z;
    return reciprocal(1.0 + exponential((double)x));
}

// What is not a number counts as minus infinity.
__device__ inline double number(double v) { return v == v ? v : -__builtin_inf(); }

// Values written by lanes of the wave are read by others.
__device__ inline void wave_sync() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// One token by one wave, lane i gets the i-th expert (-1: none) and its weight.  z, bias: of the lane's J experts.  room:
// [J 64] scores, and [J 64] values where groups are left out.
template <int TYPE, int J>
__device__ inline void route(const RouteArgs& a, const float (&z)[J], const float (&bias)[J], double* room, int& mine, float& weight) {
    const int lane = threadIdx.x & 63;
    double s[J];
    if (a.sigmoid) {
#pragma unroll
        for (int j = 0; j < J; ++j) s[j] = sigmoid(z[j]);
    } else {
        // a NaN is left out of the maximum, and makes the sum and with it all scores NaN
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) most = max(most, ordered(z[j]));
        most = wave_max(most);
        const double top = most ? (double)unordered(most) : 0.0;
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const double x = (double)z[j] - top;
            s[j] = lane * J + j < a.experts ? exponential(x < -800.0 ? -800.0 : x) : 0.0;
            sum += s[j];
        }
        const double part = reciprocal(wave_sum(sum));        // the largest one adds 1
#pragma unroll
        for (int j = 0; j < J; ++j) s[j] *= part;
    }
    // c in order: its upper half decides, and the lower one where that is equal
    const bool by_groups = a.top_groups < a.groups, own_group = a.size == J * a.group_lanes;    // a lane's experts are of one group
    uint32_t hi[J], lo[J];
    double first = -__builtin_inf(), second = -__builtin_inf();     // of a group
    auto take = [&](double f, double o) {                   // two more, f >= o
        const double low = f > first ? first : f;
        first = f > first ? f : first;
        second = o > second ? o : second;
        second = low > second ? low : second;
    };
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int e = lane * J + j;
        const double c = number(s[j] + (double)bias[j]);
        const uint64_t key = e < a.experts ? ordered(c) : 0;
        hi[j] = (uint32_t)(key >> 32), lo[j] = (uint32_t)key;
        room[e] = s[j];
        if (by_groups) {
            if (own_group) {
                const double low = c > first ? first : c;
                first = c > first ? c : first;
                second = low > second ? low : second;
            } else {
                room[J * 64 + e] = c;
            }
        }
    }
    wave_sync();
    if (by_groups) {
        // as many lanes for a group as there are, each with a share of its experts
        const int lanes = a.group_lanes, g = lane / lanes;
        if (!own_group && g < a.groups)
            for (int i = lane % lanes; i < a.size; i += lanes) take(room[J * 64 + g * a.size + i], -__builtin_inf());
        // with the other half of an aligned set of lanes: neighbours, pairs, then sets of eight and sixteen in reverse
        if (lanes > 1) take(moved<0xb1, 0xf>(first), moved<0xb1, 0xf>(second));
        if (lanes > 2) take(moved<0x4e, 0xf>(first), moved<0x4e, 0xf>(second));
        if (lanes > 4) take(moved<0x141, 0xf>(first), moved<0x141, 0xf>(second));
        if (lanes > 8) take(moved<0x140, 0xf>(first), moved<0x140, 0xf>(second));
        if (lanes > 16) take(__shfl_xor(first, 16), __shfl_xor(second, 16));
        const double own = number(a.group_best == 2 ? first + second : first);
        int before = 0;
        for (int i = 0; i < a.groups; ++i) {
            const double v = lane_value(own, i * lanes);
            before += v > own || (v == own && i < g) ? 1 : 0;
        }
        const bool stays = before < a.top_groups;
        if (own_group) {
#pragma unroll
            for (int j = 0; j < J; ++j) hi[j] = stays ? hi[j] : 0;
        } else {
            const uint64_t kept = __ballot(g < a.groups && stays);      // a bit for each lane of a group
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const uint32_t of = winof4::fast_div((uint32_t)min(lane * J + j, a.experts - 1), a.by_size);
                if (!(kept >> (of * lanes) & 1)) hi[j] = 0;
            }
        }
    }
    mine = -1;
    for (int i = 0; i < a.top; ++i) {
        uint32_t best = hi[0];
#pragma unroll
        for (int j = 1; j < J; ++j) best = max(best, hi[j]);
        const uint32_t most = wave_max(best);
        uint64_t at[J], lanes = 0;                          // the lanes that have it as their j-th
        int found = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            at[j] = __ballot(hi[j] == most);
            lanes |= at[j];
            found += __builtin_popcountll(at[j]);
        }
        if (found > 1) {
            uint32_t low = 0;
#pragma unroll
            for (int j = 0; j < J; ++j) low = hi[j] == most ? max(low, lo[j]) : low;
            low = wave_max(low);
            lanes = 0;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                at[j] &= __ballot(lo[j] == low);
                lanes |= at[j];
            }
            lanes &= -lanes;                                // the lowest lane, and its lowest expert
            bool done = false;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                at[j] = done ? 0 : at[j] & lanes;
                done = done || at[j];
            }
        }
        int e = __builtin_ctzll(lanes) * J;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (j > 0) e += at[j] ? j : 0;
            hi[j] = __builtin_amdgcn_inverse_ballot_w64(at[j]) ? 0 : hi[j];
        }
        if (lane == i) mine = e;
    }
    double w = lane < a.top ? room[mine] : 0.0;
    if (a.normalise) {
        const double all = wave_sum(w, a.top);
        w = all == 0.0 ? 0.0 : w / all;
    }
    weight = (float)(w * (double)a.scale);
    wave_sync();                                            // room is free for the next token
}

// Places the routes of a block in the order: WAVES waves with kWaveRoutes each.  next: [WAVES][experts], scan: [WAVES].
// first(e): where a block's routes of expert e begin, counting from the expert's own beginning; total(e): all of them.  EARLY:
// these are in memory, and asked for together with the routes; else they come from the counts in next.
template <int WAVES, bool EARLY, class E, class F, class G>
__device__ inline void place(const RouteArgs& a, int r0, int r1, int32_t* next, int32_t* scan, E expert, F total, G first, bool writes_ends) {
    constexpr int kThreads = 64 * WAVES, kEach = kMostExperts / kThreads;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t* own = next + wave * a.experts;
    const int w0 = r0 + wave * kWaveRoutes;
    int mine[kWaveRoutes / 64];
#pragma unroll
    for (int i = 0; i < kWaveRoutes / 64; ++i) {
        const int r = w0 + 64 * i + lane;
        mine[i] = r < r1 ? expert(r) : -1;
    }
    // neighbouring experts a thread
    const int e0 = kEach * (int)threadIdx.x;
    int count[kEach], from[kEach];
    auto ask = [&]() {
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            count[j] = e0 + j < a.experts ? total(e0 + j) : 0;
            from[j] = e0 + j < a.experts ? first(e0 + j) : 0;
        }
    };
    if constexpr (EARLY) ask();
    for (int e = threadIdx.x; e < WAVES * a.experts; e += kThreads) next[e] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWaveRoutes / 64; ++i)
        if ((uint32_t)mine[i] < (uint32_t)a.experts) atomicAdd(&own[mine[i]], 1);
    __syncthreads();
    if constexpr (!EARLY) ask();
    int sum = 0;                                            // where an expert begins
#pragma unroll
    for (int j = 0; j < kEach; ++j) sum += count[j];
    int upto = sum;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const int other = __shfl_up(upto, s);
        if (lane >= s) upto += other;
    }
    if (lane == 63) scan[wave] = upto;
    __syncthreads();
    int at = upto - sum;
    for (int w = 0; w < wave; ++w) at += scan[w];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int e = e0 + j;
        if (e >= a.experts) break;
        if (writes_ends) a.ends[e] = at;
        int begin = at + from[j];
        for (int w = 0; w < WAVES; ++w) {
            const int n = next[w * a.experts + e];
            next[w * a.experts + e] = begin;
            begin += n;
        }
        at += count[j];
        if (writes_ends && e == a.experts - 1) a.ends[a.experts] = at;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWaveRoutes / 64; ++i) {
        const int e = mine[i];
        const bool there = (uint32_t)e < (uint32_t)a.experts;
        uint64_t same = __ballot(there);
#pragma unroll
        for (int b = 0; b < 10; ++b) {
            const uint64_t set = __ballot(e >> b & 1);
            same &= e >> b & 1 ? set : ~set;
        }
        const int before = __builtin_popcountll(same & (((uint64_t)1 << lane) - 1));
        int base = 0;
        if (there) base = own[e];
        wave_sync();                                        // all have read before the first writes
        if (there) {
            a.order[base + before] = w0 + 64 * i + lane;
            if (before == 0) own[e] = base + __builtin_popcountll(same);
        }
        wave_sync();
    }
}

// Waves of a block: as many as have registers for J experts a lane.
constexpr int waves_of(int j) { return j <= 2 ? 16 : (j <= 8 ? 8 : 4); }

// A block of tokens.  ALONE: it is the only one, and its order follows at once; else its counts.
template <int TYPE, int J, bool ALONE> __global__ __launch_bounds__(64 * waves_of(J)) void route_experts_kernel(RouteArgs a) {
    constexpr int kMost = waves_of(J);
    const int waves = ALONE ? kMost : (int)blockDim.x / 64;
    extern __shared__ __attribute__((aligned(16))) double room[];                        // of each wave; the order's counts
    __shared__ int32_t scan[kMost];
    __shared__ int16_t picked[ALONE ? kAlone * kMostTop : 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int own = J * 64 * (a.top_groups < a.groups ? 2 : 1);
    int32_t* count = (int32_t*)(room + (ALONE ? 0 : waves * own));
    const bool counts = !ALONE && a.ends;
    if (counts) {
        for (int e = threadIdx.x; e < a.experts; e += 64 * waves) count[e] = 0;
        __syncthreads();
    }
    const int64_t t0 = ALONE ? 0 : (int64_t)blockIdx.x * a.block_tokens, t1 = ALONE || t0 + a.block_tokens > a.tokens ? a.tokens : t0 + a.block_tokens;
    const int64_t live = a.live ? *a.live : a.tokens;
    float z[J], ahead[J], bias[J];
    auto fetch = [&](int64_t token, float (&to)[J]) {
        if (token >= t1) return;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int e = lane * J + j;
            to[j] = e < a.experts ? load<TYPE>(a.logits, token * a.stride + e) : -__builtin_inff();
        }
    };
    fetch(t0 + wave, ahead);
#pragma unroll
    for (int j = 0; j < J; ++j) bias[j] = a.bias && lane * J + j < a.experts ? a.bias[lane * J + j] : 0.f;
    for (int64_t token = t0 + wave; token < t1; token += waves) {
#pragma unroll
        for (int j = 0; j < J; ++j) z[j] = ahead[j];
        fetch(token + waves, ahead);
        int mine = -1;
        float weight = 0.f;
        if (token < live) route<TYPE, J>(a, z, bias, room + wave * own, mine, weight);
        if (lane < a.top) {
            a.chosen[token * a.top + lane] = mine;
            a.weights[token * a.top + lane] = weight;
            if (ALONE) picked[token * a.top + lane] = (int16_t)mine;
            if (counts && mine >= 0) atomicAdd(&count[mine], 1);
        }
    }
    if (!a.ends) return;
    __syncthreads();
    if constexpr (ALONE) {
        place<kMost, false>(a, 0, (int)t1 * a.top, count, scan, [&](int r) { return (int)picked[r]; },
                      [&](int e) {
                          int n = 0;
                          for (int w = 0; w < kMost; ++w) n += count[w * a.experts + e];
                          return n;
                      },
                      [](int) { return 0; }, true);
    } else {
        for (int e = threadIdx.x; e < a.experts; e += 64 * waves) a.counts[(int64_t)e * a.row_blocks + blockIdx.x] = count[e];
    }
}

// For each expert, a wave's work, the routes of the blocks before each block, and all of them.
__global__ __launch_bounds__(64) void route_sum_kernel(RouteArgs a) {
    const int lane = threadIdx.x;
    int32_t* p = a.counts + (int64_t)blockIdx.x * a.blocks;
    int sum = 0;
    for (int b0 = 0; b0 < a.blocks; b0 += 256) {
        int n[4], all = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int b = b0 + 4 * lane + i;
            n[i] = b < a.blocks ? p[b] : 0;
            all += n[i];
        }
        int upto = all;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const int other = __shfl_up(upto, s);
            if (lane >= s) upto += other;
        }
        int at = sum + upto - all;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int b = b0 + 4 * lane + i;
            if (b < a.blocks) p[b] = at;
            at += n[i];
        }
        sum += __shfl(upto, 63);
    }
    if (lane == 0) a.totals[blockIdx.x] = sum;
}

template <int WAVES> __global__ __launch_bounds__(64 * WAVES) void route_place_kernel(RouteArgs a) {
    extern __shared__ int32_t next[];
    __shared__ int32_t scan[WAVES];
    const int64_t t0 = (int64_t)blockIdx.x * a.block_tokens, t1 = t0 + a.block_tokens < a.tokens ? t0 + a.block_tokens : a.tokens;
    // few blocks: each adds up the counts of all of them, without the launch between
    constexpr int kEach = kMostExperts / (64 * WAVES);
    int all[kEach] = {}, before[kEach] = {};
    if (a.counts && !a.totals) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int e = kEach * (int)threadIdx.x + j;
            if (e >= a.experts) break;
            const int32_t* p = a.counts + (int64_t)e * kFewBlocks;
#pragma unroll
            for (int b = 0; b < kFewBlocks; ++b) {          // read whole, in wide loads; what no block wrote counts nothing
                const int n = p[b];
                all[j] += b < a.blocks ? n : 0;
                before[j] += b < (int)blockIdx.x ? n : 0;
            }
        }
    }
    auto mine = [&](const int (&v)[kEach], int e) {
        int n = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) n = e % kEach == j ? v[j] : n;
        return n;
    };
    place<WAVES, true>(a, (int)t0 * a.top, (int)t1 * a.top, next, scan, [&](int r) { return a.chosen[r]; },
                 [&](int e) { return a.totals ? a.totals[e] : mine(all, e); },
                 [&](int e) { return a.totals ? a.counts[(int64_t)e * a.blocks + blockIdx.x] : mine(before, e); }, blockIdx.x == 0);
}

template <int TYPE, int J> void launch(const RouteArgs& a, hipStream_t stream) {
    const bool alone = a.blocks == 1 && a.ends;
    const int waves = alone ? waves_of(J) : std::min(waves_of(J), a.block_tokens);
    const size_t room = (size_t)waves * (J * 64) * (a.top_groups < a.groups ? 2 : 1) * sizeof(double);
    if (alone)
        hipLaunchKernelGGL((route_experts_kernel<TYPE, J, true>), dim3(1), dim3(64 * waves),
                           std::max(room, waves * a.experts * sizeof(int32_t)), stream, a);
    else
        hipLaunchKernelGGL((route_experts_kernel<TYPE, J, false>), dim3((unsigned)a.blocks), dim3(64 * waves),
                           room + (a.ends ? a.experts * sizeof(int32_t) : 0), stream, a);
}
// Experts that a lane holds.
int lane_experts(int experts) { return experts <= 64 ? 1 : (experts <= 128 ? 2 : (experts <= 256 ? 4 : (experts <= 512 ? 8 : 16))); }
template <int TYPE> void launch(const RouteArgs& a, hipStream_t stream) {
    switch (lane_experts(a.experts)) {
        case 1: return launch<TYPE, 1>(a, stream);
        case 2: return launch<TYPE, 2>(a, stream);
        case 4: return launch<TYPE, 4>(a, stream);
        case 8: return launch<TYPE, 8>(a, stream);
        default: return launch<TYPE, 16>(a, stream);
    }
}
void launch_place(const RouteArgs& a, hipStream_t stream) {
    const int blocks = std::max(a.blocks, 1);
    if (a.block_tokens * a.top <= 4 * kWaveRoutes)
        hipLaunchKernelGGL((route_place_kernel<4>), dim3((unsigned)blocks), dim3(256), 4 * a.experts * sizeof(int32_t), stream, a);
    else
        hipLaunchKernelGGL((route_place_kernel<16>), dim3((unsigned)blocks), dim3(1024), 16 * a.experts * sizeof(int32_t), stream, a);
}

bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }
// Tokens of a block.  Few are routed and put in order by one block: one to a wave, or two where a lane has one expert (us, one
// launch and two: 24 tokens to 6 of 64 6.7 and 8.7, 64 to 4 of 64 11.3 and 7.9, 32 to 8 of 256 16.3 and 9.4).  More are spread
// over as many blocks as need no launch for their sums, then taken one by a wave (512 tokens to 8 of 256: 16 us with four one
// after the other), and many as the launches after it would have them.
int block_tokens(int64_t tokens, int experts) {
    const int each = lane_experts(experts), waves = waves_of(each);
    if (tokens <= waves * (each == 1 ? 2 : 1)) return kAlone;
    int n = 4;
    while (n < waves && tokens > kFewBlocks * n) n *= 2;
    while (n < kTokens && tokens > 256 * n) n *= 2;
    return n;
}

}  // namespace

extern "C" size_t route_experts_workspace_bytes(int32_t tokens, int32_t experts, int32_t top) {
    if (tokens < 1 || experts < 1 || top < 1 || experts > kMostExperts || top > kMostTop || (int64_t)tokens * top > 1 << 22) return 0;
    const int n = block_tokens(tokens, experts);
    const int64_t blocks = (tokens + (int64_t)n - 1) / n;
    return blocks == 1 ? 0 : (size_t)(blocks <= kFewBlocks ? kFewBlocks : blocks + 1) * experts * sizeof(int32_t);
}

extern "C" wino_status route_experts(const void* logits, int64_t stride, const float* bias, int32_t tokens, int32_t experts,
                                     int32_t top, wino_score score, int32_t groups, int32_t top_groups, int32_t group_best,
                                     int32_t normalise, float scale, const int32_t* live, int32_t* chosen, float* weights,
                                     int32_t* order, int32_t* ends, wino_float_type type, void* workspace, size_t workspace_bytes,
                                     hipStream_t stream) {
    if (type != WINO_BF16 && type != WINO_FP16 && type != WINO_FP32) return WINO_EINVAL;
    if (score != WINO_SCORE_SOFTMAX && score != WINO_SCORE_SIGMOID) return WINO_EINVAL;
    if (tokens < 0 || experts < 1 || top < 1 || groups < 1 || top_groups < 1 || top_groups > groups || experts % groups != 0)
        return WINO_EINVAL;
    if ((group_best != 1 && group_best != 2) || (group_best == 2 && top_groups < groups && experts / groups < 2)) return WINO_EINVAL;
    if (top > top_groups * (experts / groups) || (normalise != 0 && normalise != 1) || !(__builtin_fabsf(scale) < __builtin_inff()))
        return WINO_EINVAL;
    if (tokens > 0 && (order != nullptr) != (ends != nullptr)) return WINO_EINVAL;      // an empty order may have no address
    if (experts > kMostExperts || top > kMostTop || groups > kMostGroups || (int64_t)tokens * top > 1 << 22) return WINO_EUNSUPPORTED;
    if (tokens > 0 && (!logits || !chosen || !weights)) return WINO_EINVAL;
    if (tokens > 1 && stride < experts) return WINO_EINVAL;
    if (!aligned4(bias) || !aligned4(live) || !aligned4(chosen) || !aligned4(weights) || !aligned4(order) || !aligned4(ends) ||
        !aligned4(workspace) || ((uintptr_t)logits & (type == WINO_FP32 ? 3 : 1)))
        return WINO_EUNSUPPORTED;
    const size_t need = route_experts_workspace_bytes(tokens, experts, top);
    if (ends && need > 0 && (!workspace || workspace_bytes < need)) return WINO_EINVAL;
    if (tokens == 0 && !ends) return WINO_OK;
    // without an order few tokens are spread as far as they go (32 tokens to 8 of 256: 4.8 us, by one block 14.5)
    const int32_t n = ends || tokens > 4096 ? block_tokens(tokens, experts) : 4, blocks = (int32_t)((tokens + (int64_t)n - 1) / n);
    RouteArgs a = {logits, bias, live, chosen, weights, stride, tokens, experts, top, groups, experts / groups, top_groups,
                   group_best, score == WINO_SCORE_SIGMOID, normalise, 1, scale, winof4::make_fastdiv((uint32_t)(experts / groups)),
                   order, ends, nullptr, nullptr, blocks, n, std::max(blocks, kFewBlocks)};
    while (2 * a.group_lanes * groups <= 64) a.group_lanes *= 2;
    if (blocks > 1 && ends) a.counts = (int32_t*)workspace;
    if (blocks > kFewBlocks && ends) a.totals = a.counts + (int64_t)blocks * experts;
    if (blocks > 0) type == WINO_BF16 ? launch<WINO_BF16>(a, stream) : type == WINO_FP16 ? launch<WINO_FP16>(a, stream) : launch<WINO_FP32>(a, stream);
    if (ends && blocks != 1) {
        if (a.totals) hipLaunchKernelGGL(route_sum_kernel, dim3((unsigned)experts), dim3(64), 0, stream, a);
        launch_place(a, stream);
    }
    return hipGetLastError() == hipSuccess ? WINO_OK : WINO_EHIP;
}
