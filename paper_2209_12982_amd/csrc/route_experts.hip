// Routing of tokens to experts: scores, the best experts of the best groups, their weights, and the routes in the order of
// their experts.
//
//   s = softmax(l) or 1 / (1 + exp(-l)) over a token's experts, c = s + bias
//   a group's value is the sum of its `group_best` (1 or 2) largest c; the `top_groups` groups of the largest values stay
//   chosen: the `top` largest c among their experts, the largest first; ties go to the lowest index, not-a-numbers count as
//   minus infinity;  weight = s (over the sum of the chosen s, where they are normalised) times `scale`
//
// Scores are held in 64 bits: which expert comes first hangs on differences that 32 bits do not hold, and the sizes are
// small.  A wave takes a token and holds its values, neighbouring experts in a lane; an expert is found by a maximum over
// the wave.
//
// The order is a counting sort by expert, stable: counts for each block of routes, their sums over the blocks, and then
// each route's place.  No atomics decide a place, so the order is the same each time.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "mx4.h"
#include "wino_device.h"
#include "winof4.h"

namespace {
using namespace mx4;

constexpr int kMostExperts = 1024, kMostTop = 32, kMostGroups = 64;
constexpr int kBlock = 2048;            // routes that a workgroup counts and places

struct RouteArgs {
    const void* logits;
    const float* bias;
    const int32_t* live;
    int32_t* chosen;
    float* weights;
    int64_t stride;
    int32_t tokens, experts, top, groups, size, top_groups, group_best, sigmoid, normalise;
    float scale;
    winof4::FastDiv by_size;
};
struct OrderArgs {
    const int32_t* chosen;
    int32_t *order, *ends, *counts, *totals;    // counts: [blocks][experts], later what comes before; totals: [experts]
    int32_t routes, experts, blocks;
};

template <int TYPE> __device__ inline double load(const void* p, int64_t at) {
    if (TYPE == WINO_BF16) return (double)(float)((const __bf16*)p)[at];
    if (TYPE == WINO_FP16) return (double)(float)((const _Float16*)p)[at];
    return (double)((const float*)p)[at];
}

// Order of doubles as whole numbers; every number is above 0.
__device__ inline uint64_t ordered(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v + 0.0);      // -0 is 0
    return b >> 63 ? ~b : b | (uint64_t)1 << 63;
}
__device__ inline uint64_t wave_max(uint64_t v) {
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) {
        const uint64_t o = __shfl_xor((unsigned long long)v, s);
        v = o > v ? o : v;
    }
    return v;
}

// What is not a number counts as minus infinity.
__device__ inline double number(double v) { return v == v ? v : -__builtin_inf(); }

template <int TYPE, int J> __global__ __launch_bounds__(256) void route_experts_kernel(RouteArgs a) {
    constexpr int kWaves = 4;
    __shared__ double values[kWaves][J * 64], group_value[kWaves][kMostGroups];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t token = (int64_t)blockIdx.x * kWaves + wave;
    if (token >= a.tokens) return;
    int32_t* chosen = a.chosen + token * a.top;
    float* weights = a.weights + token * a.top;
    if (a.live && token >= *a.live) {
        if (lane < a.top) chosen[lane] = -1, weights[lane] = 0.f;
        return;
    }
    const int64_t row = token * a.stride;
    double s[J], top = -__builtin_inf();
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int e = lane * J + j;
        s[j] = e < a.experts ? load<TYPE>(a.logits, row + e) : -__builtin_inf();
        top = s[j] > top || s[j] != s[j] ? s[j] : top;
    }
    double sum = 0.0;
    if (!a.sigmoid) {
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            const double o = __shfl_xor(top, d);
            top = o > top || o != o ? o : top;              // a NaN stays
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
            s[j] = lane * J + j < a.experts ? exp(s[j] - top) : 0.0;
            sum += s[j];
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    }
    uint64_t key[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int e = lane * J + j;
        s[j] = a.sigmoid ? 1.0 / (1.0 + exp(-s[j])) : s[j] / sum;
        const double c = number(a.bias && e < a.experts ? s[j] + (double)a.bias[e] : s[j]);
        key[j] = e < a.experts ? ordered(c) : 0;
        if (a.groups > 1) values[wave][e] = c;
    }
    if (a.top_groups < a.groups) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        double first = -__builtin_inf(), second = -__builtin_inf();
        if (lane < a.groups) {
            for (int i = 0; i < a.size; ++i) {
                const double c = values[wave][lane * a.size + i];
                second = c > first ? first : (c > second ? c : second);
                first = c > first ? c : first;
            }
            group_value[wave][lane] = number(a.group_best == 2 ? first + second : first);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        int before = 0;
        const double mine = group_value[wave][min(lane, a.groups - 1)];
        for (int g = 0; g < a.groups; ++g) {
            const double v = group_value[wave][g];
            before += v > mine || (v == mine && g < lane) ? 1 : 0;
        }
        const uint64_t kept = __ballot(lane < a.groups && before < a.top_groups);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const uint32_t g = winof4::fast_div((uint32_t)min(lane * J + j, a.experts - 1), a.by_size);
            if (!(kept >> g & 1)) key[j] = 0;
        }
    }
    int mine = 0;                                           // lane i: the i-th expert
    for (int i = 0; i < a.top; ++i) {
        uint64_t best = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) best = key[j] > best ? key[j] : best;
        const uint64_t most = wave_max(best);
        const int l = __builtin_ctzll(__ballot(best == most));
        int at = 0;
        bool found = false;
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (!found && key[j] == most) {
                found = true;
                at = j;
                if (lane == l) key[j] = 0;
            }
        const int e = l * J + __shfl(at, l);
        if (lane == i) mine = e;
    }
    double w = 0.0;
    if (lane < a.top) {
        const double z = load<TYPE>(a.logits, row + mine);
        w = a.sigmoid ? 1.0 / (1.0 + exp(-z)) : exp(z - top) / sum;
    }
    if (a.normalise) {
        double all = w;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) all += __shfl_xor(all, d);
        w = all == 0.0 ? 0.0 : w / all;
    }
    if (lane < a.top) {
        chosen[lane] = mine;
        weights[lane] = (float)(w * (double)a.scale);
    }
}

__global__ __launch_bounds__(256) void route_count_kernel(OrderArgs a) {
    __shared__ int32_t count[kMostExperts];
    for (int e = threadIdx.x; e < a.experts; e += 256) count[e] = 0;
    __syncthreads();
    const int r0 = blockIdx.x * kBlock, r1 = min(r0 + kBlock, a.routes);
    for (int r = r0 + (int)threadIdx.x; r < r1; r += 256) {
        const int e = a.chosen[r];
        if ((uint32_t)e < (uint32_t)a.experts) atomicAdd(&count[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += 256) a.counts[(int64_t)blockIdx.x * a.experts + e] = count[e];
}

// For each expert, the routes of the blocks before each block, and all of them.
__global__ __launch_bounds__(64) void route_sum_kernel(OrderArgs a) {
    const int e = blockIdx.x * 64 + threadIdx.x;
    if (e >= a.experts) return;
    int sum = 0;
    for (int b = 0; b < a.blocks; ++b) {
        int32_t* p = a.counts + (int64_t)b * a.experts + e;
        const int n = *p;
        *p = sum;
        sum += n;
    }
    a.totals[e] = sum;
}

__global__ __launch_bounds__(256) void route_place_kernel(OrderArgs a) {
    constexpr int kWaves = 4, kMine = kBlock / kWaves;
    __shared__ int32_t next[kWaves][kMostExperts];          // where each wave's next route of an expert goes
    __shared__ int32_t sums[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int e = threadIdx.x; e < kWaves * kMostExperts; e += 256) next[e / kMostExperts][e % kMostExperts] = 0;
    __syncthreads();
    const int r0 = blockIdx.x * kBlock + wave * kMine;
    for (int i = 0; i < kMine; i += 64) {
        const int r = r0 + i + lane, e = r < a.routes ? a.chosen[r] : -1;
        if ((uint32_t)e < (uint32_t)a.experts) atomicAdd(&next[wave][e], 1);
    }
    __syncthreads();
    // four neighbouring experts a thread: where an expert begins, and what comes before this block
    int total[4], mine = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int e = 4 * threadIdx.x + j;
        total[j] = e < a.experts && a.totals ? a.totals[e] : 0;
        mine += total[j];
    }
    int upto = mine;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const int other = __shfl_up(upto, s);
        if (lane >= s) upto += other;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int at = upto - mine;
    for (int w = 0; w < wave; ++w) at += sums[w];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int e = 4 * threadIdx.x + j;
        if (e < a.experts) {
            if (blockIdx.x == 0) a.ends[e] = at;
            int place = at + (a.totals ? a.counts[(int64_t)blockIdx.x * a.experts + e] : 0);
            for (int w = 0; w < kWaves; ++w) {
                const int n = next[w][e];
                next[w][e] = place;
                place += n;
            }
            at += total[j];
            if (blockIdx.x == 0 && e == a.experts - 1) a.ends[a.experts] = at;
        }
    }
    __syncthreads();
    for (int i = 0; i < kMine; i += 64) {
        const int r = r0 + i + lane, e = r < a.routes ? a.chosen[r] : -1;
        const bool there = (uint32_t)e < (uint32_t)a.experts;
        uint64_t same = __ballot(there);
#pragma unroll
        for (int b = 0; b < 10; ++b) {
            const uint64_t set = __ballot(e >> b & 1);
            same &= e >> b & 1 ? set : ~set;
        }
        const int before = __builtin_popcountll(same & (((uint64_t)1 << lane) - 1));
        int base = 0;
        if (there) base = next[wave][e];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // all have read before the first writes
        if (there) {
            a.order[base + before] = r;
            if (before == 0) next[wave][e] = base + __builtin_popcountll(same);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

template <int TYPE, int J> void launch(const RouteArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL((route_experts_kernel<TYPE, J>), dim3((unsigned)((a.tokens + 3) / 4)), dim3(256), 0, stream, a);
}
template <int TYPE> void launch(const RouteArgs& a, hipStream_t stream) {
    const int j = (a.experts + 63) / 64;
    j <= 1 ? launch<TYPE, 1>(a, stream)
           : j <= 2 ? launch<TYPE, 2>(a, stream)
                    : j <= 4 ? launch<TYPE, 4>(a, stream) : j <= 8 ? launch<TYPE, 8>(a, stream) : launch<TYPE, 16>(a, stream);
}

bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }
int64_t blocks_of(int64_t routes) { return (routes + kBlock - 1) / kBlock; }

}  // namespace

extern "C" size_t route_experts_workspace_bytes(int32_t tokens, int32_t experts, int32_t top) {
    if (tokens < 1 || experts < 1 || top < 1 || experts > kMostExperts || top > kMostTop || (int64_t)tokens * top > 1 << 22) return 0;
    return (size_t)(blocks_of((int64_t)tokens * top) + 1) * experts * sizeof(int32_t);
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
    const int64_t routes = (int64_t)tokens * top;
    if (ends && tokens > 0 && (!workspace || workspace_bytes < route_experts_workspace_bytes(tokens, experts, top))) return WINO_EINVAL;
    if (tokens == 0 && !ends) return WINO_OK;
    if (tokens > 0) {
        const RouteArgs a = {logits, bias, live, chosen, weights, stride, tokens, experts, top, groups, experts / groups, top_groups,
                             group_best, score == WINO_SCORE_SIGMOID, normalise, scale,
                             winof4::make_fastdiv((uint32_t)(experts / groups))};
        type == WINO_BF16 ? launch<WINO_BF16>(a, stream)
                          : type == WINO_FP16 ? launch<WINO_FP16>(a, stream) : launch<WINO_FP32>(a, stream);
    }
    if (ends && hipGetLastError() == hipSuccess) {
        OrderArgs o = {chosen, order, ends, (int32_t*)workspace, nullptr, (int32_t)routes, experts, (int32_t)blocks_of(routes)};
        if (o.blocks > 0) {
            o.totals = o.counts + (int64_t)o.blocks * experts;
            hipLaunchKernelGGL(route_count_kernel, dim3((unsigned)o.blocks), dim3(256), 0, stream, o);
            hipLaunchKernelGGL(route_sum_kernel, dim3((unsigned)((experts + 63) / 64)), dim3(64), 0, stream, o);
        }
        hipLaunchKernelGGL(route_place_kernel, dim3((unsigned)std::max(o.blocks, 1)), dim3(256), 0, stream, o);
    }
    return hipGetLastError() == hipSuccess ? WINO_OK : WINO_EHIP;
}
