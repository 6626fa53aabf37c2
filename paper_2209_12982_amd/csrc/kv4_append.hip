// Rotation of queries and keys, and quantization of keys and values into the
// paged 4-bit cache (mx4.h), in one pass over the new tokens.
//
// Rotation of the first r dimensions of a head by the token's angle a_j, with
// (c, s) = (cos a_j, sin a_j): (u, w) -> (u c - w s, w c + u s) for the pairs
// (x_j, x_{j + r/2}) or (x_{2j}, x_{2j+1}).  Every product and sum is rounded
// once to fp32 (no fused multiply-add), so the result does not depend on how
// the compiler groups them, and a key always gets the same code.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "mx4.h"
#include "wino_device.h"
#include "winof4.h"

namespace {
using namespace mx4;

struct AppendArgs {
    const void *q, *k, *v;
    void *q_out, *k_out, *v_out;
    const float* cos_sin;
    const int32_t* positions;
    const int64_t* slots;
    uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    int64_t q_stride, k_stride, v_stride, slot_end;
    int32_t first, threads;     // of a launch: its first token, and its threads (a multiple of 4)
    int32_t heads, kv_heads, dim, rot, table_rows, page, values;
    winof4::FastDiv by_eights, by_heads, by_page;       // by dim / 8, by the heads of q, k and v together, by page
};

// The bytes bound it: every value is read once and written once in 16 bits,
// keys and values once more in 4.  A thread takes 8 neighbouring dimensions of
// one head of one token; the four threads of a 32-group are neighbours in a
// wave.  With halves rotated it reads the 8 partners too (from the cache:
// another thread reads them as its own), which needs neither LDS nor a barrier.
// Its indices are 32 bits wide, divided by multiplying: with 64-bit divisions it
// took 50.0 us for 8200 tokens of 32 + 2 x 8 heads of 128, now 46.6, 4.6 TB/s
// (a copy of 2 GiB: 4.8); the first hundred calls of a burst, before the clock
// settles, take 53.
// LARGE: outputs that no L2 holds until somebody reads them do not go through it, 2.6 us of those 50.
template <int TYPE, int ROTARY, bool LARGE>
__global__ __launch_bounds__(256) void kv4_append_kernel(AppendArgs a) {
#pragma clang fp contract(off)
    typedef typename Half<TYPE>::type T;
    typedef T T8 __attribute__((ext_vector_type(8)));
    const uint32_t gid = blockIdx.x * 256 + threadIdx.x;
    if (gid >= (uint32_t)a.threads) return;           // whole groups of four
    const uint32_t th = winof4::fast_div(gid, a.by_eights), t = winof4::fast_div(th, a.by_heads);
    const int d0 = (int)(gid - th * a.by_eights.d) * 8;
    const int64_t tok = a.first + (int)t;
    int h = (int)(th - t * a.by_heads.d);
    const int kind = h < a.heads ? 0 : (h < a.heads + a.kv_heads ? 1 : 2);
    h -= kind == 0 ? 0 : (kind == 1 ? a.heads : a.heads + a.kv_heads);
    const T* src = kind == 0 ? (const T*)a.q + tok * a.q_stride
                             : (kind == 1 ? (const T*)a.k + tok * a.k_stride : (const T*)a.v + tok * a.v_stride);
    src += (int64_t)h * a.dim;

    float x[8];
    {
        const T8 t = *(const T8*)(src + d0);
        for (int i = 0; i < 8; ++i) x[i] = (float)t[i];
    }
    const int32_t pos = a.positions[tok];
    const bool placed = pos >= 0 && pos < a.table_rows;
    if (kind < 2 && d0 < a.rot && placed) {
        const int half = a.rot / 2;
        const float* row = a.cos_sin + (int64_t)pos * a.rot;
        if constexpr (ROTARY == WINO_ROTARY_HALVES) {
            const bool low = d0 < half;
            const int j = low ? d0 : d0 - half;
            const T8 t = *(const T8*)(src + (low ? d0 + half : d0 - half));
            for (int i = 0; i < 8; ++i) {
                const float p = (float)t[i], c = row[j + i], s = row[half + j + i];
                const float own = x[i] * c, other = p * s;
                x[i] = low ? own - other : own + other;
            }
        } else {
            for (int i = 0; i < 4; ++i) {
                const float c = row[d0 / 2 + i], s = row[half + d0 / 2 + i];
                const float u = x[2 * i], w = x[2 * i + 1];
                const float uc = u * c, ws = w * s, wc = w * c, us = u * s;
                x[2 * i] = uc - ws;
                x[2 * i + 1] = wc + us;
            }
        }
    }
    if (!placed)
        for (int i = 0; i < 8; ++i) x[i] = __builtin_nanf("");
    T* out = (T*)(kind == 0 ? a.q_out : (kind == 1 ? a.k_out : a.v_out));
    if (kind > 0) {
        float amax = 0.f;
        bool fine = true;
        for (int i = 0; i < 8; ++i) {
            const float b = __builtin_fabsf(x[i]);
            fine = fine && b < __builtin_inff();
            amax = b > amax ? b : amax;
        }
        if (!fine) amax = __builtin_inff();
        for (int o = 1; o < 4; o <<= 1) {
            const float b = __shfl_xor(amax, o);
            amax = b > amax ? b : amax;
        }
        const uint32_t s = scale_byte(amax);
        const float inv = inverse_scale(s);
        uint32_t word = 0;
        for (int i = 0; i < 8; ++i) word |= (s == 255u ? 0u : encode(x[i], inv)) << (4 * i);
        const int64_t slot = a.slots[tok];
        if (placed && slot >= 0 && slot < a.slot_end) {
            const int64_t pg = slot >> 31 ? slot / a.page : winof4::fast_div((uint32_t)slot, a.by_page);
            const int64_t at = (pg * a.kv_heads + h) * a.page + (slot - pg * a.page);
            *(uint32_t*)((kind == 1 ? a.k_codes : a.v_codes) + at * (a.dim / 2) + d0 / 2) = word;
            if (d0 % kGroup == 0) (kind == 1 ? a.k_scales : a.v_scales)[at * (a.dim / kGroup) + d0 / kGroup] = (uint8_t)s;
        }
        if (a.values == KV4_CACHED) {
            const float sc = scale_value(s);
            for (int i = 0; i < 8; ++i) x[i] = code_value(word >> (4 * i)) * sc;
        }
    }
    if (out) {
        T8 t;
        for (int i = 0; i < 8; ++i) t[i] = (T)x[i];
        T8* at = (T8*)(out + (tok * (kind == 0 ? a.heads : a.kv_heads) + h) * a.dim + d0);
        if constexpr (LARGE)
            __builtin_nontemporal_store(t, at);
        else
            *at = t;
    }
}

template <int TYPE, int ROTARY> void launch(const AppendArgs& a, bool large, hipStream_t stream) {
    const dim3 grid((unsigned)((a.threads + 255) / 256)), block(256);
    if (large)
        hipLaunchKernelGGL((kv4_append_kernel<TYPE, ROTARY, true>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((kv4_append_kernel<TYPE, ROTARY, false>), grid, block, 0, stream, a);
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace

extern "C" wino_status kv4_append(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                                  int64_t v_stride, int32_t tokens, int32_t heads, const float* cos_sin,
                                  int32_t table_rows, int32_t rot, const int32_t* positions, const int64_t* slots,
                                  const kv4_cache* cache, void* q_out, void* k_out, void* v_out, wino_rotary rotary,
                                  kv4_values values, wino_float_type type, hipStream_t stream) {
    if (!cache || (type != WINO_BF16 && type != WINO_FP16)) return WINO_EINVAL;
    if ((rotary != WINO_ROTARY_HALVES && rotary != WINO_ROTARY_PAIRS) || (values != KV4_ROTATED && values != KV4_CACHED))
        return WINO_EINVAL;
    const kv4_cache& c = *cache;
    if (c.pages < 0 || c.kv_heads < 1 || c.page_size < 1 || tokens < 0 || heads < 0 || table_rows < 0 || rot < 0)
        return WINO_EINVAL;
    if (c.head_dim < 1 || rot > c.head_dim) return WINO_EINVAL;
    if (c.page_size % 16 || c.head_dim % kGroup || c.head_dim > 256 || rot % 16) return WINO_EUNSUPPORTED;
    if (c.kv_heads > 4096 || heads > 65536 || c.pages > (int64_t)1 << 40 || c.page_size > 1 << 20)
        return WINO_EUNSUPPORTED;
    if (tokens == 0) return WINO_OK;                    // empty tensors may have no address
    if ((heads > 0) != (q_out != nullptr) || (heads > 0 && !q) || !k || !v || (rot > 0 && !cos_sin) || !positions || !slots) return WINO_EINVAL;
    if (c.pages > 0 && (!c.k_codes || !c.k_scales || !c.v_codes || !c.v_scales)) return WINO_EINVAL;
    const int64_t dim = c.head_dim;
    if (tokens > 1 && ((heads > 0 && q_stride < heads * dim) || k_stride < c.kv_heads * dim || v_stride < c.kv_heads * dim))
        return WINO_EINVAL;
    if (tokens > 1 && ((q_stride | k_stride | v_stride) & 7)) return WINO_EUNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(k_out) || !aligned16(v_out) ||
        !aligned16(c.k_codes) || !aligned16(c.v_codes) || !aligned16(cos_sin))
        return WINO_EUNSUPPORTED;
    AppendArgs a = {q, k, v, q_out, k_out, v_out, cos_sin, positions, slots,
                    c.k_codes, c.k_scales, c.v_codes, c.v_scales, q_stride, k_stride, v_stride,
                    c.pages * c.page_size, 0, 0, heads, c.kv_heads, c.head_dim, rot, table_rows, c.page_size, values,
                    winof4::make_fastdiv((uint32_t)(dim / 8)), winof4::make_fastdiv((uint32_t)(heads + 2 * c.kv_heads)),
                    winof4::make_fastdiv((uint32_t)c.page_size)};
    // threads of a token; as many tokens a launch as 32 bits count the threads of
    const int64_t each = (int64_t)(heads + 2 * c.kv_heads) * (dim / 8), most = (1 << 30) / each;
    const bool large = tokens * each * 16 > 32 << 20;
    for (int64_t t0 = 0; t0 < tokens; t0 += most) {
        a.first = (int32_t)t0;
        a.threads = (int32_t)(std::min<int64_t>(most, tokens - t0) * each);
        if (type == WINO_BF16)
            rotary == WINO_ROTARY_HALVES ? launch<WINO_BF16, WINO_ROTARY_HALVES>(a, large, stream)
                                         : launch<WINO_BF16, WINO_ROTARY_PAIRS>(a, large, stream);
        else
            rotary == WINO_ROTARY_HALVES ? launch<WINO_FP16, WINO_ROTARY_HALVES>(a, large, stream)
                                         : launch<WINO_FP16, WINO_ROTARY_PAIRS>(a, large, stream);
        if (hipGetLastError() != hipSuccess) return WINO_EHIP;
    }
    return WINO_OK;
}
