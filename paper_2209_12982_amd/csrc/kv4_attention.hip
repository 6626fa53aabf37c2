// Attention over the paged 4-bit cache (mx4.h) for one or a few query tokens
// of each sequence.
#include <hip/hip_runtime.h>

#include "mx4.h"
#include "winof4.h"

namespace {
using namespace mx4;

struct DecodeArgs {
    const void* q;
    void* out;
    const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    const int32_t *table, *lens;
    int64_t q_stride, pages;
    int32_t q_len, heads, kv_heads, dim, page, max_pages;
    float scale;
};

// One wave per query row and head, 64 tokens at a time: a lane scores one
// token, then the lanes take dimensions.
template <int TYPE>
__global__ __launch_bounds__(64) void kv4_attention_kernel(DecodeArgs a) {
    typedef typename Half<TYPE>::type T;
    __shared__ float qs[256], ps[64];
    __shared__ int64_t at_s[64];
    const int lane = threadIdx.x, h = blockIdx.x % a.heads, kvh = h / (a.heads / a.kv_heads);
    const int64_t row = blockIdx.x / a.heads;
    const int b = (int)(row / a.q_len), i = (int)(row % a.q_len);
    const int64_t room = (int64_t)a.max_pages * a.page;
    int64_t len = a.lens[b];
    len = len < 0 ? 0 : (len > room ? room : len);
    const int64_t end = len - a.q_len + 1 + i;        // tokens that the row sees
    const T* q = (const T*)a.q + row * a.q_stride + (int64_t)h * a.dim;
    for (int d = lane; d < a.dim; d += 64) qs[d] = (float)q[d] * a.scale;
    float top = -__builtin_inff(), sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t t0 = 0; t0 < end; t0 += 64) {
        const int64_t t = t0 + lane;
        int64_t pg = t < end ? a.table[(int64_t)b * a.max_pages + t / a.page] : -1;
        const bool there = pg >= 0 && pg < a.pages;
        const int64_t at = there ? (pg * a.kv_heads + kvh) * a.page + t % a.page : -1;
        float z = -__builtin_inff();
        __syncthreads();
        if (there) {
            z = 0.f;
            for (int g = 0; g < a.dim / kGroup; ++g) {
                float part = 0.f;
                for (int d = 0; d < 16; ++d) {
                    const uint32_t c = a.k_codes[at * (a.dim / 2) + g * 16 + d];
                    part += code_value(c & 15u) * qs[g * 32 + 2 * d] + code_value(c >> 4) * qs[g * 32 + 2 * d + 1];
                }
                z += part * scale_value(a.k_scales[at * (a.dim / kGroup) + g]);
            }
        }
        float m = z;
        for (int s = 32; s; s >>= 1) m = fmaxf(m, __shfl_xor(m, s));
        m = fmaxf(m, top);
        const float base = m == -__builtin_inff() ? 0.f : m;
        const float p = there ? expf(z - base) : 0.f, alpha = expf(top - base);
        top = m;
        ps[lane] = p;
        at_s[lane] = at;
        float s = p;
        for (int k = 32; k; k >>= 1) s += __shfl_xor(s, k);
        sum = sum * alpha + s;
        __syncthreads();
        for (int e = 0; e < 4; ++e) {
            const int d = lane + 64 * e;
            if (d >= a.dim) break;
            float acc = o[e] * alpha;
            for (int k = 0; k < 64; ++k) {
                if (at_s[k] < 0) continue;
                const uint32_t c = a.v_codes[at_s[k] * (a.dim / 2) + d / 2] >> (4 * (d & 1));
                acc += ps[k] * (code_value(c) * scale_value(a.v_scales[at_s[k] * (a.dim / kGroup) + d / kGroup]));
            }
            o[e] = acc;
        }
    }
    T* out = (T*)a.out + (row * a.heads + h) * a.dim;
    for (int e = 0; e < 4; ++e) {
        const int d = lane + 64 * e;
        if (d < a.dim) out[d] = (T)(sum == 0.f ? 0.f : o[e] / sum);
    }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace

extern "C" size_t kv4_attention_workspace_bytes(int32_t batch, int32_t q_len, int32_t heads, int32_t kv_heads,
                                                int32_t head_dim, int32_t max_pages, int32_t page_size) {
    (void)batch, (void)q_len, (void)heads, (void)kv_heads, (void)head_dim, (void)max_pages, (void)page_size;
    return 0;
}

extern "C" wino_status kv4_attention(const void* q, int64_t q_stride, const kv4_cache* cache,
                                     const int32_t* block_table, int32_t max_pages, const int32_t* lens, void* out,
                                     int32_t batch, int32_t q_len, int32_t heads, float scale, wino_float_type type,
                                     void* workspace, size_t workspace_bytes, hipStream_t stream) {
    (void)workspace, (void)workspace_bytes;
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
    if ((many && (q_stride & 7)) || !aligned16(q) || !aligned16(out) || !aligned16(c.k_codes) || !aligned16(c.v_codes))
        return WINO_EUNSUPPORTED;
    const int64_t blocks = (int64_t)batch * q_len * heads;
    if (blocks > 0x7fffffffll) return WINO_EUNSUPPORTED;
    DecodeArgs a = {q, out, c.k_codes, c.k_scales, c.v_codes, c.v_scales, block_table, lens, q_stride, c.pages,
                    q_len, heads, c.kv_heads, c.head_dim, c.page_size, max_pages, scale};
    if (type == WINO_BF16)
        hipLaunchKernelGGL(kv4_attention_kernel<WINO_BF16>, dim3((unsigned)blocks), dim3(64), 0, stream, a);
    else
        hipLaunchKernelGGL(kv4_attention_kernel<WINO_FP16>, dim3((unsigned)blocks), dim3(64), 0, stream, a);
    return hipGetLastError() == hipSuccess ? WINO_OK : WINO_EHIP;
}
