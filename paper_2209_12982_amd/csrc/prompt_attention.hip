// Causal attention over whole prompts: packed sequences of different lengths,
// grouped heads, keys and values in 16 bits.
#include <hip/hip_runtime.h>

#include "mx4.h"
#include "winof4.h"

namespace {
using namespace mx4;

struct PromptArgs {
    const void *q, *k, *v;
    void* out;
    const int32_t *cu_q, *cu_k;
    int64_t q_stride, k_stride, v_stride;
    int32_t seqs, total_q, total_k, heads, kv_heads, dim, causal;
    float scale;
};

// One wave per query row and head, 64 keys at a time.
template <int TYPE>
__global__ __launch_bounds__(64) void prompt_attention_kernel(PromptArgs a) {
    typedef typename Half<TYPE>::type T;
    __shared__ float qs[256], ps[64];
    const int lane = threadIdx.x, h = blockIdx.x % a.heads, kvh = h / (a.heads / a.kv_heads);
    const int row = blockIdx.x / a.heads;
    int s = 0;
    while (s < a.seqs && !(row >= a.cu_q[s] && row < a.cu_q[s + 1])) ++s;
    T* out = (T*)a.out + ((int64_t)row * a.heads + h) * a.dim;
    if (s == a.seqs) return;
    const int q0 = max(0, a.cu_q[s]), q1 = min(a.cu_q[s + 1], a.total_q);
    const int k0 = max(0, min(a.cu_k[s], a.total_k)), n = max(0, min(a.cu_k[s + 1], a.total_k) - k0);
    const int end = a.causal ? n - (q1 - q0) + 1 + (row - q0) : n;
    const T* q = (const T*)a.q + (int64_t)row * a.q_stride + (int64_t)h * a.dim;
    for (int d = lane; d < a.dim; d += 64) qs[d] = (float)q[d] * a.scale;
    float top = -__builtin_inff(), sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int t0 = 0; t0 < end; t0 += 64) {
        const int t = t0 + lane;
        __syncthreads();
        float z = -__builtin_inff();
        if (t < end) {
            const T* k = (const T*)a.k + (int64_t)(k0 + t) * a.k_stride + (int64_t)kvh * a.dim;
            z = 0.f;
            for (int d = 0; d < a.dim; ++d) z += qs[d] * (float)k[d];
        }
        float m = z;
        for (int i = 32; i; i >>= 1) m = fmaxf(m, __shfl_xor(m, i));
        m = fmaxf(m, top);
        const float base = m == -__builtin_inff() ? 0.f : m;
        const float p = t < end ? expf(z - base) : 0.f, alpha = expf(top - base);
        top = m;
        ps[lane] = p;
        float part = p;
        for (int i = 32; i; i >>= 1) part += __shfl_xor(part, i);
        sum = sum * alpha + part;
        __syncthreads();
        for (int e = 0; e < 4; ++e) {
            const int d = lane + 64 * e;
            if (d >= a.dim) break;
            float acc = o[e] * alpha;
            for (int i = 0; i < 64 && t0 + i < end; ++i)
                acc += ps[i] * (float)((const T*)a.v)[(int64_t)(k0 + t0 + i) * a.v_stride + (int64_t)kvh * a.dim + d];
            o[e] = acc;
        }
    }
    for (int e = 0; e < 4; ++e) {
        const int d = lane + 64 * e;
        if (d < a.dim) out[d] = (T)(sum == 0.f ? 0.f : o[e] / sum);
    }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

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
    if (seqs > 65536 || heads > 65536) return WINO_EUNSUPPORTED;
    if (total_q == 0) return WINO_OK;
    if (!q || !out || (total_k > 0 && (!k || !v)) || (seqs > 0 && (!cu_q || !cu_k))) return WINO_EINVAL;
    const int64_t dim = head_dim;
    if ((total_q > 1 && q_stride < heads * dim) || (total_k > 1 && (k_stride < kv_heads * dim || v_stride < kv_heads * dim)))
        return WINO_EINVAL;
    if ((total_q > 1 && (q_stride & 7)) || (total_k > 1 && ((k_stride | v_stride) & 7)) || !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out))
        return WINO_EUNSUPPORTED;
    const int64_t blocks = (int64_t)total_q * heads;
    if (blocks > 0x7fffffffll) return WINO_EUNSUPPORTED;
    PromptArgs a = {q, k, v, out, cu_q, cu_k, q_stride, k_stride, v_stride, seqs, total_q, total_k,
                    heads, kv_heads, head_dim, causal, scale};
    if (type == WINO_BF16)
        hipLaunchKernelGGL(prompt_attention_kernel<WINO_BF16>, dim3((unsigned)blocks), dim3(64), 0, stream, a);
    else
        hipLaunchKernelGGL(prompt_attention_kernel<WINO_FP16>, dim3((unsigned)blocks), dim3(64), 0, stream, a);
    return hipGetLastError() == hipSuccess ? WINO_OK : WINO_EHIP;
}
