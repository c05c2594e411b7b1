// Attention over the quantized cache of kv_cache.hip.
//
// Sequence b has kv_lens[b] cached tokens, the last lq of which its lq queries belong to:
// query i sees the keys j < kv_lens[b], and with the causal rule j <= kv_lens[b] - lq + i. Its
// output is sum_j p_j v_j / sum_j p_j with p_j = exp(scale q.k_j - max), zeros where it sees
// no key.
#include "mx_internal.hpp"
#include "mx_math.hpp"

namespace w8a8 {
namespace {

using namespace mx;

__device__ __forceinline__ float bf(uint32_t h) { return __uint_as_float(h << 16); }

// Value e of a token's codes (uniform format) at `codes`, its scale byte at `scales`.
__device__ __forceinline__ float value(const uint8_t *codes, const uint8_t *scales, int e, int fmt) {
    const float s = scale_operand(scales[e / 32]);
    if (fmt == KV_FP8)
        return bf(decode8<0>(codes[e], s) & 0xFFFFu);
    return bf(decode4<0>((codes[e / 2] >> (4 * (e & 1))) & 15, s) & 0xFFFFu);
}

// One wavefront per query and head.
__global__ void __launch_bounds__(64)
kv_attention_simple_kernel(KvShape c, KvAttnArgs a) {
    __shared__ float p[64];
    __shared__ int64_t at[64];
    const int lane = threadIdx.x;
    const int q_heads = c.heads * a.group;
    const int64_t t = blockIdx.x / q_heads;
    const int h = (int)(blockIdx.x % q_heads), kvh = h / a.group;
    int b = 0;
    int64_t q0, lq;
    if (a.q_starts) {
        while (b + 1 < a.seqs && a.q_starts[b + 1] <= t)
            ++b;
        q0 = a.q_starts[b];
        lq = a.q_starts[b + 1] - q0;
    } else {
        lq = a.T / a.seqs;
        b = (int)(t / lq);
        q0 = b * lq;
    }
    const int64_t kv = min((int64_t)a.kv_lens[b], (int64_t)a.table_pages * c.page);
    const int64_t n = a.causal ? min(kv, kv - lq + (t - q0) + 1) : kv;
    const uint16_t *q = a.q + t * a.q_token + h * a.q_head;
    float o[4] = {}, top = -INFINITY, sum = 0;
    for (int64_t j0 = 0; j0 < n; j0 += 64) {
        const int64_t j = j0 + lane;
        float s = -INFINITY;
        if (j < n) {
            int64_t page = a.table[b * a.table_stride + j / c.page];
            page = min(max(page, (int64_t)0), c.pages - 1);
            const int64_t base = (page * 2 * c.heads + kvh) * c.head_bytes();
            const int tok = (int)(j % c.page);
            at[lane] = base;
            const uint8_t *kc = a.cache + base + (int64_t)tok * c.code_bytes();
            const uint8_t *ks = a.cache + base + (int64_t)c.page * c.code_bytes() + tok * (c.dim / 32);
            s = 0;
            for (int e = 0; e < c.dim; ++e)
                s = __builtin_fmaf(bf(q[e]), value(kc, ks, e, c.fmt), s);
            s *= a.scale;
        }
        float m = s;
        for (int d = 32; d; d >>= 1)
            m = fmaxf(m, __shfl_xor(m, d));
        m = fmaxf(m, top);
        const float keep = m == -INFINITY ? 1.0f : exp2f(top - m);
        p[lane] = j < n ? exp2f(s - (m == -INFINITY ? 0.0f : m)) : 0.0f;
        float ps = p[lane];
        for (int d = 32; d; d >>= 1)
            ps += __shfl_xor(ps, d);
        sum = sum * keep + ps;
        top = m;
        __syncthreads();
        for (int i = 0; i < 4; ++i) {
            const int e = lane + 64 * i;
            o[i] *= keep;
            if (e >= c.dim)
                break;
            for (int jj = 0; jj < 64 && j0 + jj < n; ++jj) {
                const int64_t base = at[jj] + c.heads * c.head_bytes();
                const int tok = (int)((j0 + jj) % c.page);
                o[i] = __builtin_fmaf(p[jj],
                                      value(a.cache + base + (int64_t)tok * c.code_bytes(),
                                            a.cache + base + (int64_t)c.page * c.code_bytes() +
                                                tok * (c.dim / 32),
                                            e, c.fmt),
                                      o[i]);
            }
        }
        __syncthreads();
    }
    for (int i = 0; i < 4 && lane + 64 * i < c.dim; ++i)
        a.out[(t * q_heads + h) * c.dim + lane + 64 * i] =
            __builtin_bit_cast(uint16_t, (__bf16)(n > 0 ? o[i] / sum : 0.0f));
}

}  // namespace

size_t kv_attention_workspace_bytes(const KvShape &, int64_t, int, int, int, int) { return 0; }

hipError_t launch_kv_attention(const KvShape &c, const KvAttnArgs &a, void *, size_t,
                               hipStream_t s) {
    const int64_t blocks = a.T * c.heads * a.group;
    if (blocks > 0x7FFFFFFF)
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(kv_attention_simple_kernel, dim3((unsigned)blocks), dim3(64), 0, s, c, a);
    return hipGetLastError();
}

}  // namespace w8a8
