// C ABI of the microscaled operators: argument validation and launches on the caller's
// stream. Nothing here allocates, frees or synchronizes.
#include "../../include/w8a8.h"
#include "mx_internal.hpp"

namespace {

using namespace w8a8;

constexpr int64_t kMaxElems = int64_t(1) << 62;
constexpr size_t kAlign = 256;

size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
bool product_ok(int64_t a, int64_t b) { return a == 0 || b <= kMaxElems / a; }
hipStream_t as_stream(void *s) { return reinterpret_cast<hipStream_t>(s); }
w8a8_status from_hip(hipError_t e) { return e == hipSuccess ? W8A8_OK : W8A8_ERR_HIP; }
bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

static_assert(W8A8_KV_FP8 == KV_FP8 && W8A8_KV_FP4 == KV_FP4, "cache formats");

w8a8_status check_matrix(int64_t R, int64_t K) {
    if (R < 0 || K < 0 || !product_ok(R, K))
        return W8A8_ERR_SHAPE;
    return K > W8A8_MX4_MAX_K ? W8A8_ERR_K_OVERFLOW : W8A8_OK;
}

int64_t blocks_of(int64_t K) { return (K + 31) / 32; }
size_t code_bytes(int64_t R, int64_t K) { return (size_t)(R * blocks_of(K) * 16); }
size_t scale_bytes(int64_t R, int64_t K) { return (size_t)((K + 255) / 256 * R * 8); }

w8a8_status check_product(int64_t M, int64_t N, int64_t K) {
    if (M < 0 || N < 0 || K < 0 || !product_ok(M, K) || !product_ok(N, K) || !product_ok(M, N))
        return W8A8_ERR_SHAPE;
    return K > W8A8_MX4_MAX_K ? W8A8_ERR_K_OVERFLOW : W8A8_OK;
}

Mx4Args product(const uint8_t *xq, const uint8_t *xs, const uint8_t *wq, const uint8_t *ws,
                const uint16_t *bias, uint16_t *y, int64_t M, int64_t N, int64_t K) {
    Mx4Args a;
    a.xq = xq;
    a.xs = xs;
    a.wq = wq;
    a.ws = ws;
    a.bias = bias;
    a.y = y;
    a.M = M;
    a.N = N;
    a.nb = blocks_of(K);
    return a;
}

bool cache_shape(KvShape &c, int64_t pages, int page, int heads, int dim, int fmt) {
    if ((fmt != W8A8_KV_FP8 && fmt != W8A8_KV_FP4) || page < 16 || page % 16 != 0 ||
        page > W8A8_KV_MAX_PAGE || heads < 1 || heads > W8A8_KV_MAX_HEADS || dim < 64 ||
        dim > 256 || dim % 64 != 0 || pages < 0)
        return false;
    c = {pages, page, heads, dim, fmt};
    return product_ok(pages, 2 * heads * c.head_bytes());
}

w8a8_status check_rows(const KvShape &c, const void *k, const void *v, const int64_t *slots,
                       int64_t T) {
    if (T < 0 || !product_ok(T, 2 * (int64_t)c.heads * c.dim))
        return W8A8_ERR_SHAPE;
    return T > 0 && (!k || !v || !slots) ? W8A8_ERR_NULL : W8A8_OK;
}

// The bound on a sequence's queries that a launch is laid out for: a loose one, so never 0.
int query_bound(int max_q) { return max_q > 1 ? max_q : 1; }

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

w8a8_status w8a8_mx4_quantize(const uint16_t *x, int64_t R, int64_t K, int act,
                              const float *col_mul, uint8_t *codes, uint8_t *scales,
                              void *stream) {
    if (act != W8A8_ACT_NONE && act != W8A8_ACT_GELU)
        return W8A8_ERR_ARG;
    const w8a8_status st = check_matrix(R, K);
    if (st != W8A8_OK || R == 0 || K == 0)
        return st;
    if (!x || !codes || !scales)
        return W8A8_ERR_NULL;
    if (!aligned(codes, 16) || !aligned(scales, 16))
        return W8A8_ERR_ARG;
    return from_hip(launch_mx4_quant(x, R, K, act, col_mul, codes, scales, as_stream(stream)));
}

w8a8_status w8a8_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t R,
                                int64_t K, uint16_t *y, void *stream) {
    const w8a8_status st = check_matrix(R, K);
    if (st != W8A8_OK || R == 0 || K == 0)
        return st;
    if (!y || !codes || !scales)
        return W8A8_ERR_NULL;
    if (!aligned(codes, 16) || !aligned(scales, 16))
        return W8A8_ERR_ARG;
    return from_hip(launch_mx4_dequant(codes, scales, R, K, y, as_stream(stream)));
}

size_t w8a8_mx4_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (check_product(M, N, K) != W8A8_OK || M == 0 || N == 0)
        return 0;
    return mx4_gemm_workspace_bytes(M, N, blocks_of(K));
}

w8a8_status w8a8_mx4_gemm(const uint8_t *xq, const uint8_t *x_scale, const uint8_t *wq,
                          const uint8_t *w_scale, const uint16_t *bias, uint16_t *y, int64_t M,
                          int64_t N, int64_t K, void *workspace, size_t workspace_bytes,
                          void *stream) {
    const w8a8_status st = check_product(M, N, K);
    if (st != W8A8_OK || M == 0 || N == 0)
        return st;
    if (!y || (K > 0 && (!xq || !x_scale || !wq || !w_scale)))
        return W8A8_ERR_NULL;
    if (!aligned(xq, 16) || !aligned(x_scale, 16) || !aligned(wq, 16) || !aligned(w_scale, 16))
        return W8A8_ERR_ARG;
    const size_t need = w8a8_mx4_gemm_workspace_bytes(M, N, K);
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, kAlign)))
        return W8A8_ERR_WORKSPACE;
    return from_hip(launch_mx4_gemm(product(xq, x_scale, wq, w_scale, bias, y, M, N, K), workspace,
                                    as_stream(stream)));
}

size_t w8a8_mx4_linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    if (check_product(M, N, K) != W8A8_OK || M == 0 || N == 0 || mx4_linear_one_launch(M, N, K))
        return 0;
    return align_up(code_bytes(M, K)) + align_up(scale_bytes(M, K)) +
           mx4_gemm_workspace_bytes(M, N, blocks_of(K));
}

w8a8_status w8a8_mx4_linear(const uint16_t *x, int act, const float *col_mul, const uint8_t *wq,
                            const uint8_t *w_scale, const uint16_t *bias, uint16_t *y, int64_t M,
                            int64_t N, int64_t K, void *workspace, size_t workspace_bytes,
                            void *stream) {
    if (act != W8A8_ACT_NONE && act != W8A8_ACT_GELU)
        return W8A8_ERR_ARG;
    const w8a8_status st = check_product(M, N, K);
    if (st != W8A8_OK || M == 0 || N == 0)
        return st;
    if (!y || (K > 0 && (!x || !wq || !w_scale)))
        return W8A8_ERR_NULL;
    if (!aligned(wq, 16) || !aligned(w_scale, 16))
        return W8A8_ERR_ARG;
    const size_t need = w8a8_mx4_linear_workspace_bytes(M, N, K);
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, kAlign)))
        return W8A8_ERR_WORKSPACE;
    if (mx4_linear_one_launch(M, N, K))
        return from_hip(launch_mx4_linear(product(nullptr, nullptr, wq, w_scale, bias, y, M, N, K), x, K,
                                          act, col_mul, as_stream(stream)));
    uint8_t *xq = static_cast<uint8_t *>(workspace);
    uint8_t *xs = xq + align_up(code_bytes(M, K));
    uint8_t *rest = xs + align_up(scale_bytes(M, K));
    if (launch_mx4_quant(x, M, K, act, col_mul, xq, xs, as_stream(stream)) != hipSuccess)
        return W8A8_ERR_HIP;
    return from_hip(launch_mx4_gemm(product(xq, xs, wq, w_scale, bias, y, M, N, K), rest,
                                    as_stream(stream)));
}

int64_t w8a8_kv_page_bytes(int page, int heads, int dim, int fmt) {
    KvShape c;
    return cache_shape(c, 1, page, heads, dim, fmt) ? 2 * heads * c.head_bytes() : -1;
}

w8a8_status w8a8_kv_write(uint8_t *cache, int64_t pages, int page, int heads, int dim, int fmt,
                          const uint16_t *k, int64_t k_token, int64_t k_head, const uint16_t *v,
                          int64_t v_token, int64_t v_head, const int64_t *slots, int64_t T,
                          void *stream) {
    KvShape c;
    if (!cache_shape(c, pages, page, heads, dim, fmt))
        return W8A8_ERR_ARG;
    const w8a8_status st = check_rows(c, k, v, slots, T);
    if (st != W8A8_OK || T == 0 || pages == 0)
        return st;
    if (!cache)
        return W8A8_ERR_NULL;
    if (!aligned(cache, 16) || k_token < 0 || k_head < 0 || v_token < 0 || v_head < 0)
        return W8A8_ERR_ARG;
    return from_hip(launch_kv_write(cache, c, {const_cast<uint16_t *>(k), k_token, k_head},
                                    {const_cast<uint16_t *>(v), v_token, v_head}, slots, T,
                                    as_stream(stream)));
}

w8a8_status w8a8_kv_read(const uint8_t *cache, int64_t pages, int page, int heads, int dim,
                         int fmt, const int64_t *slots, int64_t T, uint16_t *k, uint16_t *v,
                         void *stream) {
    KvShape c;
    if (!cache_shape(c, pages, page, heads, dim, fmt))
        return W8A8_ERR_ARG;
    const w8a8_status st = check_rows(c, k, v, slots, T);
    if (st != W8A8_OK || T == 0)
        return st;
    if (!cache && pages > 0)
        return W8A8_ERR_NULL;
    if (!aligned(cache, 16))
        return W8A8_ERR_ARG;
    const int64_t token = (int64_t)heads * dim;
    return from_hip(launch_kv_read(cache, c, {k, token, dim}, {v, token, dim}, slots, T,
                                   as_stream(stream)));
}

size_t w8a8_kv_attention_workspace_bytes(int page, int heads, int dim, int fmt, int group,
                                         int64_t T, int seqs, int max_q, int max_kv) {
    KvShape c;
    if (!cache_shape(c, 1, page, heads, dim, fmt) || group < 1 || T < 1 || seqs < 1 ||
        max_q < 0 || max_kv < 0)
        return 0;
    return kv_attention_workspace_bytes(c, T, seqs, group, query_bound(max_q), max_kv);
}

w8a8_status w8a8_kv_attention(const uint16_t *q, int64_t q_token, int64_t q_head,
                              const uint8_t *cache, int64_t pages, int page, int heads, int dim,
                              int fmt, const int32_t *table, int64_t table_stride,
                              int table_pages, const int32_t *kv_lens, const int32_t *q_starts,
                              int64_t T, int seqs, int group, float scale, int causal, int max_q,
                              int max_kv, uint16_t *out, void *workspace, size_t workspace_bytes,
                              void *stream) {
    KvShape c;
    if (!cache_shape(c, pages, page, heads, dim, fmt) || group < 1 ||
        group > W8A8_KV_MAX_HEADS || (causal != 0 && causal != 1) || !__builtin_isfinite(scale))
        return W8A8_ERR_ARG;
    if (T < 0 || seqs < 0 || table_pages < 0 || table_stride < 0 || q_token < 0 || q_head < 0 ||
        max_q < 0 || max_kv < 0 || !product_ok(T, (int64_t)heads * group * dim) ||
        (int64_t)table_pages * page > W8A8_KV_MAX_TOKENS)
        return W8A8_ERR_SHAPE;
    if (T == 0 || seqs == 0)
        return T == 0 ? W8A8_OK : W8A8_ERR_SHAPE;
    if (!q_starts && T % seqs != 0)
        return W8A8_ERR_SHAPE;
    if (!q || !out || !kv_lens || (table_pages > 0 && pages > 0 && (!cache || !table)))
        return W8A8_ERR_NULL;
    if (!aligned(cache, 16))
        return W8A8_ERR_ARG;
    KvAttnArgs a;
    a.q = q;
    a.q_token = q_token;
    a.q_head = q_head;
    a.cache = cache;
    a.table = table;
    a.table_stride = table_stride;
    a.kv_lens = kv_lens;
    a.q_starts = q_starts;
    a.out = out;
    a.T = T;
    a.seqs = seqs;
    a.group = group;
    a.table_pages = pages > 0 ? table_pages : 0;
    a.causal = causal;
    a.max_q = query_bound(max_q);
    a.max_kv = max_kv;
    // The kernels scale a maximum instead of every score, and mask with minus infinity: a
    // positive factor. A zero becomes so small a one that all weights are 1.
    a.q_sign = scale < 0.0f ? 0x80008000u : 0u;
    a.scale = __builtin_fabsf(scale) * 1.44269504088896341f;
    if (a.scale < 0x1p-126f)
        a.scale = 0x1p-126f;
    const size_t need = kv_attention_workspace_bytes(c, T, seqs, group, a.max_q, max_kv);
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, kAlign)))
        return W8A8_ERR_WORKSPACE;
    return from_hip(launch_kv_attention(c, a, workspace, as_stream(stream)));
}

}  // extern "C"
#pragma GCC visibility pop
