// C ABI of the operators around a decoding step's linears: argument validation and launches on
// the caller's stream. Nothing here allocates, frees or synchronizes.
#include "../../include/w8a8.h"
#include "lm_internal.hpp"

namespace {

using namespace w8a8;

constexpr int64_t kMaxElems = int64_t(1) << 62;

bool product_ok(int64_t a, int64_t b) { return a == 0 || b <= kMaxElems / a; }
hipStream_t as_stream(void *s) { return reinterpret_cast<hipStream_t>(s); }
w8a8_status from_hip(hipError_t e) { return e == hipSuccess ? W8A8_OK : W8A8_ERR_HIP; }
bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Two ranges of n bytes that share some but not all.
bool partly_same(const void *p, const void *q, int64_t n) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return a != b && (a > b ? a - b : b - a) < (uintptr_t)n;
}

w8a8_status norm(int fmt, const uint16_t *x, const uint16_t *residual, uint16_t *sum,
                 const float *weight, double eps, int64_t R, int64_t K, uint8_t *codes, float *scale,
                 uint8_t *scales, void *stream) {
    if (R < 0 || K < 0 || !product_ok(R, K))
        return W8A8_ERR_SHAPE;
    if (K > (fmt == NORM_INT8 ? W8A8_MAX_K : W8A8_MX4_MAX_K))
        return W8A8_ERR_K_OVERFLOW;
    if (!(eps >= 0x1p-126) || !__builtin_isfinite(eps))       // below: 1 / sqrt(eps) may be no float32
        return W8A8_ERR_ARG;
    if (R == 0 || (K == 0 && fmt == NORM_MX4))
        return W8A8_OK;
    if ((fmt == NORM_INT8 && !scale) || (K > 0 && (!x || !codes || (residual && !sum))) ||
        (fmt == NORM_MX4 && !scales))
        return W8A8_ERR_NULL;
    if (fmt == NORM_MX4 && (!aligned(codes, 16) || !aligned(scales, 16)))
        return W8A8_ERR_ARG;
    if (residual && (partly_same(sum, x, 2 * R * K) || partly_same(sum, residual, 2 * R * K)))
        return W8A8_ERR_ARG;
    NormArgs a;
    a.x = x;
    a.residual = residual;
    a.sum = sum;
    a.weight = weight;
    a.R = R;
    a.K = K;
    a.eps = eps;
    a.codes = codes;
    a.scale = scale;
    a.scales = scales;
    return from_hip(launch_norm_quant(a, fmt, as_stream(stream)));
}

bool logprobs_ok(int64_t T, int64_t V, int top) {
    return T >= 0 && V >= 1 && V <= W8A8_LOGPROBS_MAX_V && T <= kMaxElems / V && top >= 0 &&
           top <= W8A8_LOGPROBS_MAX_TOP && top <= V;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

w8a8_status w8a8_rms_norm_quantize(const uint16_t *x, const uint16_t *residual, uint16_t *sum,
                                   const float *weight, double eps, int64_t M, int64_t K, int8_t *xq,
                                   float *x_scale, void *stream) {
    return norm(NORM_INT8, x, residual, sum, weight, eps, M, K, reinterpret_cast<uint8_t *>(xq),
                x_scale, nullptr, stream);
}

w8a8_status w8a8_rms_norm_mx4_quantize(const uint16_t *x, const uint16_t *residual, uint16_t *sum,
                                       const float *weight, double eps, int64_t M, int64_t K,
                                       uint8_t *codes, uint8_t *scales, void *stream) {
    return norm(NORM_MX4, x, residual, sum, weight, eps, M, K, codes, nullptr, scales, stream);
}

size_t w8a8_token_logprobs_workspace_bytes(int64_t T, int64_t V, int top) {
    return logprobs_ok(T, V, top) && T > 0 ? logprobs_workspace_bytes(T, V, top) : 0;
}

w8a8_status w8a8_token_logprobs(const void *logits, int f32, int64_t row_stride, int64_t T, int64_t V,
                                const int64_t *tokens, int top, float temperature, float *logp,
                                float *entropy, float *top_logp, int64_t *top_ids, void *workspace,
                                size_t workspace_bytes, void *stream) {
    if ((f32 != 0 && f32 != 1) || top < 0 || top > W8A8_LOGPROBS_MAX_TOP || !(temperature > 0.0f) ||
        !__builtin_isfinite(temperature) || !__builtin_isnormal(1.44269504f / temperature))
        return W8A8_ERR_ARG;
    if (!logprobs_ok(T, V, top) || row_stride < 0 || !product_ok(T, row_stride))
        return W8A8_ERR_SHAPE;
    if (T == 0)
        return W8A8_OK;
    if (!logits || !tokens || !logp || !entropy || (top > 0 && (!top_logp || !top_ids)))
        return W8A8_ERR_NULL;
    const size_t need = logprobs_workspace_bytes(T, V, top);
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 256)))
        return W8A8_ERR_WORKSPACE;
    LogprobArgs a;
    a.logits = logits;
    a.row_stride = row_stride;
    a.T = T;
    a.V = V;
    a.f32 = f32;
    a.tokens = tokens;
    a.top = top;
    a.factor = 1.44269504088896341f / temperature;
    a.logp = logp;
    a.entropy = entropy;
    a.top_logp = top_logp;
    a.top_ids = top_ids;
    return from_hip(launch_logprobs(a, workspace, as_stream(stream)));
}

}  // extern "C"
#pragma GCC visibility pop
