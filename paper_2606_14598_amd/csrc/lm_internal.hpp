// Internal declarations of the operators around a decoding step's linears and attention: the
// norm that quantizes for the next linear, and the log probabilities of its tokens.
#pragma once

#include "mx_internal.hpp"

namespace w8a8 {

enum NormFormat : int { NORM_INT8 = 0, NORM_MX4 = 1 };

struct NormArgs {
    const uint16_t *x, *residual;   // [R, K] bf16; residual may be nullptr
    uint16_t *sum;                  // [R, K] bf16, with a residual: x + residual
    const float *weight;            // [K] or nullptr
    int64_t R, K;
    double eps;
    uint8_t *codes;                 // int8 [R, K], or 4-bit codes
    float *scale;                   // [R] (NORM_INT8)
    uint8_t *scales;                // of 4-bit blocks (NORM_MX4)
};

hipError_t launch_norm_quant(const NormArgs &a, int fmt, hipStream_t s);

// ---------------------------------------------------------------- cache
constexpr int kMaxAxes = 4;

struct AppendArgs {
    KvRows q, k, v;                 // q: q_heads heads, k and v the cache's
    uint16_t *q_out;                // [T, q_heads, dim] contiguous
    int q_heads;
    const int64_t *slots;           // [T]
    const int64_t *positions;       // [T, axes]
    const float *inv_freq;          // [pairs]
    int axes, pairs, interleaved;
    int section_end[kMaxAxes];      // axis n has the pairs section_end[n - 1] .. section_end[n] - 1
    int64_t T;
};

hipError_t launch_kv_append(uint8_t *cache, const KvShape &c, const AppendArgs &a, hipStream_t s);

// ---------------------------------------------------------------- log probabilities
struct LogprobArgs {
    const void *logits;             // [T, V] bf16 or float32, rows row_stride elements apart
    int64_t row_stride, T, V;
    int f32;                        // logits are float32
    const int64_t *tokens;          // [T]
    int top;
    float factor;                   // log2(e) / temperature
    float *logp, *entropy;          // [T]
    float *top_logp;                // [T, top]
    int64_t *top_ids;               // [T, top]
};

size_t logprobs_workspace_bytes(int64_t T, int64_t V, int top);
hipError_t launch_logprobs(const LogprobArgs &a, void *ws, hipStream_t s);

}  // namespace w8a8
