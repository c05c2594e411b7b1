// Internal declarations of the microscaled operators: the 4-bit quantizer and product, the
// quantized key/value cache and the attention over it.
#pragma once

#include "w8a8_internal.hpp"

namespace w8a8 {

// A dimension of a grid holds fewer than 2^32 threads. With more the launch reports nothing and
// runs the remainder of 2^32, so every grid whose size follows from a call's is checked first.
constexpr bool launchable(int64_t blocks, int threads) {
    return blocks <= (int64_t)UINT32_MAX / threads;
}

// ---------------------------------------------------------------- matrices
hipError_t launch_mx4_quant(const uint16_t *x, int64_t R, int64_t K, int act,
                            const float *col_mul, uint8_t *codes, uint8_t *scales,
                            hipStream_t s);
hipError_t launch_mx4_dequant(const uint8_t *codes, const uint8_t *scales, int64_t R, int64_t K,
                              uint16_t *y, hipStream_t s);

struct Mx4Args {
    const uint8_t *xq, *xs;   // [M, 16 nb] codes, [ceil(nb/8), M, 8] scales; nb = ceil(K/32)
    const uint8_t *wq, *ws;   // the same with N rows
    const uint16_t *bias;     // [N] or nullptr
    uint16_t *y;              // [M, N] bf16
    int64_t M, N, nb;
};

size_t mx4_gemm_workspace_bytes(int64_t M, int64_t N, int64_t nb);
hipError_t launch_mx4_gemm(const Mx4Args &a, void *ws, hipStream_t s);

// Whether the linear runs as one launch, which quantizes the tokens as it multiplies (a.xq and
// a.xs unused then).
bool mx4_linear_one_launch(int64_t M, int64_t N, int64_t K);
hipError_t launch_mx4_linear(const Mx4Args &a, const uint16_t *x, int64_t K, int act,
                             const float *col_mul, hipStream_t s);

// ---------------------------------------------------------------- cache
enum KvFormat : int { KV_FP8 = 0, KV_FP4 = 1 };

// A cache [pages][2][heads][page bytes]: per page, keys and values, and head the codes of its
// tokens, then their scales.
struct KvShape {
    int64_t pages;
    int page, heads, dim, fmt;
    __host__ __device__ int code_bytes() const { return fmt == KV_FP8 ? dim : dim / 2; }    // of one token and head
    __host__ __device__ int64_t head_bytes() const { return (int64_t)page * (code_bytes() + dim / 32); }
};

struct KvRows {          // [T, heads, dim] bf16, strides in elements, dim contiguous
    uint16_t *p;
    int64_t token, head;
};

hipError_t launch_kv_write(uint8_t *cache, const KvShape &c, const KvRows &k, const KvRows &v,
                           const int64_t *slots, int64_t T, hipStream_t s);
hipError_t launch_kv_read(const uint8_t *cache, const KvShape &c, const KvRows &k,
                          const KvRows &v, const int64_t *slots, int64_t T, hipStream_t s);

struct KvAttnArgs {
    const uint16_t *q;            // [T, heads * group, dim], strides in elements
    int64_t q_token, q_head;
    const uint8_t *cache;
    const int32_t *table;         // [seqs, table_pages], rows table_stride apart
    int64_t table_stride;
    const int32_t *kv_lens;       // [seqs]
    const int32_t *q_starts;      // [seqs + 1] or nullptr: T / seqs queries each
    uint16_t *out;                // [T, heads * group, dim] contiguous
    int64_t T;
    int seqs, group, table_pages, causal;
    int max_q, max_kv;            // what the grid is laid out for; the results don't depend on them
    float scale;                  // of the scores, times log2(e); above 0
    uint32_t q_sign;              // 0x80008000: the scale's sign, taken into q; else 0
    const uint32_t *tree;         // [T, tree_words] or nullptr: which of a sequence's last lq tokens
    int tree_words;               // a query sees, a bit each (causal is not read then)
};

size_t kv_attention_workspace_bytes(const KvShape &c, int64_t T, int seqs, int group, int max_q,
                                    int max_kv);
hipError_t launch_kv_attention(const KvShape &c, const KvAttnArgs &a, void *ws, hipStream_t s);

size_t kv_tree_workspace_bytes(const KvShape &c, int64_t T, int seqs, int group, int max_q,
                               int max_kv);
hipError_t launch_kv_tree(const KvShape &c, const KvAttnArgs &a, void *ws, hipStream_t s);

}  // namespace w8a8
