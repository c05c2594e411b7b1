// What the attention kernels over the quantized cache share: a sequence's place, the decoding of
// its keys and values, and the running maximum.
#pragma once

#include "../../include/w8a8.h"
#include "mx_internal.hpp"
#include "mx_math.hpp"
#include "quant_math.hpp"

namespace w8a8 {
namespace {

using namespace mx;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// The maximum that exponents are taken from may lag behind by this much: O and l are rescaled
// only when a row's maximum rises further. Weights up to 2^8 instead of 1 lose nothing, as
// float32 sums and bf16 roundings are relative; a rescaling costs as much as a product. 4 x 1000
// queries on 6000 keys, 18 heads of 256: 783 us rescaling at every rise, 670 so.
constexpr float kSlack = 8.0f;
constexpr int kMaxChunk = 4096;

struct Seq {
    int64_t q0;      // first query
    int lq, kv;
};

__device__ __forceinline__ Seq sequence(const KvShape &c, const KvAttnArgs &a, int b) {
    Seq s;
    if (a.q_starts) {      // kept inside the queries whatever the array holds
        s.q0 = min(max((int64_t)a.q_starts[b], (int64_t)0), a.T);
        s.lq = (int)(min((int64_t)a.q_starts[b + 1], a.T) - s.q0);
    } else {
        s.lq = (int)(a.T / a.seqs);
        s.q0 = (int64_t)b * s.lq;
    }
    s.kv = min(a.kv_lens[b], a.table_pages * c.page);
    return s;
}

// What a row of a tree sees: the tokens in front of it, and nodes by its bits.
struct TreeRow {
    const uint32_t *bits;     // nullptr: no row, sees nothing
    int words, prefix, kv;    // the tree's first token (below 0: its first nodes are not cached)
    __device__ __forceinline__ TreeRow(const KvAttnArgs &a, const Seq &s, int qi, bool live)
        : bits(live ? a.tree + (s.q0 + qi) * a.tree_words : nullptr), words(a.tree_words),
          prefix(s.kv - s.lq), kv(s.kv) {}
    __device__ __forceinline__ uint32_t word(int i) const { return i < words ? bits[i] : 0; }
    // Tokens j .. j + 31, the first in the lowest bit.
    __device__ __forceinline__ uint32_t window(int j) const {
        if (!bits || j >= kv)
            return 0;
        const int node = j - prefix;
        uint32_t w;
        if (node <= -32)
            w = ~0u;
        else if (node < 0)
            w = word(0) << -node | ((1u << -node) - 1);
        else
            w = (uint32_t)((word(node / 32) | (uint64_t)word(node / 32 + 1) << 32) >> node % 32);
        return kv - j < 32 ? w & ((1u << (kv - j)) - 1) : w;
    }
    __device__ __forceinline__ bool any() const {
        uint32_t w = bits && prefix > 0;       // else at most as many tokens as nodes
        if (!bits)
            return false;
        for (int j = 0; w == 0 && j < kv; j += 32)
            w = window(j);
        return w != 0;
    }
};

// A row's maximum before its first key: minus infinity where it sees none, else the least finite
// number. A sum of zero then tells a row without keys (zeros) from one all of whose scores are
// minus infinity, as a query with an infinity has them (NaN, as exp(-inf - -inf) is).
__device__ __forceinline__ float start_of(bool sees) { return sees ? -__FLT_MAX__ : -INFINITY; }

__device__ __forceinline__ float inverse(float l, float m) {
    return l == 0.0f ? (m == -INFINITY ? 0.0f : NAN) : 1.0f / l;
}

// In a branch that few tiles take: without it the compiler computes both sides in every tile.
__device__ __forceinline__ void keep_branch() { asm volatile(""); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)lo, (__bf16)hi});
}

// Four neighbouring outputs: v times inv. bf16 tensors may begin at any element.
__device__ __forceinline__ void store_outputs(uint16_t *out, const f32x4 &v, float inv) {
    *reinterpret_cast<Bytes8 *>(out) =
        Bytes8{{pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv)}};
}

// Element E8 (8 values, four words) of a unit's codes.
template <int FMT, int E8>
__device__ __forceinline__ u32x4 decode_part(const u32x4 &codes, float s) {
    if constexpr (FMT == KV_FP8) {
        return u32x4{decode8<0>(codes[2 * E8], s), decode8<1>(codes[2 * E8], s),
                     decode8<0>(codes[2 * E8 + 1], s), decode8<1>(codes[2 * E8 + 1], s)};
    } else {
        return u32x4{decode4<0>(codes[E8], s), decode4<1>(codes[E8], s),
                     decode4<2>(codes[E8], s), decode4<3>(codes[E8], s)};
    }
}

template <int N>
struct Unit;
template <>
struct Unit<16> {
    static __device__ __forceinline__ u32x4 load(const uint8_t *p) {
        return *reinterpret_cast<const u32x4 *>(p);
    }
};
template <>
struct Unit<8> {
    static __device__ __forceinline__ u32x4 load(const uint8_t *p) {
        const u32x2 v = *reinterpret_cast<const u32x2 *>(p);
        return u32x4{v[0], v[1], 0, 0};
    }
};

// Where the tokens of a chunk lie, 16 at a time: the first one's place in its page, and the
// page's keys of the head, from which its codes, scales and values follow.
struct Places {
    int64_t page[kMaxChunk / 16];
    int at[kMaxChunk / 16];
};

// Fills `count` entries from token j_first on; those past token j_end - 1 repeat its block.
__device__ __forceinline__ void fill_places(Places &pl, const KvShape &c, const KvAttnArgs &a,
                                            uint64_t magic, int b, int head, int j_first, int j_end,
                                            int count) {
    const uint32_t last = (uint32_t)(j_end - 1) / 16;
    const int32_t *table = a.table + b * a.table_stride;
    for (int i = threadIdx.x; i < count; i += 256) {
        const uint32_t blk = min((uint32_t)(j_first / 16 + i), last);
        const uint32_t entry = (uint32_t)(blk * magic >> 32);
        const int64_t page = min((int64_t)max(table[entry], 0), c.pages - 1);
        pl.page[i] = (page * 2 * c.heads + head) * c.head_bytes();
        pl.at[i] = (int)(blk - entry * (uint32_t)(c.page / 16)) * 16;
    }
}

// Barrier that orders LDS only: loads from memory stay in flight across it.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The other half's value beside this one's: lanes l and l ^ 32 hold the same row.
__device__ __forceinline__ u32x2 both_halves(float v) {
    return __builtin_bit_cast(
        u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
}

}  // namespace
}  // namespace w8a8
