// Where a token's keys and values lie in the quantized cache.
#pragma once

#include "mx_internal.hpp"
#include "mx_math.hpp"

namespace w8a8 {
namespace {

struct Token {
    int64_t t;                 // of the call; past its tokens: nothing to do
    int64_t keys;              // its page in the cache; below 0 for padding
    int at;                    // its place in the page
};

// Token t (the same in all lanes) of the T of a call.
__device__ __forceinline__ Token token_of(const KvShape &c, const int64_t *slots, int64_t t, int64_t T) {
    Token k;
    k.t = t;
    k.keys = -1;
    k.at = 0;
    if (k.t >= T)
        return k;
    const int64_t slot = slots[k.t];
    if (slot < 0 || slot >= c.pages * c.page)
        return k;
    const int64_t page = slot >> 31 ? slot / c.page : (uint32_t)slot / (uint32_t)c.page;
    k.at = (int)(slot - page * c.page);
    k.keys = page * 2 * c.heads * c.head_bytes();
    return k;
}

// Unit u of a token: 8 values of keys or values; heads * 2 * D / 8 of them.
template <int FMT, int D>
struct Unit8 {
    static constexpr int CB = FMT == KV_FP8 ? D : D / 2;
    int head, e;               // head over keys, then values; first of the 8 values
    int64_t codes, scale;      // in the cache
    __device__ __forceinline__ Unit8(const KvShape &c, const Token &k, int u) {
        head = u / (D / 8);
        e = u % (D / 8) * 8;
        const int64_t base = k.keys + head * c.head_bytes();
        codes = base + k.at * CB + (FMT == KV_FP8 ? e : e / 2);
        scale = base + c.page * CB + k.at * (D / 32) + e / 32;
    }
};

}  // namespace
}  // namespace w8a8
