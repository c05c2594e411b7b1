// Quantizing a key/value cache as it is written, and reading it back.
//
// A token's key (or value) of one head is head_dim values in blocks of 32 (mx_math.hpp). The
// cache keeps, for each page, keys then values, and each head, the codes of the page's tokens
// one after the other and behind them their scale bytes, so that a head's keys of a page are
// one piece of memory. Slot s is token s % page of page s / page; a slot below 0 or past the
// cache is padding: not written, and read as zeros.
//
// Four lanes hold a block, 8 values each; bound by memory: 20000 tokens of 8 heads of 128 are
// written in 4 bits in 19 us (5.4 TB/s read and written) and read back in 19.
#include "mx_internal.hpp"
#include "mx_math.hpp"

namespace w8a8 {
namespace {

using namespace mx;

// A wavefront takes one token and up to 64 * kLoads of its units of 8 values, keys then values;
// where the token lies in the cache is then the same for all lanes, and the divisions that it
// takes are done once.
constexpr int kLoads = 4;

struct Token {
    int64_t t;                 // of the call; past its tokens: nothing to do
    int64_t keys;              // its page in the cache; below 0 for padding
    int at;                    // its place in the page
};

__device__ __forceinline__ Token token_of(const KvShape &c, const int64_t *slots, int64_t T) {
    Token k;
    k.t = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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

template <int FMT, int D>
__global__ void __launch_bounds__(256)
kv_write_kernel(uint8_t *cache, KvShape c, KvRows k, KvRows v, const int64_t *slots, int64_t T) {
    const Token tok = token_of(c, slots, T);
    if (tok.keys < 0)
        return;
    const int units = 2 * c.heads * (D / 8), u0 = blockIdx.y * (64 * kLoads) + (threadIdx.x & 63);
    Bytes16 in[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int u = min(u0 + 64 * i, units - 1), head = u / (D / 8), e = u % (D / 8) * 8;
        const uint16_t *src = head < c.heads ? k.p + tok.t * k.token + head * k.head
                                             : v.p + tok.t * v.token + (head - c.heads) * v.head;
        in[i] = *reinterpret_cast<const Bytes16 *>(src + e);
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int u = u0 + 64 * i;
        if (u >= units)        // units is a multiple of the four lanes of a block
            return;
        const Unit8<FMT, D> unit(c, tok, u);
        const uint32_t w[4] = {in[i].w[0], in[i].w[1], in[i].w[2], in[i].w[3]};
        uint32_t m = max_halves(max_halves(magnitudes(w[0]), magnitudes(w[1])),
                                max_halves(magnitudes(w[2]), magnitudes(w[3])));
        m = quad_max(max(m & 0xFFFFu, m >> 16));
        const uint32_t byte = scale_byte<FMT == KV_FP8 ? kTop8 : kTop4>(m >> 7);
        const bool bad = byte == kNaNScale;
        const float s = scale_operand(byte);
        if constexpr (FMT == KV_FP8) {
            uint2 q = make_uint2(encode8_bf16(w[0], w[1], m >> 7, s), encode8_bf16(w[2], w[3], m >> 7, s));
            if (bad)
                q = make_uint2(0, 0);
            *reinterpret_cast<uint2 *>(cache + unit.codes) = q;
        } else {
            *reinterpret_cast<uint32_t *>(cache + unit.codes) = bad ? 0 : encode4_bf16(w, s);
        }
        if (unit.e % 32 == 0)
            cache[unit.scale] = (uint8_t)byte;
    }
}

template <int FMT, int D>
__global__ void __launch_bounds__(256)
kv_read_kernel(const uint8_t *cache, KvShape c, KvRows k, KvRows v, const int64_t *slots, int64_t T) {
    const Token tok = token_of(c, slots, T);
    if (tok.t >= T)
        return;
    const int units = 2 * c.heads * (D / 8), u0 = blockIdx.y * (64 * kLoads) + (threadIdx.x & 63);
    uint2 codes[kLoads];
    uint32_t byte[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        codes[i] = make_uint2(0, 0);
        byte[i] = 0;
        if (tok.keys >= 0) {
            const Unit8<FMT, D> unit(c, tok, min(u0 + 64 * i, units - 1));
            byte[i] = cache[unit.scale];
            if constexpr (FMT == KV_FP8)
                codes[i] = *reinterpret_cast<const uint2 *>(cache + unit.codes);
            else
                codes[i].x = *reinterpret_cast<const uint32_t *>(cache + unit.codes);
        }
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int u = u0 + 64 * i, head = u / (D / 8), e = u % (D / 8) * 8;
        if (u >= units)
            return;
        const float s = scale_operand(byte[i]);
        Bytes16 out;
        if constexpr (FMT == KV_FP8) {
            out.w[0] = decode8<0>(codes[i].x, s);
            out.w[1] = decode8<1>(codes[i].x, s);
            out.w[2] = decode8<0>(codes[i].y, s);
            out.w[3] = decode8<1>(codes[i].y, s);
        } else {
            out.w[0] = decode4<0>(codes[i].x, s);
            out.w[1] = decode4<1>(codes[i].x, s);
            out.w[2] = decode4<2>(codes[i].x, s);
            out.w[3] = decode4<3>(codes[i].x, s);
        }
        uint16_t *dst = head < c.heads ? k.p + tok.t * k.token + head * k.head
                                       : v.p + tok.t * v.token + (head - c.heads) * v.head;
        *reinterpret_cast<Bytes16 *>(dst + e) = out;
    }
}

// Calls go(kernel format, head_dim, grid, first token, tokens), the first two as compile-time
// constants, for up to kTokens of the T tokens at a time: four make a workgroup of 256 threads.
constexpr int64_t kTokens = 1 << 25;
static_assert(launchable(kTokens / 4, 256));

template <typename F>
hipError_t by_shape(const KvShape &c, int64_t T, F go) {
    const int64_t pieces = (2 * c.heads * (c.dim / 8) + 64 * kLoads - 1) / (64 * kLoads);
    const auto run = [&](auto fmt, auto dim) {
        for (int64_t t0 = 0; t0 < T; t0 += kTokens) {
            const int64_t n = T - t0 < kTokens ? T - t0 : kTokens;
            go(fmt, dim, dim3((unsigned)((n + 3) / 4), (unsigned)pieces), t0, n);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess)
                return e;
        }
        return hipSuccess;
    };
    const auto with_dim = [&](auto dim) {
        return c.fmt == KV_FP8 ? run(std::integral_constant<int, KV_FP8>{}, dim)
                               : run(std::integral_constant<int, KV_FP4>{}, dim);
    };
    switch (c.dim) {
    case 64: return with_dim(std::integral_constant<int, 64>{});
    case 128: return with_dim(std::integral_constant<int, 128>{});
    case 192: return with_dim(std::integral_constant<int, 192>{});
    default: return with_dim(std::integral_constant<int, 256>{});
    }
}

KvRows rows_from(const KvRows &r, int64_t t0) { return {r.p + t0 * r.token, r.token, r.head}; }

}  // namespace

hipError_t launch_kv_write(uint8_t *cache, const KvShape &c, const KvRows &k, const KvRows &v,
                           const int64_t *slots, int64_t T, hipStream_t s) {
    return by_shape(c, T, [&](auto fmt, auto dim, dim3 grid, int64_t t0, int64_t n) {
        hipLaunchKernelGGL((kv_write_kernel<decltype(fmt)::value, decltype(dim)::value>), grid, dim3(256), 0,
                           s, cache, c, rows_from(k, t0), rows_from(v, t0), slots + t0, n);
    });
}

hipError_t launch_kv_read(const uint8_t *cache, const KvShape &c, const KvRows &k,
                          const KvRows &v, const int64_t *slots, int64_t T, hipStream_t s) {
    return by_shape(c, T, [&](auto fmt, auto dim, dim3 grid, int64_t t0, int64_t n) {
        hipLaunchKernelGGL((kv_read_kernel<decltype(fmt)::value, decltype(dim)::value>), grid, dim3(256), 0,
                           s, cache, c, rows_from(k, t0), rows_from(v, t0), slots + t0, n);
    });
}

}  // namespace w8a8
