// Quantizing a key/value cache as it is written, and reading it back.
//
// A token's key (or value) of one head is head_dim values in blocks of 32 (mx_math.hpp). The
// cache keeps, for each page, keys then values, and each head, the codes of the page's tokens
// one after the other and behind them their scale bytes, so that a head's keys of a page are
// one piece of memory. Slot s is token s % page of page s / page; a slot below 0 or past the
// cache is padding: not written, and read as zeros.
//
// Four lanes hold a block, 8 values each; bound by memory.
#include "mx_internal.hpp"
#include "mx_math.hpp"

namespace w8a8 {
namespace {

using namespace mx;

struct Place {
    int64_t t;        // token of the call
    int kv, head, e;  // keys or values, head, first of the lane's 8 elements
    int64_t codes, scales;   // of the token's element 0 in the cache; codes < 0: padding
};

// Lane index g over [T][2][heads][dim / 8].
__device__ __forceinline__ Place place(int64_t g, const KvShape &c, const int64_t *slots) {
    Place p;
    const int per = c.dim / 8;
    p.e = (int)(g % per) * 8;
    const int64_t h = g / per;
    p.head = (int)(h % c.heads);
    p.kv = (int)(h / c.heads % 2);
    p.t = h / c.heads / 2;
    const int64_t slot = slots[p.t];
    if (slot < 0 || slot >= c.pages * c.page) {
        p.codes = p.scales = -1;
        return p;
    }
    const int64_t base = ((slot / c.page * 2 + p.kv) * c.heads + p.head) * c.head_bytes();
    const int at = (int)(slot % c.page);
    p.codes = base + (int64_t)at * c.code_bytes();
    p.scales = base + (int64_t)c.page * c.code_bytes() + at * (c.dim / 32);
    return p;
}

template <int FMT>
__global__ void __launch_bounds__(256)
kv_write_kernel(uint8_t *cache, KvShape c, KvRows k, KvRows v, const int64_t *slots, int64_t n) {
    const int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (g >= n)          // n is a multiple of the four lanes of a block
        return;
    const Place p = place(g, c, slots);
    if (p.codes < 0)
        return;
    const KvRows &src = p.kv ? v : k;
    const Bytes16 in =
        *reinterpret_cast<const Bytes16 *>(src.p + p.t * src.token + p.head * src.head + p.e);
    const uint32_t w[4] = {in.w[0], in.w[1], in.w[2], in.w[3]};
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
        *reinterpret_cast<uint2 *>(cache + p.codes + p.e) = q;
    } else {
        *reinterpret_cast<uint32_t *>(cache + p.codes + p.e / 2) = bad ? 0 : encode4_bf16(w, s);
    }
    if (p.e % 32 == 0)
        cache[p.scales + p.e / 32] = (uint8_t)byte;
}

template <int FMT>
__global__ void __launch_bounds__(256)
kv_read_kernel(const uint8_t *cache, KvShape c, KvRows k, KvRows v, const int64_t *slots,
               int64_t n) {
    const int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (g >= n)
        return;
    const Place p = place(g, c, slots);
    Bytes16 out = {};
    if (p.codes >= 0) {
        const float s = scale_operand(cache[p.scales + p.e / 32]);
        if constexpr (FMT == KV_FP8) {
            const uint2 q = *reinterpret_cast<const uint2 *>(cache + p.codes + p.e);
            out.w[0] = decode8<0>(q.x, s);
            out.w[1] = decode8<1>(q.x, s);
            out.w[2] = decode8<0>(q.y, s);
            out.w[3] = decode8<1>(q.y, s);
        } else {
            const uint32_t q = *reinterpret_cast<const uint32_t *>(cache + p.codes + p.e / 2);
            out.w[0] = decode4<0>(q, s);
            out.w[1] = decode4<1>(q, s);
            out.w[2] = decode4<2>(q, s);
            out.w[3] = decode4<3>(q, s);
        }
    }
    const KvRows &dst = p.kv ? v : k;
    *reinterpret_cast<Bytes16 *>(dst.p + p.t * dst.token + p.head * dst.head + p.e) = out;
}

}  // namespace

hipError_t launch_kv_write(uint8_t *cache, const KvShape &c, const KvRows &k, const KvRows &v,
                           const int64_t *slots, int64_t T, hipStream_t s) {
    const int64_t n = T * 2 * c.heads * (c.dim / 8), blocks = (n + 255) / 256;
    if (blocks == 0)
        return hipSuccess;
    if (blocks > 0x7FFFFFFF)
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(c.fmt == KV_FP8 ? kv_write_kernel<KV_FP8> : kv_write_kernel<KV_FP4>,
                       dim3((unsigned)blocks), dim3(256), 0, s, cache, c, k, v, slots, n);
    return hipGetLastError();
}

hipError_t launch_kv_read(const uint8_t *cache, const KvShape &c, const KvRows &k,
                          const KvRows &v, const int64_t *slots, int64_t T, hipStream_t s) {
    const int64_t n = T * 2 * c.heads * (c.dim / 8), blocks = (n + 255) / 256;
    if (blocks == 0)
        return hipSuccess;
    if (blocks > 0x7FFFFFFF)
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(c.fmt == KV_FP8 ? kv_read_kernel<KV_FP8> : kv_read_kernel<KV_FP4>,
                       dim3((unsigned)blocks), dim3(256), 0, s, cache, c, k, v, slots, n);
    return hipGetLastError();
}

}  // namespace w8a8
