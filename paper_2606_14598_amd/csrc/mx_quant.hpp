// The 4-bit quantizer's arithmetic on a block spread over four lanes, shared by the quantizer
// and by the linear for few tokens, so that both give the same codes.
#pragma once

#include "gelu.hpp"
#include "mx_math.hpp"
#include "w8a8_internal.hpp"

namespace w8a8 {
namespace {

// Channel multipliers k .. k + 7 of K, zeros behind K.
__device__ __forceinline__ void load_multipliers(const float *col_mul, int64_t k, int64_t K,
                                                 float (&c)[8]) {
    if (k + 8 <= K) {
        const Bytes16 lo = *reinterpret_cast<const Bytes16 *>(col_mul + k);
        const Bytes16 hi = *reinterpret_cast<const Bytes16 *>(col_mul + k + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            c[e] = __uint_as_float(lo.w[e]);
            c[e + 4] = __uint_as_float(hi.w[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            c[e] = k + e < K ? col_mul[k + e] : 0.0f;
    }
}

// Codes and scale byte of T(x) * c for a lane's 8 neighbouring bf16 values w; the four lanes of
// a block (lanes 4i .. 4i + 3) call it together. gelu: the table, in LDS (ACT_GELU).
template <int ACT, bool CM>
__device__ __forceinline__ uint32_t quantize_quad(const uint32_t (&w)[4], const float (&c)[8],
                                                  const float *gelu, uint32_t &byte) {
    using namespace mx;
    uint32_t q;
    if constexpr (ACT == ACT_NONE && !CM) {
        uint32_t m = max_halves(max_halves(magnitudes(w[0]), magnitudes(w[1])),
                                max_halves(magnitudes(w[2]), magnitudes(w[3])));
        m = quad_max(max(m & 0xFFFFu, m >> 16));
        byte = scale_byte<kTop4>(m >> 7);
        q = encode4_bf16(w, scale_operand(byte));
    } else {
        float v[8];
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t h = (w[e / 2] >> (16 * (e & 1))) & 0xFFFFu;
            v[e] = ACT == ACT_GELU ? gelu_lookup(h, gelu) : bf16_to_f32(h);
            if constexpr (CM)
                v[e] *= c[e];
            m = max(m, __float_as_uint(v[e]) & 0x7FFFFFFFu);
        }
        m = quad_max(m);
        byte = scale_byte<kTop4>(m >> 23);
        q = encode4_f32(v, scale_operand(byte));
    }
    return byte == kNaNScale ? 0 : q;
}

}  // namespace
}  // namespace w8a8
