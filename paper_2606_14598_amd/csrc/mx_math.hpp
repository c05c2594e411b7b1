// Microscaled (MX) blocks: 32 neighbouring values that share one power-of-two scale, after
// the OCP Microscaling Formats specification (v1.0). A block's scale byte s stands for
// 2^(s - 127); its elements are e2m1 (4 bits, up to 6) or e4m3 (8 bits, up to 448).
//   s = floor(log2(a)) - m + 127, at least 0, with a the block's largest magnitude and
//   m = 2 (e2m1) or 8 (e4m3), the exponents of the formats' largest values;
//   element = v / 2^(s - 127), rounded to nearest even and saturated.
// A block that holds an infinity or a NaN gets s = 255 and zero elements, and stands for 32
// NaN. The hardware conversions take the scale as the exponent field of a float32: for s = 0
// that is a zero, which they read as 2^-127. They round to nearest even (checked on all bf16
// values); the e4m3 one does not saturate, so its inputs are clamped first.
#pragma once

#include "quant_math.hpp"

namespace w8a8 {
namespace mx {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));

constexpr int kTop4 = 2, kTop8 = 8;         // exponents of 6 and 448
constexpr uint32_t kNaNScale = 255;

// The scale byte of a block whose largest magnitude has exponent field e (bf16's and
// float32's are alike): 255 for an infinity or a NaN.
template <int TOP>
__device__ __forceinline__ uint32_t scale_byte(uint32_t e) {
    return e == 255 ? kNaNScale : (uint32_t)max((int)e - TOP, 0);
}

__device__ __forceinline__ float scale_operand(uint32_t byte) {
    return __uint_as_float(byte << 23);
}

// Larger of the halves of both words, as 16-bit magnitudes.
__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                                                  __builtin_bit_cast(u16x2, b)));
}

__device__ __forceinline__ uint32_t min_halves(uint32_t a, uint32_t b) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u16x2, a),
                                                                  __builtin_bit_cast(u16x2, b)));
}

// Magnitude bits of two bf16 values.
__device__ __forceinline__ uint32_t magnitudes(uint32_t w) { return w & 0x7FFF7FFFu; }

// Eight e2m1 elements of eight bf16 values (four words), the first in the low bits.
__device__ __forceinline__ uint32_t encode4_bf16(const uint32_t (&w)[4], float scale) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[0]), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[1]), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[2]), scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[3]), scale, 3);
    return c;
}

// The same of eight float32 values.
__device__ __forceinline__ uint32_t encode4_f32(const float (&v)[8], float scale) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
    return c;
}

// Two words of bf16 values to four e4m3 elements. Magnitudes above 448 scales (mantissa over
// 0x60 in the block's largest binade, whose exponent field is top) become 448 scales first;
// below exponent field 8, where the scale byte stays 0, all magnitudes are under 256 scales.
__device__ __forceinline__ uint32_t encode8_bf16(uint32_t a, uint32_t b, uint32_t top,
                                                 float scale) {
    const uint32_t most = (max(top, (uint32_t)kTop8) << 7 | 0x60u) * 0x10001u;
    const auto clamp = [&](uint32_t w) {
        return (w & 0x80008000u) | min_halves(magnitudes(w), most);
    };
    i16x2 c = {0, 0};
    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, clamp(a)), scale,
                                                  false);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, clamp(b)), scale,
                                                  true);
    return __builtin_bit_cast(uint32_t, c);
}

// Two bf16 values (a word) of byte SEL of e2m1 codes, or of half SEL of e4m3 codes. Exact:
// both formats' values times a power of two are bf16 values (scale 255 gives NaN).
template <int SEL>
__device__ __forceinline__ uint32_t decode4(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
}

template <int SEL>
__device__ __forceinline__ uint32_t decode8(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, SEL != 0));
}

// 8 bf16 values of row `row` (K of them) from channel k, zeros behind K. Any alignment.
__device__ __forceinline__ void load8(const uint16_t *row, int64_t k, int64_t K,
                                      uint32_t (&w)[4]) {
    if (k + 8 <= K) {
        const Bytes16 b = *reinterpret_cast<const Bytes16 *>(row + k);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = b.w[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = k + 2 * i < K ? row[k + 2 * i] : 0;
            const uint32_t hi = k + 2 * i + 1 < K ? row[k + 2 * i + 1] : 0;
            w[i] = lo | hi << 16;
        }
    }
}

// Largest of v over the four lanes of a block.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));
}

}  // namespace mx
}  // namespace w8a8
