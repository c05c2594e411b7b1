// GELU in front of the quantizers: the exact (erf) form, evaluated in float32 or looked up
// for bf16 inputs.
#pragma once

#include "quant_math.hpp"

namespace w8a8 {
namespace {

using qmath::bf16_to_f32;

// erfc(z) for z >= 0 by the Chebyshev fit of Numerical Recipes (Press, Teukolsky,
// Vetterling, Flannery, "erfcc"): t = 1 / (1 + z/2), erfc(z) ~ t exp(-z^2 + P(t)) with a
// degree-9 polynomial P, fractional error below 1.2e-7 for every z >= 0. One hardware
// reciprocal, one hardware exp2 and ten FMAs: the quantizer stays near the HBM bound.
__device__ __forceinline__ float erfc_nonneg(float z) {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.5f, z, 1.0f));
    float p = 0.17087277f;
    p = __builtin_fmaf(t, p, -0.82215223f);
    p = __builtin_fmaf(t, p, 1.48851587f);
    p = __builtin_fmaf(t, p, -1.13520398f);
    p = __builtin_fmaf(t, p, 0.27886807f);
    p = __builtin_fmaf(t, p, -0.18628806f);
    p = __builtin_fmaf(t, p, 0.09678418f);
    p = __builtin_fmaf(t, p, 0.37409196f);
    p = __builtin_fmaf(t, p, 1.00002368f);
    const float arg = __builtin_fmaf(t, p, __builtin_fmaf(-z, z, -1.26551223f));
    return t * __builtin_amdgcn_exp2f(arg * 1.44269504088896341f);
}

// GELU(x) = x * Phi(x) with 2 Phi(x) = erfc(-x / sqrt(2)): for x < 0 that is
// erfc(|x| / sqrt(2)) (no cancellation in the left tail), for x >= 0 it is 2 - erfc.
__device__ __forceinline__ float gelu_f32(float x) {
    const float e = erfc_nonneg(__builtin_fabsf(x) * 0.70710678118654752440f);
    return 0.5f * x * (x < 0.0f ? e : 2.0f - e);
}

// The same factor from a table: the inputs are bf16, so h = erfc(|x| / sqrt(2)) / 2 takes one
// value per magnitude. From 16 up it is 0; below 2^-8 it is 1/2 - |x| / sqrt(2 pi) to within
// |x|^3 / 15 (4e-9). The 12 binades between (128 magnitudes each) and the end make 6 KB, which
// every block copies to LDS: with 28 binades (down to 2^-24, where h is 1/2) the copy cost
// short calls 0.3 us more. The entries are computed here at compile time in double: a series
// up to z = 1.5, the continued fraction of erfc above.
constexpr int kGeluLo = (127 - 8) << 7, kGeluHi = (127 + 4) << 7;   // bf16 magnitude bits
constexpr int kGeluN = kGeluHi - kGeluLo + 1;

constexpr double exp_nonpos(double x) {
    int n = 0;
    for (; x < -0.01; x *= 0.5)
        ++n;
    double s = 1.0, term = 1.0;
    for (int i = 1; i <= 7; ++i) {
        term *= x / i;
        s += term;
    }
    for (; n > 0; --n)
        s *= s;
    return s;
}

constexpr double erfc_const(double z) {
    constexpr double kInvSqrtPi = 0.56418958354775628695;
    if (z < 1.5) {
        double sum = z, term = z;
        for (int n = 1; n < 60 && (term > 1e-19 || term < -1e-19); ++n) {
            term *= -z * z / n;
            sum += term / (2 * n + 1);
        }
        return 1.0 - 2.0 * kInvSqrtPi * sum;
    }
    double f = z;
    for (int n = 60; n >= 1; --n)
        f = z + 0.5 * n / f;
    return exp_nonpos(-z * z) * kInvSqrtPi / f;
}
static_assert(erfc_const(1.0) > 0.157299207050 && erfc_const(1.0) < 0.157299207051, "series");
static_assert(erfc_const(2.0) > 0.004677734981047 && erfc_const(2.0) < 0.004677734981048, "fraction");

struct alignas(16) GeluTable {
    float h[(kGeluN + 3) / 4 * 4];   // erfc(|x| / sqrt(2)) / 2 at magnitude kGeluLo + i
};

constexpr GeluTable make_gelu_table() {
    GeluTable t{};
    for (int i = 0; i + 1 < kGeluN; ++i) {
        double x = 1.0 + (i & 127) / 128.0;
        for (int e = i >> 7; e < 8; ++e)
            x *= 0.5;
        for (int e = 8; e < (i >> 7); ++e)
            x *= 2.0;
        const double h = 0.5 * erfc_const(x * 0.70710678118654752440);
        t.h[i] = h < 1e-45 ? 0.0f : (float)h;
    }
    return t;   // the last entry (|x| >= 16) is 0
}
__device__ const GeluTable kGeluTable = make_gelu_table();

// GELU of a bf16 value given by its bits h (0 .. 0xFFFF): x * Phi(x) with Phi(x) = h(|x|)
// for x < 0 and 1 - h(|x|) otherwise, the table in LDS.
__device__ __forceinline__ float gelu_lookup(uint32_t h, const float *table) {
    const float x = bf16_to_f32(h);
    const int mag = (int)(h & 0x7FFFu);
    const float tail = table[min(max(mag, kGeluLo), kGeluHi) - kGeluLo];
    const float e = mag < kGeluLo
                        ? __builtin_fmaf(__builtin_fabsf(x), -0.39894228040143267794f, 0.5f)
                        : tail;
    return x * (x < 0.0f ? e : 1.0f - e);
}

}  // namespace
}  // namespace w8a8
