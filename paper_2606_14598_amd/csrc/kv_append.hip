// New tokens into the quantized cache, with their rotary positions applied on the way: queries
// and keys are turned, queries written out, keys and values quantized into their slots.
//
// Pair p of a head, (x[p], x[p + P]) or, interleaved, (x[2p], x[2p + 1]) with P pairs a head, is
// turned by the angle position * inv_freq[p]; the position is that of the pair's axis (time,
// height, width ...), what lies behind the 2 P channels stays as it is:
//   a' = a cos - b sin, b' = b cos + a sin, float32, every operation rounded.
// Angles, their sines and cosines are taken in 64 bits and rounded once: an angle of 10^5 radians
// has 7 bits left in 32. A token's keys are quantized from float32, by the rule of mx_math.hpp.
//
// Bound by memory: queries are read and written, keys and values read and their codes written.
#include "kv_layout.hpp"
#include "lm_internal.hpp"

namespace w8a8 {
namespace {

using namespace mx;

enum Pairing : int { HALVES = 0, HALVES_ANY = 1, NEIGHBOURS = 2 };   // HALVES: P a multiple of 8

// cos and sin of an angle of a * b radians. Turns a b / 2 pi in two terms, less whole ones, then
// quarters of a turn and a remainder of at most 1/8 turn, for which the Taylor polynomials are
// exact to 2^-45 (x^15 / 15! of sin, x^16 / 16! of cos).
__device__ __forceinline__ void cos_sin(double a, double b, float &cosine, float &sine) {
    constexpr double kHi = 0.15915494309189535, kLo = -9.839338337591243e-18;   // 1 / (2 pi)
    const double x = a * b, hi = x * kHi;
    const double lo = __builtin_fma(x, kHi, -hi) + x * kLo;
    const double quarters = (hi - __builtin_rint(hi) + lo) * 4.0;
    const double whole = __builtin_rint(quarters);
    const double t = (quarters - whole) * 1.57079632679489661923, t2 = t * t;
    double s = 1.0 / 6227020800.0;
    s = __builtin_fma(s, t2, -1.0 / 39916800.0);
    s = __builtin_fma(s, t2, 1.0 / 362880.0);
    s = __builtin_fma(s, t2, -1.0 / 5040.0);
    s = __builtin_fma(s, t2, 1.0 / 120.0);
    s = __builtin_fma(s, t2, -1.0 / 6.0);
    s = __builtin_fma(s * t2, t, t);
    double c = -1.0 / 87178291200.0;
    c = __builtin_fma(c, t2, 1.0 / 479001600.0);
    c = __builtin_fma(c, t2, -1.0 / 3628800.0);
    c = __builtin_fma(c, t2, 1.0 / 40320.0);
    c = __builtin_fma(c, t2, -1.0 / 720.0);
    c = __builtin_fma(c, t2, 1.0 / 24.0);
    c = __builtin_fma(c, t2, -0.5);
    c = __builtin_fma(c, t2, 1.0);
    const int q = (int)whole & 3;
    const float cf = (float)c, sf = (float)s;
    cosine = (q & 1) ? ((q & 2) ? sf : -sf) : ((q & 2) ? -cf : cf);
    sine = (q & 1) ? ((q & 2) ? -cf : cf) : ((q & 2) ? -sf : sf);
}

// A workgroup takes a token. Thread -> unit of 8 channels, the same in every head that it works
// on, so that its cosines and sines stay in registers; HEADS heads at a time, LOADS times that in
// flight. Queries first, then keys, then values.
template <int D>
constexpr int append_threads() { return D == 192 ? 192 : 256; }

template <int FMT, int D, int PAIRING>
__global__ void __launch_bounds__(append_threads<D>())
kv_append_kernel(uint8_t *cache, KvShape c, AppendArgs a) {
    constexpr int UNITS = D / 8, HEADS = append_threads<D>() / UNITS, LOADS = 4;
    __shared__ float cosines[D / 2], sines[D / 2];
    const int unit = threadIdx.x % UNITS, first = threadIdx.x / UNITS, e = unit * 8;
    const int64_t t = blockIdx.x;
    const Token tok = token_of(c, a.slots, t, a.T);
    // padding has no keys or values to write
    const int rotated = a.q_heads + c.heads, heads = tok.keys < 0 ? a.q_heads : rotated + c.heads;

    const auto row_of = [&](int h) {
        return h < a.q_heads ? a.q.p + t * a.q.token + h * a.q.head
               : h < rotated ? a.k.p + t * a.k.token + (h - a.q_heads) * a.k.head
                             : a.v.p + t * a.v.token + (h - rotated) * a.v.head;
    };
    for (int i = threadIdx.x; i < a.pairs; i += append_threads<D>()) {
        int axis = 0;
#pragma unroll
        for (int n = 0; n < kMaxAxes - 1; ++n)
            axis += n < a.axes - 1 && i >= a.section_end[n];
        cos_sin((double)a.positions[t * a.axes + axis], (double)a.inv_freq[i], cosines[i], sines[i]);
    }
    __syncthreads();
    // This thread's channels e + i: turned where on[i]; sines with the sign of the pair's half.
    float cs[8], sn[8];
    bool on[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int ch = e + i;
        on[i] = ch < 2 * a.pairs;
        const int p = PAIRING == NEIGHBOURS ? ch / 2 : ch < a.pairs ? ch : ch - a.pairs;
        const bool second = PAIRING == NEIGHBOURS ? ch & 1 : ch >= a.pairs;
        const float s = on[i] ? sines[p] : 0.0f;
        cs[i] = on[i] ? cosines[p] : 1.0f;
        sn[i] = second ? s : -s;
    }
    // Where the other half of each pair lies, from this thread's unit (HALVES: of all 8).
    const int across = e < a.pairs ? a.pairs : on[0] ? -a.pairs : 0;

    for (int h0 = first; h0 < heads; h0 += HEADS * LOADS) {
        uint32_t x[LOADS][4], y[LOADS][4];
#pragma unroll
        for (int n = 0; n < LOADS; ++n) {
            const int h = min(h0 + n * HEADS, heads - 1);
            const uint16_t *src = row_of(h) + e;
            const Bytes16 own = *reinterpret_cast<const Bytes16 *>(src);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[n][i] = own.w[i];
            if constexpr (PAIRING == HALVES) {
                const Bytes16 other = *reinterpret_cast<const Bytes16 *>(src + across);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    y[n][i] = other.w[i];
            } else if constexpr (PAIRING == HALVES_ANY) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const auto other = [&](int k) -> uint32_t {
                        const int ch = e + k;
                        return src[k + (ch < a.pairs ? a.pairs : ch < 2 * a.pairs ? -a.pairs : 0)];
                    };
                    y[n][i] = other(2 * i) | other(2 * i + 1) << 16;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    y[n][i] = x[n][i] >> 16 | x[n][i] << 16;
            }
        }
#pragma unroll
        for (int n = 0; n < LOADS; ++n) {
            const int h = h0 + n * HEADS;
            if (h >= heads)              // the four lanes of a block have one head
                break;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float own = __uint_as_float(i & 1 ? x[n][i / 2] & 0xFFFF0000u : x[n][i / 2] << 16);
                const float other = __uint_as_float(i & 1 ? y[n][i / 2] & 0xFFFF0000u : y[n][i / 2] << 16);
                v[i] = on[i] && h < rotated ? own * cs[i] + other * sn[i] : own;
            }
            if (h < a.q_heads) {
                Bytes16 out;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    out.w[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)v[2 * i], (__bf16)v[2 * i + 1]});
                *reinterpret_cast<Bytes16 *>(a.q_out + (t * a.q_heads + h) * D + e) = out;
                continue;
            }
            const Unit8<FMT, D> at(c, tok, (h - a.q_heads) * UNITS + unit);
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
            m = quad_max(m) >> 23;
            const uint32_t byte = scale_byte<FMT == KV_FP8 ? kTop8 : kTop4>(m);
            const float s = scale_operand(byte);
            if constexpr (FMT == KV_FP8) {
                uint2 q = make_uint2(encode8_f32(v[0], v[1], v[2], v[3], m, s),
                                     encode8_f32(v[4], v[5], v[6], v[7], m, s));
                if (byte == kNaNScale)
                    q = make_uint2(0, 0);
                *reinterpret_cast<uint2 *>(cache + at.codes) = q;
            } else {
                *reinterpret_cast<uint32_t *>(cache + at.codes) =
                    byte == kNaNScale ? 0 : encode4_f32(v, s);
            }
            if (e % 32 == 0)
                cache[at.scale] = (uint8_t)byte;
        }
    }
}

// Tokens of a launch: more than a grid holds are taken in pieces.
constexpr int64_t kTokens = 1 << 23;
static_assert(launchable(kTokens, 256));

}  // namespace

hipError_t launch_kv_append(uint8_t *cache, const KvShape &c, const AppendArgs &args, hipStream_t s) {
    const int pairing = args.interleaved ? NEIGHBOURS : args.pairs % 8 == 0 ? HALVES : HALVES_ANY;
    const auto run = [&](auto fmt, auto dim) {
        constexpr int F = decltype(fmt)::value, D = decltype(dim)::value;
        for (int64_t t0 = 0; t0 < args.T; t0 += kTokens) {
            AppendArgs a = args;
            a.T = args.T - t0 < kTokens ? args.T - t0 : kTokens;
            a.q.p += t0 * a.q.token;
            a.k.p += t0 * a.k.token;
            a.v.p += t0 * a.v.token;
            a.q_out += t0 * a.q_heads * D;
            a.slots += t0;
            a.positions += t0 * a.axes;
            const dim3 grid((unsigned)a.T), block(append_threads<D>());
            if (pairing == HALVES)
                hipLaunchKernelGGL((kv_append_kernel<F, D, HALVES>), grid, block, 0, s, cache, c, a);
            else if (pairing == HALVES_ANY)
                hipLaunchKernelGGL((kv_append_kernel<F, D, HALVES_ANY>), grid, block, 0, s, cache, c, a);
            else
                hipLaunchKernelGGL((kv_append_kernel<F, D, NEIGHBOURS>), grid, block, 0, s, cache, c, a);
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

}  // namespace w8a8
