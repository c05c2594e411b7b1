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
// Bound by memory: queries are read and written, keys and values read and their codes written. 20000
// tokens of 32 + 2 x 8 heads of 128 take 86 us in 4 bits (5.0 TB/s; a large copy reaches 5.1), 4600 of
// 18 + 2 x 18 heads of 256, three axes, neighbouring pairs, 49 (4.4), 64 of the first 4.6 (a launch, an
// angle and two loads in series). Halves of a number of pairs that 8 does not divide: 4000 tokens of 54
// heads of 256, 85 pairs 78, 80 pairs 45 (loads at 2-byte alignment, shifts of the one unit).
#include "kv_layout.hpp"
#include "lm_internal.hpp"

#include <algorithm>

namespace w8a8 {
namespace {

using namespace mx;

// HALVES: P a multiple of 8. HALVES_ANY: any other.
enum Pairing : int { HALVES = 0, HALVES_ANY = 1, NEIGHBOURS = 2 };

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
// flight. Queries first, then keys, then values. The other half of a unit's pairs is a second load of
// 16 bytes, at the row's own alignment. Where the first half ends inside a unit (HALVES_ANY: one unit
// of a head), the partners of its channels are the last of the second half and the first of the first:
// two loads, shifted together; with fewer than 8 pairs they are loaded one by one.
template <int D>
constexpr int append_threads() { return D == 192 ? 192 : 256; }
template <int D>
constexpr int append_heads() { return append_threads<D>() / (D / 8); }

template <int FMT, int D, int PAIRING, int LOADS>
__global__ void __launch_bounds__(append_threads<D>())
kv_append_kernel(uint8_t *cache, KvShape c, AppendArgs a) {
    constexpr int UNITS = D / 8, HEADS = append_heads<D>();
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
    // Where the other half of each pair lies, from this thread's unit.
    const bool mixed = PAIRING == HALVES_ANY && e < a.pairs && e + 8 > a.pairs;
    const int across = mixed ? max(2 * a.pairs - 8, 0) - e : e < a.pairs ? a.pairs : on[0] ? -a.pairs : 0;

    for (int h0 = first + blockIdx.y * (HEADS * LOADS); h0 < heads; h0 += gridDim.y * (HEADS * LOADS)) {
        uint32_t x[LOADS][4], y[LOADS][4];
#pragma unroll
        for (int n = 0; n < LOADS; ++n) {
            const int h = min(h0 + n * HEADS, heads - 1);
            const uint16_t *src = row_of(h) + e;
            const Bytes16 own = *reinterpret_cast<const Bytes16 *>(src);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[n][i] = own.w[i];
            if constexpr (PAIRING != NEIGHBOURS) {
                const Bytes16 other = *reinterpret_cast<const Bytes16 *>(src + across);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    y[n][i] = other.w[i];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    y[n][i] = x[n][i] >> 16 | x[n][i] << 16;
            }
        }
        if constexpr (PAIRING == HALVES_ANY) {
            if (mixed) {
                const int skip = e + 8 - a.pairs;          // of the second half's last 8
#pragma unroll
                for (int n = 0; n < LOADS; ++n) {
                    const uint16_t *row = row_of(min(h0 + n * HEADS, heads - 1));
                    if (a.pairs < 8) {                     // unit 0 holds all pairs
                        const auto other = [&](int k) -> uint32_t {
                            return row[k < a.pairs ? k + a.pairs : k < 2 * a.pairs ? k - a.pairs : k];
                        };
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            y[n][i] = other(2 * i) | other(2 * i + 1) << 16;
                    } else {
                        const Bytes16 head = *reinterpret_cast<const Bytes16 *>(row);
                        uint32_t w[8];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            w[i] = y[n][i];
                            w[i + 4] = head.w[i];
                        }
                        // selects on values: one between array elements would put the array in memory
                        const auto moved = [&](bool by, uint32_t here, uint32_t there) {
                            return by ? there : here;
                        };
#pragma unroll
                        for (int i = 0; i < 6; ++i)
                            w[i] = moved(skip & 4, w[i], w[i + 2]);
#pragma unroll
                        for (int i = 0; i < 5; ++i)
                            w[i] = moved(skip & 2, w[i], w[i + 1]);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            y[n][i] = moved(skip & 1, w[i], w[i] >> 16 | w[i + 1] << 16);
                    }
                }
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
            const int passes = (args.q_heads + 2 * c.heads + append_heads<D>() - 1) / append_heads<D>();
            const auto go = [&](auto pairing, auto loads) {
                // Few tokens: several workgroups a token, up to what the card holds at once.
                constexpr int L = decltype(loads)::value;
                const int64_t parts = std::min<int64_t>((passes + L - 1) / L, std::max<int64_t>(2048 / a.T, 1));
                const dim3 grid((unsigned)a.T, (unsigned)parts), block(append_threads<D>());
                hipLaunchKernelGGL((kv_append_kernel<F, D, decltype(pairing)::value, decltype(loads)::value>),
                                   grid, block, 0, s, cache, c, a);
            };
            const auto with_loads = [&](auto pairing) {
                // As many in flight as divide the passes over the heads best, the more the better:
                // 20000 tokens of 48 heads of 128 (three passes) 86.9 us with three, 96.6 with four; 9000 of
                // 45 heads of 64 (two) 25.0 with two, 30.2 with four.
                const auto over = [&](int n) { return (passes + n - 1) / n * n; };
                if (over(4) <= std::min(over(3), over(2)))
                    go(pairing, std::integral_constant<int, 4>{});
                else if (over(3) <= over(2))
                    go(pairing, std::integral_constant<int, 3>{});
                else
                    go(pairing, std::integral_constant<int, 2>{});
            };
            if (pairing == HALVES)
                with_loads(std::integral_constant<int, HALVES>{});
            else if (pairing == HALVES_ANY)
                with_loads(std::integral_constant<int, HALVES_ANY>{});
            else
                with_loads(std::integral_constant<int, NEIGHBOURS>{});
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
