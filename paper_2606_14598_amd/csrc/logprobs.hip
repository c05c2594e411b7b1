// Log probabilities of given tokens, the entropy and the most likely alternatives of rows of
// logits, in one pass over them. In powers of two, with z = x log2(e) / temperature, m a number near
// the row's largest z, y = z - m (one fused operation), s = sum 2^y and t = sum 2^y y:
//   log p(i) = (y_i - log2 s) ln 2,   H = -sum p log p = (log2 s - t / s) ln 2
// Everything in float32. Every lane keeps its own m, s and t and rescales them only when its maximum
// rises by more than kSlack; lanes, wavefronts and workgroups are joined at the end, always in the
// same order. A row whose largest z has no place in that (below kFloor, as one of nothing but masks
// has it, or above kCeiling) is read again by one wavefront, differences first.
//
// Alternatives: a wavefront keeps the best 64 of what it has read, sorted over its lanes, as keys
// of 64 bits: the value's bits in an order of integers above the complement of its index, so that
// the lower of equal values wins. Values above the k-th best are collected in LDS, and 64 of them
// at a time sorted and merged. The first values that a wavefront reads would all be collected: the
// k-th largest of its lanes' maxima is a bound that k values reach.
//
// Bound by reading the logits once: 4096 x 131072 bf16 in 161 us without alternatives (6.7 TB/s; a
// plain read of as much reaches 6.8 to 7.0), 180 with 5, 199 with 20; 1024 x 131072 float32 in 82. Beside that
// read stand about 10 vector instructions a value, the exponential counted as four. One row of 131072
// takes 5.1 us in two launches, 11.0 with 20 alternatives (the networks of the workgroups and of the
// join, one after the other). us for loads without branches around them (a branch makes the compiler
// wait for all in flight), the networks in registers and one bar a workgroup, 4096 x 131072 with 5:
// 285 before, 211; streaming loads and one fused operation a value less: 195.
#include "lm_internal.hpp"
#include "quant_math.hpp"

#include <algorithm>

namespace w8a8 {
namespace {

constexpr int kWaves = 4, kThreads = kWaves * 64;
// Log2 of how far a lane's maximum may rise before its sums are rescaled. What it lags behind stands in
// log2 s and in t / s, whose difference is the entropy, and every weight added to t beside a larger one
// rounds at its size: up to 20 the entropy of 3000 x 16000 sharpened logits was 4 10^-6 off, in the
// mean, up to 4 it is 3 10^-7, as by float32 sums relative to the row's maximum. us up to 20, 4 and 0:
// 4096 x 131072 with 5 alternatives 178, 180, 182, 2500 x 30000 41.3, 41.8, 42.0.
constexpr float kSlack = 4.0f;
// Up to 2^24 the rounding of m is a distance of 1 at most, which s and log p have alike.
constexpr float kFloor = -0x1p24f, kCeiling = 0x1p24f;
constexpr double kLn2 = 0.693147180559945309;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint64_t Key;         // value's order above the complement of its index; 0: none

// Float order as unsigned integers; -0 counts as 0 and a NaN as the largest.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return x != x ? 0xFFFFFFFFu : b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}

// The value of lane l ^ D, in register operations (a shuffle goes through LDS).
template <int D>
__device__ __forceinline__ uint32_t across(uint32_t v, int lane) {
    const auto dpp = [](uint32_t x, auto ctrl) {
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xF, 0xF, false);
    };
    using std::integral_constant;
    if constexpr (D == 1)
        return dpp(v, integral_constant<int, 0xB1>{});        // quad_perm [1, 0, 3, 2]
    else if constexpr (D == 2)
        return dpp(v, integral_constant<int, 0x4E>{});        // quad_perm [2, 3, 0, 1]
    else if constexpr (D == 4)                                // l ^ 7, then ^ 3
        return dpp(dpp(v, integral_constant<int, 0x141>{}), integral_constant<int, 0x1B>{});
    else if constexpr (D == 8)
        return dpp(v, integral_constant<int, 0x128>{});       // row_ror:8
    else {
        const u32x2 r = __builtin_bit_cast(
            u32x2, D == 16 ? __builtin_amdgcn_permlane16_swap(v, v, false, false)
                           : __builtin_amdgcn_permlane32_swap(v, v, false, false));
        return lane & D ? r[0] : r[1];
    }
}

template <int D>
__device__ __forceinline__ Key across(Key k, int lane) {
    return (Key)across<D>((uint32_t)(k >> 32), lane) << 32 | across<D>((uint32_t)k, lane);
}

// One step of a sorting network: lanes l and l ^ D, the larger to the one that keeps it.
template <int D, typename K>
__device__ __forceinline__ K keep(K k, int lane, bool larger) {
    const K o = across<D>(k, lane);
    return (k > o) == larger ? k : o;
}

// Steps of D, D / 2 ... 1: a list that first rises and then falls is sorted over groups of 2 D
// lanes, largest first where `down`.
template <int D, typename K>
__device__ __forceinline__ K clean(K k, int lane, bool down) {
    k = keep<D>(k, lane, ((lane & D) == 0) == down);
    if constexpr (D > 1)
        k = clean<D / 2>(k, lane, down);
    return k;
}

// Sorts over the lanes, largest in lane 0, or in lane 63.
template <bool DOWN, typename K>
__device__ __forceinline__ K sort64(K k, int lane) {
    k = clean<1>(k, lane, (lane & 2) == 0);
    k = clean<2>(k, lane, (lane & 4) == 0);
    k = clean<4>(k, lane, (lane & 8) == 0);
    k = clean<8>(k, lane, (lane & 16) == 0);
    k = clean<16>(k, lane, (lane & 32) == 0);
    return clean<32>(k, lane, DOWN);
}

// The 64 largest of two lists, a's largest in lane 0, b's in lane 63: sorted, largest in lane 0.
__device__ __forceinline__ Key merge64(Key a, Key b, int lane) {
    return clean<32>(a > b ? a : b, lane, true);
}

__device__ __forceinline__ Key lane_of(Key k, int lane) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)k, lane);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(k >> 32), lane);
    return (Key)hi << 32 | lo;
}

// m, s and t of a part of a row.
struct Sums {
    float m, s, t;
};

// Of two parts, relative to the larger m. The distance is bounded: times a sum of zero, or a weight
// of zero, an infinite one would be no number.
__device__ __forceinline__ Sums join(const Sums &a, const Sums &b) {
    const float m = fmaxf(a.m, b.m);
    const float da = fmaxf(a.m - m, -300.0f), db = fmaxf(b.m - m, -300.0f);
    const float wa = __builtin_amdgcn_exp2f(da), wb = __builtin_amdgcn_exp2f(db);
    return {m, a.s * wa + b.s * wb, __builtin_fmaf(a.s, da, a.t) * wa + __builtin_fmaf(b.s, db, b.t) * wb};
}

__device__ __forceinline__ Sums wave_join(Sums a) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const Sums b = {__shfl_xor(a.m, d), __shfl_xor(a.s, d), __shfl_xor(a.t, d)};
        a = join(a, b);
    }
    return a;
}

// What is known of a row's part once it is read: sums, then the best `top` keys.
struct Part {
    Sums sums;
    float pad;
};

// A wavefront's best 64 and what waits to be merged into them.
struct Best {
    Key list;              // lane l: the (l + 1)-th best
    uint32_t bar;          // order that a value has to pass to be one of the best
    float bar_value;       // the same as a value; NaN while any value passes
    int waiting;
};

__device__ __forceinline__ void set_bar(Best &b, uint32_t bar) {
    b.bar = __builtin_amdgcn_readfirstlane((int)bar);
    // No value has the order of -0, which as a float would hold back zeros: the next one below.
    b.bar_value = b.bar == 0 ? NAN : value_of(b.bar == 0x7FFFFFFFu ? 0x7FFFFFFEu : b.bar);
}

// Merges the first 64 that wait (or all, with fewer), and moves the others up.
__device__ __forceinline__ void merge_waiting(Best &b, Key *wait, int lane, int top) {
    const int n = min(b.waiting, 64);
    __builtin_amdgcn_wave_barrier();           // other lanes' entries: in order, as one wavefront
    const Key k = lane < n ? wait[lane] : 0;
    const Key rest = 64 + lane < b.waiting ? wait[64 + lane] : 0;
    b.waiting -= n;
    if (lane < b.waiting)
        wait[lane] = rest;
    __builtin_amdgcn_wave_barrier();
    b.list = merge64(b.list, sort64<false>(k, lane), lane);
    const uint32_t bar = (uint32_t)(lane_of(b.list, top - 1) >> 32);
    if (bar > b.bar)
        set_bar(b, bar);
}

// The largest of three. fmaxf of values that come out of bit operations costs a second maximum each,
// which quiets them (4096 x 131072 with 5 alternatives: 187 us, so 183). Without that a signalling NaN
// hides what stands before it: the result is then another value of the three or a NaN, and the row's
// results are NaN anyway.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// 16 bytes of a row: the values i .. i + PER - 1, as float32.
template <bool F32>
struct Unit {
    static constexpr int PER = F32 ? 4 : 8;
    uint32_t raw[4];
    __device__ __forceinline__ void load(const uint8_t *row, int64_t i) {
        // Streaming: nothing is read twice (4096 x 131072: 188 us with plain loads, 170 so). Rows begin
        // at any element.
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(2)));
        const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(row + i * (F32 ? 4 : 2)));
#pragma unroll
        for (int w = 0; w < 4; ++w)
            raw[w] = v[w];
    }
    // What lies behind n becomes minus infinity.
    __device__ __forceinline__ void load_up_to(const uint8_t *row, int64_t i, int64_t n) {
        if (i + PER <= n)
            return load(row, i);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if constexpr (F32) {
                raw[w] = i + w < n ? reinterpret_cast<const uint32_t *>(row)[i + w] : 0xFF800000u;
            } else {
                const uint16_t *p = reinterpret_cast<const uint16_t *>(row) + i + 2 * w;
                const uint32_t lo = i + 2 * w < n ? p[0] : 0xFF80u, hi = i + 2 * w + 1 < n ? p[1] : 0xFF80u;
                raw[w] = lo | hi << 16;
            }
        }
    }
    __device__ __forceinline__ float operator[](int e) const {
        if constexpr (F32)
            return __uint_as_float(raw[e]);
        else
            return __uint_as_float(e & 1 ? raw[e / 2] & 0xFFFF0000u : raw[e / 2] << 16);
    }
    __device__ __forceinline__ float largest() const {
        float m = max3((*this)[0], (*this)[1], (*this)[2]);
#pragma unroll
        for (int e = 3; e < PER; e += 2)
            m = max3(m, (*this)[e], (*this)[e + 1 < PER ? e + 1 : e]);
        return m;
    }
};

template <bool F32>
__device__ __forceinline__ float value_at(const LogprobArgs &a, int64_t t, int64_t i) {
    return F32 ? static_cast<const float *>(a.logits)[t * a.row_stride + i]
               : qmath::bf16_to_f32(static_cast<const uint16_t *>(a.logits)[t * a.row_stride + i]);
}

// A row's largest value, and its sums relative to that, by one wavefront in two passes.
template <bool F32>
__device__ __forceinline__ Sums sums_again(const LogprobArgs &a, int64_t t, int lane) {
    typedef Unit<F32> U;
    const uint8_t *row = static_cast<const uint8_t *>(a.logits) + t * a.row_stride * (F32 ? 4 : 2);
    Sums r = {-INFINITY, 0.0f, 0.0f};
    for (int64_t i = lane * U::PER; i < a.V; i += 64 * U::PER) {
        U x;
        x.load_up_to(row, i, a.V);
        r.m = fmaxf(r.m, x.largest());
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
        r.m = fmaxf(r.m, __shfl_xor(r.m, d));
    for (int64_t i = lane * U::PER; i < a.V; i += 64 * U::PER) {
        U x;
        x.load_up_to(row, i, a.V);
#pragma unroll
        for (int e = 0; e < U::PER; ++e) {
            const float y = (x[e] - r.m) * a.factor, p = __builtin_amdgcn_exp2f(y);
            r.s += p;
            r.t = __builtin_fmaf(p, fmaxf(y, -300.0f), r.t);
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        r.s += __shfl_xor(r.s, d);
        r.t += __shfl_xor(r.t, d);
    }
    return r;
}

// The row's results from its sums and its best (sorted over the lanes of the one wavefront that
// calls this).
template <bool F32>
__device__ __forceinline__ void finish(const LogprobArgs &a, int64_t t, Sums r, Key list, int lane) {
    double m = r.m;
    if (!(r.m > kFloor && r.m < kCeiling)) {
        r = sums_again<F32>(a, t, lane);
        m = (double)r.m * a.factor;
    }
    const float log_s = __builtin_amdgcn_logf(r.s);        // base 2
    // In 64 bits, where every z and difference has a value.
    const auto logp = [&](float x) {
        const float p = (float)(((double)x * a.factor - m - log_s) * kLn2);
        return p > 0.0f ? 0.0f : p;                // by a rounding
    };
    if (lane == 0) {
        const int64_t token = a.tokens[t];
        const float h = (log_s - r.t / r.s) * (float)kLn2;
        a.entropy[t] = h < 0.0f ? 0.0f : h;
        a.logp[t] = token >= 0 && token < a.V ? logp(value_at<F32>(a, t, token)) : 0.0f;
    }
    if (lane < a.top) {
        a.top_logp[t * a.top + lane] = logp(value_of((uint32_t)(list >> 32)));
        a.top_ids[t * a.top + lane] = (int64_t)~(uint32_t)list;
    }
}

// WAVES wavefronts read part `split` of `splits` of a row, LOADS units of 16 bytes a lane at a time
// and the next ones meanwhile. One part: the results; several: what is known of each.
template <bool F32, bool TOP, int WAVES>
__global__ void __launch_bounds__(kThreads)
logprobs_kernel(LogprobArgs a, int splits, int64_t share, Part *parts, Key *keys) {
    typedef Unit<F32> U;
    // Two units in flight beside two in work: four take the registers of three wavefronts a SIMD
    // (4096 x 131072 with 5 alternatives 208 us, with two 201).
    constexpr int LOADS = 2, PER = U::PER, ROWS = kWaves / WAVES;
    constexpr int64_t STEP = WAVES * 64 * PER;        // values of a load of all lanes
    __shared__ Key waits[TOP ? kWaves : 1][128];
    __shared__ Sums all[kWaves];
    __shared__ Key lists[TOP ? kWaves : 1][64];
    __shared__ uint32_t bars[2][kWaves];
    __shared__ int left[kWaves];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int first_wave = wave / WAVES * WAVES;      // of this row
    int64_t t = blockIdx.x;
    int split = 0;
    if constexpr (ROWS > 1) {
        t = t * ROWS + wave / WAVES;
        if (t >= a.T)
            return;
    } else {
        t /= splits;
        split = (int)(blockIdx.x - t * splits);
    }
    const int64_t begin = split * share, end = min(begin + share, a.V);
    const uint8_t *row = static_cast<const uint8_t *>(a.logits) + t * a.row_stride * (F32 ? 4 : 2);
    Sums r = {kFloor, 0.0f, 0.0f};
    Best best = {0, 0, NAN, 0};
    Key *const wait = waits[TOP ? wave : 0];

    // n units from value `at` of this lane on; those of a whole load all lie before `end`.
    const auto process = [&](const U (&x)[LOADS], int64_t at, bool first) __attribute__((always_inline)) {
        static_assert(LOADS == 2);
        const float tops[LOADS] = {x[0].largest(), x[1].largest()};
        float top = max3(tops[0], tops[1], tops[1]);
        if (TOP && first) {
            // A bar that a.top values reach: the a.top-th largest of a wavefront's lanes' maxima (of
            // lanes that have any; a NaN's lane counts by one of its values), or the least of the
            // wavefronts' (a.top / WAVES)-th.
            const uint32_t o = sort64<true>(at < end ? order_of(top) : 0u, lane);
            uint32_t bar = (uint32_t)__builtin_amdgcn_readlane((int)o, a.top - 1);
            if constexpr (WAVES > 1) {
                if (lane == 0) {
                    bars[0][wave] = bar;
                    bars[1][wave] = (uint32_t)__builtin_amdgcn_readlane((int)o, (a.top - 1) / WAVES);
                }
                __syncthreads();
                uint32_t least = bars[1][0];
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    bar = max(bar, bars[0][w]);
                    least = min(least, bars[1][w]);
                }
                bar = max(bar, least);
            }
            set_bar(best, bar > 0 ? bar - 1 : 0);
        }
        if (TOP && __any(!(top <= best.bar_value))) {
#pragma unroll
            for (int u = 0; u < LOADS; ++u) {
                const float bar_value = best.bar_value;
                if (!__any(!(tops[u] <= bar_value)))
                    continue;
                const int64_t i = at + u * STEP;
                const uint32_t bar = best.bar;     // an equal value of this load may be an earlier one
#pragma unroll
                for (int e = 0; e < PER; ++e) {
                    if (!__any(!(x[u][e] <= bar_value)))
                        continue;
                    const uint32_t o = order_of(x[u][e]);
                    const bool passes = o > bar && i + e < end;
                    const uint64_t who = __ballot(passes);
                    if (passes)
                        wait[best.waiting + __popcll(who & ((1ull << lane) - 1))] =
                            (Key)o << 32 | (uint32_t)~(uint32_t)(i + e);
                    best.waiting += __popcll(who);
                    if (best.waiting >= 64)
                        merge_waiting(best, wait, lane, a.top);
                }
            }
        }
        top *= a.factor;
        if (__any(top - r.m > kSlack)) {
            const float m = fmaxf(r.m, top);
            const float d = fmaxf(r.m - m, -300.0f), w = __builtin_amdgcn_exp2f(d);
            r.t = __builtin_fmaf(r.s, d, r.t) * w;
            r.s *= w;
            r.m = m;
        }
#pragma unroll
        for (int u = 0; u < LOADS; ++u)
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                const float y = __builtin_fmaf(x[u][e], a.factor, -r.m);
                const float p = __builtin_amdgcn_exp2f(y);
                r.s += p;
                r.t = __builtin_fmaf(p, fmaxf(y, -300.0f), r.t);     // no 0 times infinity
            }
    };
    const int64_t lane_at = begin + ((wave - first_wave) * 64 + lane) * (int64_t)PER;
    const int64_t whole = (end - begin) / (LOADS * STEP);
    const auto load = [&](U (&x)[LOADS], int64_t n) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < LOADS; ++u)
            x[u].load(row, lane_at + (n * LOADS + u) * STEP);
    };
    U x[LOADS], y[LOADS];
    if (whole > 0) {
        // Loads without branches, so that the compiler can count those in flight: past the last
        // ones the last are loaded again.
        load(x, 0);
        for (int64_t n = 0;; n += 2) {
            load(y, min(n + 1, whole - 1));
            process(x, lane_at + n * LOADS * STEP, n == 0);
            if (n + 1 >= whole)
                break;
            load(x, min(n + 2, whole - 1));
            process(y, lane_at + (n + 1) * LOADS * STEP, false);
            if (n + 2 >= whole)
                break;
        }
    }
    if (begin + whole * LOADS * STEP < end) {
#pragma unroll
        for (int u = 0; u < LOADS; ++u)
            x[u].load_up_to(row, lane_at + (whole * LOADS + u) * STEP, end);
        process(x, lane_at + whole * LOADS * STEP, whole == 0);
    }

    r = wave_join(r);
    if constexpr (WAVES == 1) {
        while (TOP && best.waiting > 0)
            merge_waiting(best, wait, lane, a.top);
        finish<F32>(a, t, r, best.list, lane);
        return;
    }
    if (lane == 0) {
        all[wave] = r;
        // what waits, and whether there is a list
        left[wave] = TOP ? best.waiting : 0;
    }
    if constexpr (TOP)
        lists[wave][lane] = best.list;
    __syncthreads();
    if (wave > 0)
        return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w)
        r = join(r, all[w]);
    if constexpr (TOP) {
        // Most wavefronts have no list yet but a few values that wait: all of them together, sorted
        // 64 at a time.
        int from[WAVES + 1] = {};
#pragma unroll
        for (int w = 0; w < WAVES; ++w)
            from[w + 1] = from[w] + left[w];
        for (int n = 0; n < from[WAVES]; n += 64) {
            const int i = n + lane;
            Key k = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w)
                if (i >= from[w] && i < from[w + 1])
                    k = waits[w][i - from[w]];
            best.list = merge64(best.list, sort64<false>(k, lane), lane);
        }
#pragma unroll
        for (int w = 1; w < WAVES; ++w)
            if (lists[w][0] != 0)
                best.list = merge64(best.list, lists[w][63 - lane], lane);
    }
    if (splits == 1) {
        finish<F32>(a, t, r, best.list, lane);
    } else {
        if (lane == 0)
            parts[blockIdx.x].sums = r;
        if (TOP && lane < a.top)
            keys[(int64_t)blockIdx.x * a.top + lane] = best.list;
    }
}

// Joins the parts of a row: lanes take the sums, wavefronts the lists, which then meet in pairs.
constexpr int kJoinWaves = 16;

template <bool F32>
__global__ void __launch_bounds__(kJoinWaves * 64)
logprobs_join_kernel(LogprobArgs a, int splits, const Part *parts, const Key *keys) {
    __shared__ Key lists[kJoinWaves][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = blockIdx.x;
    const int waves = a.top > 0 ? min(splits, kJoinWaves) : 1;      // of them have lists
    Sums r = {kFloor, 0.0f, 0.0f};
    if (wave == 0 && lane < splits)
        r = parts[t * splits + lane].sums;
    Key list = 0;
    if (a.top > 0 && wave < waves) {
        const Key *own = keys + t * splits * a.top;
        list = lane < a.top ? own[wave * a.top + lane] : 0;
        for (int s = wave + kJoinWaves; s < splits; s += kJoinWaves)
            list = merge64(list, 63 - lane < a.top ? own[s * a.top + 63 - lane] : 0, lane);
    }
    if (wave == 0)
        r = wave_join(r);
    for (int n = 1; n < waves; n *= 2) {
        if (wave % (2 * n) == n)
            lists[wave][lane] = list;
        __syncthreads();
        if (wave % (2 * n) == 0 && wave + n < waves)
            list = merge64(list, lists[wave + n][63 - lane], lane);
    }
    if (wave == 0)
        finish<F32>(a, t, r, list, lane);
}

// A row is divided where there are few: into parts of at least 4096 values, up to 64 (lanes of the
// join) and about 1024 workgroups in all; one of up to 8192 stays whole. us with 1024 and 2048
// workgroups: 231 x 100003 float32 28.5, 31.2; 1024 x 131072 87, 95. With parts of 4096 and 8192: 1 x
// 131072, 20 alternatives, 10.8, 12.9. Divided and whole: 300 x 5000 10.8, 8.5.
constexpr int64_t kLeastShare = 4096, kWholeRow = 8192;

// Rows that a wavefront takes by itself, four a workgroup: short ones, whose four lists and sums are
// otherwise as much work as their values, where there are enough of them. us by four wavefronts and by
// one: 8192 x 8000 54, 45; 3000 x 4000 float32 19.7, 17.0; 2048 x 16000 25.3, 26.9; 1500 x 8000 13.7, 18.4.
constexpr int64_t kShortRow = 16384, kManyRows = 2560;

int splits_of(int64_t T, int64_t V) {
    if (V <= kWholeRow)
        return 1;
    const int64_t want = std::min<int64_t>(64, 1024 / T), most = (V + kLeastShare - 1) / kLeastShare;
    return (int)std::max<int64_t>(1, std::min(want, most));
}

// Rows of a launch: more are taken in pieces.
constexpr int64_t kRows = 1 << 23;
static_assert(launchable(kRows, kThreads));

}  // namespace

size_t logprobs_workspace_bytes(int64_t T, int64_t V, int top) {
    const int64_t splits = splits_of(T, V);
    return splits == 1 ? 0 : (size_t)(T * splits) * (sizeof(Part) + top * sizeof(Key));
}

hipError_t launch_logprobs(const LogprobArgs &args, void *ws, hipStream_t s) {
    const int splits = splits_of(args.T, args.V);
    // parts of whole loads, so that only the last one of a row ends inside a vector
    const int64_t share = splits == 1 ? args.V : ((args.V + splits - 1) / splits + 7) / 8 * 8;
    const bool short_rows = splits == 1 && args.V <= kShortRow && args.T >= kManyRows;
    Part *parts = static_cast<Part *>(ws);
    Key *keys = reinterpret_cast<Key *>(parts + args.T * splits);
    for (int64_t t0 = 0; t0 < args.T; t0 += kRows) {
        LogprobArgs a = args;
        a.T = std::min(args.T - t0, kRows);
        a.logits = static_cast<const uint8_t *>(args.logits) + t0 * args.row_stride * (args.f32 ? 4 : 2);
        a.tokens += t0;
        a.logp += t0;
        a.entropy += t0;
        a.top_logp += t0 * a.top;
        a.top_ids += t0 * a.top;
        const dim3 block(kThreads);
        const auto go = [&](auto f32, auto top) {
            if (short_rows)
                hipLaunchKernelGGL((logprobs_kernel<decltype(f32)::value, decltype(top)::value, 1>),
                                   dim3((unsigned)((a.T + kWaves - 1) / kWaves)), block, 0, s, a, 1, share,
                                   parts, keys);
            else
                hipLaunchKernelGGL((logprobs_kernel<decltype(f32)::value, decltype(top)::value, kWaves>),
                                   dim3((unsigned)(a.T * splits)), block, 0, s, a, splits, share, parts, keys);
            if (splits > 1 && hipPeekAtLastError() == hipSuccess)
                hipLaunchKernelGGL((logprobs_join_kernel<decltype(f32)::value>), dim3((unsigned)a.T),
                                   dim3(a.top > 0 ? kJoinWaves * 64 : 64), 0, s, a, splits, parts, keys);
            return hipGetLastError();
        };
        const auto with_top = [&](auto f32) {
            return a.top > 0 ? go(f32, std::true_type{}) : go(f32, std::false_type{});
        };
        const hipError_t e = a.f32 ? with_top(std::true_type{}) : with_top(std::false_type{});
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

}  // namespace w8a8
