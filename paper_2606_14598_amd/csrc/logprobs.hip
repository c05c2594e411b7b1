// Log probabilities of given tokens, the entropy and the most likely alternatives of rows of
// logits, in one pass over them. With x the row over the temperature, m a bound near its maximum,
// s = sum exp(x - m) and t = sum exp(x - m) (x - m):
//   log p(i) = x_i - m - log s,   H = -sum p log p = log s - t / s
// Everything in float32 and in powers of two (factor = log2(e) / temperature). Differences x - m
// are taken before they are scaled, so that a row of the type's lowest values is as any other.
// Every lane keeps its own m, s and t and rescales them only when its maximum rises by more than
// kSlack; lanes, wavefronts and workgroups are joined at the end, always in the same order.
//
// Alternatives: a wavefront keeps the best 64 of what it has read, sorted over its lanes, as keys
// of 64 bits: the value's bits in an order of integers above the complement of its index, so that
// the lower of equal values wins. Values above the k-th best are collected in LDS, and 64 of them
// at a time sorted and merged. The first values that a wavefront reads would all be collected: the
// k-th largest of its lanes' maxima is a bound that k values reach.
//
// Bound by reading the logits once.
#include "lm_internal.hpp"
#include "quant_math.hpp"

#include <algorithm>

namespace w8a8 {
namespace {

constexpr int kWaves = 4, kThreads = kWaves * 64;
// Log2 of how far a lane's maximum may rise before its sums are rescaled: s stays below 2^20 V.
constexpr float kSlack = 20.0f;
constexpr float kLowest = -3.402823466e38f;
constexpr float kLn2 = 0.693147180559945309f;

typedef uint64_t Key;         // value's order above the complement of its index; 0: none

// Float order as unsigned integers; -0 counts as 0 and a NaN as the largest.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return x != x ? 0xFFFFFFFFu : b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}

__device__ __forceinline__ Key shuffle_xor(Key k, int lanes) {
    const uint32_t lo = (uint32_t)__shfl_xor((int)(uint32_t)k, lanes);
    const uint32_t hi = (uint32_t)__shfl_xor((int)(uint32_t)(k >> 32), lanes);
    return (Key)hi << 32 | lo;
}

// One step of a sorting network: lanes l and l ^ d, the larger to the one that keeps it.
__device__ __forceinline__ Key keep(Key k, int d, bool larger) {
    const Key o = shuffle_xor(k, d);
    return (k > o) == larger ? k : o;
}

// Sorts over the lanes, largest in lane 0.
__device__ __forceinline__ Key sort64(Key k, int lane) {
#pragma unroll
    for (int n = 2; n <= 64; n *= 2)
#pragma unroll
        for (int d = n / 2; d > 0; d /= 2)
            k = keep(k, d, ((lane & d) == 0) == ((lane & n) == 0));
    return k;
}

// The 64 largest of two lists sorted over the lanes, sorted.
__device__ __forceinline__ Key merge64(Key a, Key b, int lane) {
    b = shuffle_xor(b, 63);                    // reversed: the larger of each pair are the 64
    Key k = a > b ? a : b;
#pragma unroll
    for (int d = 32; d > 0; d /= 2)
        k = keep(k, d, (lane & d) == 0);
    return k;
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
__device__ __forceinline__ Sums join(const Sums &a, const Sums &b, float factor) {
    const float m = fmaxf(a.m, b.m);
    const float da = fmaxf((a.m - m) * factor, -300.0f), db = fmaxf((b.m - m) * factor, -300.0f);
    const float wa = __builtin_amdgcn_exp2f(da), wb = __builtin_amdgcn_exp2f(db);
    return {m, a.s * wa + b.s * wb, __builtin_fmaf(a.s, da, a.t) * wa + __builtin_fmaf(b.s, db, b.t) * wb};
}

__device__ __forceinline__ Sums wave_join(Sums a, float factor) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const Sums b = {__shfl_xor(a.m, d), __shfl_xor(a.s, d), __shfl_xor(a.t, d)};
        a = join(a, b, factor);
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
    b.list = merge64(b.list, sort64(k, lane), lane);
    const uint32_t bar = (uint32_t)(lane_of(b.list, top - 1) >> 32);
    if (bar > b.bar)
        set_bar(b, bar);
}

// 8 neighbouring values of a row from element i, minus infinity behind n.
template <bool F32>
__device__ __forceinline__ void load8_values(const void *row, int64_t i, int64_t n, float (&x)[8]) {
    if (i + 8 <= n) {
        if constexpr (F32) {
            const Bytes16 *p = reinterpret_cast<const Bytes16 *>(static_cast<const float *>(row) + i);
            const Bytes16 lo = p[0], hi = p[1];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = __uint_as_float(lo.w[e]);
                x[e + 4] = __uint_as_float(hi.w[e]);
            }
        } else {
            const Bytes16 b = *reinterpret_cast<const Bytes16 *>(static_cast<const uint16_t *>(row) + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[2 * e] = __uint_as_float(b.w[e] << 16);
                x[2 * e + 1] = __uint_as_float(b.w[e] & 0xFFFF0000u);
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = -INFINITY;
            if (i + e < n)
                x[e] = F32 ? static_cast<const float *>(row)[i + e]
                           : qmath::bf16_to_f32(static_cast<const uint16_t *>(row)[i + e]);
        }
    }
}

template <bool F32>
__device__ __forceinline__ float value_at(const LogprobArgs &a, int64_t t, int64_t i) {
    return F32 ? static_cast<const float *>(a.logits)[t * a.row_stride + i]
               : qmath::bf16_to_f32(static_cast<const uint16_t *>(a.logits)[t * a.row_stride + i]);
}

// The row's results from its sums and its best (sorted over the lanes of the one wavefront that
// calls this).
template <bool F32>
__device__ __forceinline__ void finish(const LogprobArgs &a, int64_t t, const Sums &r, Key list, int lane) {
    const float log_s = __builtin_amdgcn_logf(r.s);        // base 2
    // In 64 bits, as the difference of two logits may have no float32 value where its part of the
    // temperature has.
    const auto logp = [&](float x) {
        return (float)(((double)x - r.m) * a.inverse - (double)log_s * 0.693147180559945309);
    };
    if (lane == 0) {
        const int64_t token = a.tokens[t];
        a.entropy[t] = (log_s - r.t / r.s) * kLn2;
        a.logp[t] = token >= 0 && token < a.V ? logp(value_at<F32>(a, t, token)) : 0.0f;
    }
    if (lane < a.top) {
        a.top_logp[t * a.top + lane] = logp(value_of((uint32_t)(list >> 32)));
        a.top_ids[t * a.top + lane] = (int64_t)~(uint32_t)list;
    }
}

// A workgroup reads the part blockIdx.x of `splits` of a row, 8 values a lane and LOADS loads of
// all lanes at a time. One part: the results; several: what is known of each.
template <bool F32, bool TOP>
__global__ void __launch_bounds__(kThreads)
logprobs_kernel(LogprobArgs a, int splits, int64_t share, Part *parts, Key *keys) {
    constexpr int LOADS = F32 ? 2 : 4;
    __shared__ Key waits[TOP ? kWaves : 1][128];
    __shared__ Sums all[kWaves];
    __shared__ Key lists[TOP ? kWaves : 1][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = blockIdx.x / splits;
    const int split = (int)(blockIdx.x - t * splits);
    const int64_t begin = split * share, end = min(begin + share, a.V);
    const void *row = F32 ? static_cast<const void *>(static_cast<const float *>(a.logits) + t * a.row_stride)
                          : static_cast<const uint16_t *>(a.logits) + t * a.row_stride;
    Sums r = {kLowest, 0.0f, 0.0f};
    Best best = {0, 0, NAN, 0};
    Key *const wait = waits[TOP ? wave : 0];

    for (int64_t at = begin; at < end; at += LOADS * kThreads * 8) {
        float x[LOADS][8];
#pragma unroll
        for (int u = 0; u < LOADS; ++u)
            load8_values<F32>(row, at + ((int64_t)u * kThreads + threadIdx.x) * 8, end, x[u]);
        if (TOP && at == begin) {
            // At least `top` values are as large as the top-th largest of the lanes' maxima.
            uint32_t o = 0;
#pragma unroll
            for (int u = 0; u < LOADS; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (at + ((int64_t)u * kThreads + threadIdx.x) * 8 + e < end)
                        o = max(o, order_of(x[u][e]));
            const uint32_t bar = (uint32_t)(lane_of(sort64((Key)o << 32, lane), a.top - 1) >> 32);
            set_bar(best, bar > 0 ? bar - 1 : 0);
        }
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            float top = fmaxf(fmaxf(fmaxf(x[u][0], x[u][1]), fmaxf(x[u][2], x[u][3])),
                              fmaxf(fmaxf(x[u][4], x[u][5]), fmaxf(x[u][6], x[u][7])));
            if (TOP && __any(!(top <= best.bar_value))) {
                const int64_t i = at + ((int64_t)u * kThreads + threadIdx.x) * 8;
                const uint32_t bar = best.bar;     // equal values of these 512 may be earlier ones
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t o = order_of(x[u][e]);
                    const bool passes = o > bar && i + e < end;
                    const uint64_t who = __ballot(passes);
                    if (who == 0)
                        continue;
                    if (passes)
                        wait[best.waiting + __popcll(who & ((1ull << lane) - 1))] =
                            (Key)o << 32 | (uint32_t)~(uint32_t)(i + e);
                    best.waiting += __popcll(who);
                    if (best.waiting >= 64)
                        merge_waiting(best, wait, lane, a.top);
                }
            }
            if (__any((top - r.m) * a.factor > kSlack)) {
                const float m = fmaxf(r.m, top);
                const float d = fmaxf((r.m - m) * a.factor, -300.0f), w = __builtin_amdgcn_exp2f(d);
                r.t = __builtin_fmaf(r.s, d, r.t) * w;
                r.s *= w;
                r.m = m;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = (x[u][e] - r.m) * a.factor;
                const float p = __builtin_amdgcn_exp2f(y);
                r.s += p;
                r.t = __builtin_fmaf(p, fmaxf(y, -300.0f), r.t);     // no 0 times infinity
            }
        }
    }

    r = wave_join(r, a.factor);
    if (lane == 0)
        all[wave] = r;
    if constexpr (TOP) {
        while (best.waiting > 0)
            merge_waiting(best, wait, lane, a.top);
        lists[wave][lane] = best.list;
    }
    __syncthreads();
    if (wave > 0)
        return;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
        r = join(r, all[w], a.factor);
        if constexpr (TOP)
            best.list = merge64(best.list, lists[w][lane], lane);
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

// Joins the parts of a row: lanes take the sums, wavefronts the lists.
template <bool F32>
__global__ void __launch_bounds__(kThreads)
logprobs_join_kernel(LogprobArgs a, int splits, const Part *parts, const Key *keys) {
    __shared__ Key lists[kWaves][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = blockIdx.x;
    Key list = 0;
    if (a.top > 0) {
        for (int s = wave; s < splits; s += kWaves)
            list = merge64(list, lane < a.top ? keys[(t * splits + s) * a.top + lane] : 0, lane);
        lists[wave][lane] = list;
    }
    __syncthreads();
    if (wave > 0)
        return;
    Sums r = lane < splits ? parts[t * splits + lane].sums : Sums{kLowest, 0.0f, 0.0f};
    r = wave_join(r, a.factor);
    if (a.top > 0)
#pragma unroll
        for (int w = 1; w < kWaves; ++w)
            list = merge64(list, lists[w][lane], lane);
    finish<F32>(a, t, r, list, lane);
}

// A row is divided where there are few: into parts of at least 4096 values, up to 64 (lanes of the
// join) and about 1024 workgroups in all.
constexpr int64_t kLeastShare = 4096;

int splits_of(int64_t T, int64_t V) {
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
        const dim3 grid((unsigned)(a.T * splits)), block(kThreads);
        const auto go = [&](auto f32, auto top) {
            hipLaunchKernelGGL((logprobs_kernel<decltype(f32)::value, decltype(top)::value>), grid, block, 0,
                               s, a, splits, share, parts, keys);
            if (splits > 1 && hipPeekAtLastError() == hipSuccess)
                hipLaunchKernelGGL((logprobs_join_kernel<decltype(f32)::value>), dim3((unsigned)a.T), block,
                                   0, s, a, splits, parts, keys);
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
