// Attention over the quantized cache of kv_cache.hip.
//
// Sequence b has kv_lens[b] cached tokens, the last lq of which its lq queries belong to:
// query i sees the keys j < kv_lens[b], and with the causal rule j <= kv_lens[b] - lq + i. Its
// output is sum_j p_j v_j / sum_j p_j with p_j = exp(scale q.k_j - max), zeros where it sees
// no key.
//
// The queries of all the heads that share a key/value head are the rows of one problem: row
// i * group + g. One pass over the keys keeps a running maximum m and sum l for each row
// (float32); exponentials are powers of two, their arguments scaled by log2(e).
//   S^T = K Q^T and O^T = V^T P^T on the bf16 matrix instructions: an accumulator lane then
// holds one row, so maxima, sums and the rescaling of O stay inside a lane but for one
// exchange of the maximum between the lanes that share a row, and the weights P^T come out of
// S^T in the layout the second product takes them in. Codes decode to bf16 exactly; the
// weights are rounded to bf16 for the second product (2^-9 of each weight; their sum is taken
// before).
#include "../../include/w8a8.h"
#include "mx_internal.hpp"
#include "mx_math.hpp"
#include "quant_math.hpp"

namespace w8a8 {
namespace {

using namespace mx;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// How the keys of a launch are divided: chunks of `chunk` tokens (a multiple of 128), of which
// workgroup s of `splits` takes numbers s, s + splits, ...
struct Split {
    int chunk, splits;
    float *part;     // splits > 1: [splits][T * q heads][dim + 4]: O, m, l, two unused
    uint64_t magic;  // n / (page / 16) = n * magic >> 32 for n < 2^22 (kMaxTokens / 16)
};

constexpr int kMaxChunk = 8192;
constexpr int kSplitRows = 16;
static_assert(W8A8_KV_MAX_TOKENS / 16 <= 1 << 22 && W8A8_KV_MAX_PAGE / 16 <= 1 << 10, "magic");

struct Seq {
    int64_t q0;      // first query
    int lq, kv;
};

__device__ __forceinline__ Seq sequence(const KvShape &c, const KvAttnArgs &a, int b) {
    Seq s;
    if (a.q_starts) {      // kept inside the queries whatever the array holds
        s.q0 = min(max((int64_t)a.q_starts[b], (int64_t)0), a.T);
        s.lq = (int)(min((int64_t)a.q_starts[b + 1], a.T) - s.q0);
    } else {
        s.lq = (int)(a.T / a.seqs);
        s.q0 = (int64_t)b * s.lq;
    }
    s.kv = min(a.kv_lens[b], a.table_pages * c.page);
    return s;
}

// Tokens that query i sees.
__device__ __forceinline__ int seen(const Seq &s, int i, int causal) {
    return max(0, causal ? min(s.kv, s.kv - s.lq + i + 1) : s.kv);
}

// Chunks with a token that some row of row tile rt (of `rows` rows) sees.
__device__ __forceinline__ int chunks_of(const Seq &s, int rt, int rows, const KvAttnArgs &a,
                                         int chunk) {
    const int last = min(rt * rows + rows, s.lq * a.group) - 1;
    return (seen(s, last / a.group, a.causal) + chunk - 1) / chunk;
}

__device__ __forceinline__ float max_of_row(float v) {
    // lanes l, l ^ 16, l ^ 32, l ^ 48 hold the same row
    u32x2 r = __builtin_bit_cast(
        u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_bit_cast(
        u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float sum_of_row(float v) {
    u32x2 r = __builtin_bit_cast(
        u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_bit_cast(
        u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)lo, (__bf16)hi});
}

// Element E8 (8 values, four words) of a unit's codes.
template <int FMT, int E8>
__device__ __forceinline__ u32x4 decode_part(const u32x4 &codes, float s) {
    if constexpr (FMT == KV_FP8) {
        return u32x4{decode8<0>(codes[2 * E8], s), decode8<1>(codes[2 * E8], s),
                     decode8<0>(codes[2 * E8 + 1], s), decode8<1>(codes[2 * E8 + 1], s)};
    } else {
        return u32x4{decode4<0>(codes[E8], s), decode4<1>(codes[E8], s),
                     decode4<2>(codes[E8], s), decode4<3>(codes[E8], s)};
    }
}

template <int N>
struct Unit;
template <>
struct Unit<16> {
    static __device__ __forceinline__ u32x4 load(const uint8_t *p) {
        return *reinterpret_cast<const u32x4 *>(p);
    }
};
template <>
struct Unit<8> {
    static __device__ __forceinline__ u32x4 load(const uint8_t *p) {
        const u32x2 v = *reinterpret_cast<const u32x2 *>(p);
        return u32x4{v[0], v[1], 0, 0};
    }
};

// Few rows (16 a workgroup): the keys are divided among workgroups, and among the four
// wavefronts of each in tiles of 32 tokens; every wavefront keeps its own m, l and O, joined
// in LDS at the end. Keys go from memory to the matrix registers as they are: lane (t, g) =
// (lane % 16, lane / 16) holds of token t the elements whose unit number is g modulo 4, and Q
// is loaded in the same order. Values pass through the wavefront's own piece of LDS, decoded,
// and come back transposed. The next tile's codes are loaded while this one is worked on.
template <int FMT, int D>
__global__ void __launch_bounds__(256, 2)
kv_attention_split_kernel(KvShape c, KvAttnArgs a, Split sp) {
    constexpr int KU = FMT == KV_FP4 && D % 128 == 0 ? 32 : 16;   // elements of a key unit
    constexpr int KB = FMT == KV_FP8 ? KU : KU / 2;               // its bytes
    constexpr int NK = D / (4 * KU);                              // a lane's, for 16 tokens
    constexpr int VU = FMT == KV_FP8 ? 16 : 32;                   // a value unit: 16 bytes
    constexpr int VT = D / VU;                                    // of a token
    constexpr int NV = 32 * VT / 64;                              // a lane's, for 32 tokens
    constexpr int CB = FMT == KV_FP8 ? D : D / 2;                 // code bytes of a token
    constexpr int RS = 2 * D + 32;       // LDS row of a decoded value; 4 rows x 32 bytes of a
                                         // transposing read then lie in different banks
    constexpr int F = D / 16;
    __shared__ __attribute__((aligned(16))) uint8_t lds[4][32 * RS];
    __shared__ int block_page[kMaxChunk / 16];
    __shared__ float row_m[4][16], row_l[4][16], all_l[16], all_m[16];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, g = lane >> 4;
    const int split = blockIdx.x % sp.splits, head = blockIdx.x / sp.splits % c.heads;
    const int b = blockIdx.x / sp.splits / c.heads;
    const Seq seq = sequence(c, a, b);
    const int rows = seq.lq * a.group, q_heads = c.heads * a.group;
    const int64_t head_bytes = c.head_bytes();
    uint8_t *const vt = lds[wave];

    for (int rt = blockIdx.y; rt * kSplitRows < rows; rt += gridDim.y) {
        const int nch = chunks_of(seq, rt, kSplitRows, a, sp.chunk);
        const int used = min(sp.splits, nch);
        if (split >= max(used, 1))
            continue;
        const int row = rt * kSplitRows + r16;
        const bool live = row < rows;
        const int qi = live ? row / a.group : 0;
        const int qh = head * a.group + (live ? row % a.group : 0);
        const int limit = live ? seen(seq, qi, a.causal) : 0;
        const int all_see = seen(seq, rt * kSplitRows / a.group, a.causal);   // every live row
        const int some_see =
            seen(seq, (min(rt * kSplitRows + kSplitRows, rows) - 1) / a.group, a.causal);
        u32x4 q[NK][KU / 8];
        {
            const uint16_t *src = a.q + (seq.q0 + qi) * a.q_token + qh * a.q_head;
#pragma unroll
            for (int s = 0; s < NK; ++s)
#pragma unroll
                for (int e = 0; e < KU / 8; ++e) {
                    const Bytes16 v =
                        *reinterpret_cast<const Bytes16 *>(src + (4 * s + g) * KU + 8 * e);
                    q[s][e] = live ? u32x4{v.w[0], v.w[1], v.w[2], v.w[3]} : u32x4{};
                }
        }
        f32x4 o[F];
#pragma unroll
        for (int f = 0; f < F; ++f)
            o[f] = f32x4{};
        float m = -INFINITY, l = 0.0f;
        uint32_t row_nan = 0;      // blocks of the row's output that a seen NaN value reaches

        for (int ch = split; ch < nch; ch += sp.splits) {
            const int j_first = ch * sp.chunk;
            const int j_end = min(j_first + sp.chunk, some_see);
            const int ntile = (j_end - j_first + 31) / 32;
            __syncthreads();       // the table and the LDS rows of what came before are read
            {
                const int n_blocks = (j_end - j_first + 15) / 16;
                const int32_t *t = a.table + b * a.table_stride;
                for (int i = threadIdx.x; i < ntile * 2; i += 256) {
                    const uint32_t blk = (uint32_t)(j_first / 16 + min(i, n_blocks - 1));
                    const int page = t[blk * sp.magic >> 32];
                    block_page[i] = (int)min((int64_t)max(page, 0), c.pages - 1);
                }
            }
            __syncthreads();

            u32x4 kc[2][NK], vc[NV];
            uint32_t ks[2][NK], vs[NV];
            const auto load = [&](int tile) {
                const uint8_t *kbase[2], *kscale[2];
                int64_t vofs[2];
                int at[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int page = __builtin_amdgcn_readfirstlane(block_page[2 * tile + h]);
                    const uint32_t blk = (uint32_t)(j_first / 16 + 2 * tile + h);
                    const uint32_t pb = (uint32_t)c.page / 16;
                    // its place in the page; blocks past the last one repeat it
                    const uint32_t last = (uint32_t)(j_end - 1) / 16;
                    const uint32_t bb = min(blk, last);
                    at[h] = (int)(bb - (uint32_t)(bb * sp.magic >> 32) * pb) * 16;
                    const int64_t base = ((int64_t)page * 2 * c.heads + head) * head_bytes;
                    kbase[h] = a.cache + base + (int64_t)at[h] * CB;
                    kscale[h] = a.cache + base + (int64_t)c.page * CB + at[h] * (D / 32);
                    vofs[h] = base + c.heads * head_bytes;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int s = 0; s < NK; ++s) {
                        kc[h][s] = Unit<KB>::load(kbase[h] + (uint32_t)(r16 * CB + (4 * s + g) * KB));
                        ks[h][s] = kscale[h][(uint32_t)(r16 * (D / 32) + (4 * s + g) * KU / 32)];
                    }
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int unit = i * 64 + lane, tok = unit / VT, part = unit % VT;
                    // NV even: an instruction's tokens lie in one half of the tile
                    const int h = NV % 2 == 0 ? 2 * i / NV : 0;
                    int64_t base = vofs[h];
                    int in = at[h] + tok - 16 * h;
                    if constexpr (NV % 2 != 0) {
                        base = tok < 16 ? vofs[0] : vofs[1];
                        in = tok < 16 ? at[0] + tok : at[1] + tok - 16;
                    }
                    const uint8_t *p = a.cache + base;
                    vc[i] = Unit<16>::load(p + (uint32_t)(in * CB + part * 16));
                    vs[i] = p[(uint32_t)(c.page * CB + in * (D / 32) + part * VU / 32)];
                }
            };

            if (wave < ntile)
                load(wave);
            for (int tile = wave; tile < ntile; tile += 4) {
                const int j0 = j_first + tile * 32;
                // Scores: token 16 h + 4 g + e in s[h][e].
                f32x4 s[2] = {f32x4{}, f32x4{}};
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int u = 0; u < NK; ++u) {
                        const float sc = scale_operand(ks[h][u]);
                        const auto mul = [&](auto e8) {
                            s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                __builtin_bit_cast(bf16x8,
                                                   decode_part<FMT, decltype(e8)::value>(kc[h][u], sc)),
                                __builtin_bit_cast(bf16x8, q[u][decltype(e8)::value]), s[h], 0, 0, 0);
                        };
                        mul(std::integral_constant<int, 0>{});
                        mul(std::integral_constant<int, 1>{});
                        if constexpr (KU == 32) {
                            mul(std::integral_constant<int, 2>{});
                            mul(std::integral_constant<int, 3>{});
                        }
                    }
                // Values to LDS. Tokens past the end, and in tiles that some rows see only in
                // part the NaN blocks, become zeros (a zero weight would not silence them).
                const bool part_seen = j0 + 32 > all_see;
                bool any_nan = false;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int unit = i * 64 + lane, tok = unit / VT, part = unit % VT;
                    if (part_seen) {
                        const bool past = j0 + tok >= seq.kv;
                        const bool nan = vs[i] == kNaNScale && !past;
                        any_nan |= nan;
                        if (past || nan) {
                            vc[i] = u32x4{};
                            vs[i] = nan ? 256 : 0;     // 256: marked, and a zero scale operand
                        }
                    }
                    const float sc = scale_operand(vs[i] & 255);
                    u32x4 *dst = reinterpret_cast<u32x4 *>(vt + tok * RS + part * VU * 2);
                    dst[0] = decode_part<FMT, 0>(vc[i], sc);
                    dst[1] = decode_part<FMT, 1>(vc[i], sc);
                    if constexpr (VU == 32) {
                        dst[2] = decode_part<FMT, 2>(vc[i], sc);
                        dst[3] = decode_part<FMT, 3>(vc[i], sc);
                    }
                }
                if (part_seen && __any(any_nan)) {
                    // Rare: which rows see a NaN value, and in which blocks of 32 outputs.
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        uint64_t marked = __ballot(vs[i] == 256);
                        while (marked) {
                            const int src = __builtin_ctzll(marked);
                            marked &= marked - 1;
                            const int unit = i * 64 + src;
                            if (j0 + unit / VT < limit)
                                row_nan |= 1u << (unit % VT * VU / 32);
                        }
                    }
                }
                if (tile + 4 < ntile)
                    load(tile + 4);

                float top = -INFINITY;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float v = s[h][e] * a.scale;
                        if (part_seen)
                            v = j0 + 16 * h + 4 * g + e < limit ? v : -INFINITY;
                        s[h][e] = v;
                        top = fmaxf(top, v);
                    }
                top = fmaxf(max_of_row(top), m);
                const float base = top == -INFINITY ? 0.0f : top;
                const float keep = __builtin_amdgcn_exp2f(m - base);   // 0 for the first keys
                m = top;
                float ps = 0.0f;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[h][e] = __builtin_amdgcn_exp2f(s[h][e] - base);
                        ps += s[h][e];
                    }
                l = l * keep + ps;
                const u32x4 p = {pack_bf16(s[0][0], s[0][1]), pack_bf16(s[0][2], s[0][3]),
                                 pack_bf16(s[1][0], s[1][1]), pack_bf16(s[1][2], s[1][3])};
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
                    const uint8_t *src = vt + (4 * g + (r16 >> 2)) * RS + f * 32 + (r16 & 3) * 8;
                    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)src);
                    const i16x4 hi =
                        __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(src + 16 * RS));
                    const u32x2 x = __builtin_bit_cast(u32x2, lo), y = __builtin_bit_cast(u32x2, hi);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[f][e] *= keep;
                    o[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        __builtin_bit_cast(bf16x8, u32x4{x[0], x[1], y[0], y[1]}),
                        __builtin_bit_cast(bf16x8, p), o[f], 0, 0, 0);
                }
            }
        }

        // Join the four wavefronts: row r16, outputs 16 f + 4 g + e.
        l = sum_of_row(l);
        if (g == 0) {
            row_m[wave][r16] = m;
            row_l[wave][r16] = l;
        }
        if (row_nan) {
#pragma unroll
            for (int f = 0; f < F; ++f)
                if (row_nan >> (f / 2) & 1)
                    o[f] = f32x4{NAN, NAN, NAN, NAN};
        }
        __syncthreads();
        float mm = -INFINITY, ll = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w)
            mm = fmaxf(mm, row_m[w][r16]);
        const float base = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
        for (int w = 0; w < 4; ++w)
            ll += row_l[w][r16] * __builtin_amdgcn_exp2f(row_m[w][r16] - base);
        const float mine = __builtin_amdgcn_exp2f(m - base);
        float *const os = reinterpret_cast<float *>(vt);
#pragma unroll
        for (int f = 0; f < F; ++f)
            *reinterpret_cast<f32x4 *>(os + r16 * D + f * 16 + g * 4) =
                f32x4{o[f][0] * mine, o[f][1] * mine, o[f][2] * mine, o[f][3] * mine};
        static_assert(16 * D * 4 <= 32 * RS, "a wavefront's O in its LDS rows");
        if (wave == 0 && g == 0) {
            all_m[r16] = mm;
            all_l[r16] = ll;
        }
        __syncthreads();
        constexpr int PER = D / 4;
        for (int i = threadIdx.x; i < 16 * PER; i += 256) {
            const int r = i / PER, d = i % PER * 4, rr = rt * kSplitRows + r;
            if (rr >= rows)
                break;
            f32x4 v = {};
#pragma unroll
            for (int w = 0; w < 4; ++w)
                v += *reinterpret_cast<const f32x4 *>(reinterpret_cast<float *>(lds[w]) + r * D + d);
            const int64_t out_row =
                (seq.q0 + rr / a.group) * q_heads + head * a.group + rr % a.group;
            if (used <= 1) {
                const float inv = all_l[r] == 0.0f ? 0.0f : 1.0f / all_l[r];
                *reinterpret_cast<u32x2 *>(a.out + out_row * D + d) =
                    u32x2{pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv)};
            } else {
                float *p = sp.part + (split * a.T * q_heads + out_row) * (D + 4);
                *reinterpret_cast<f32x4 *>(p + d) = v;
                if (d == 0) {
                    p[D] = all_m[r];
                    p[D + 1] = all_l[r];
                }
            }
        }
        __syncthreads();           // the next row tile writes the same LDS
    }
}

// Joins the splits of each row: weights 2^(m_s - max m).
template <int D>
__global__ void __launch_bounds__(256)
kv_attention_join_kernel(KvShape c, KvAttnArgs a, Split sp, int tile_rows) {
    constexpr int PER = D / 4;                 // lanes that hold a row's outputs
    constexpr int WAYS = 256 / PER;            // splits read side by side
    __shared__ float red[WAYS][D + 4];
    const int q_heads = c.heads * a.group;
    const int64_t out_row = blockIdx.x;
    const int64_t t = out_row / q_heads;
    const int h = (int)(out_row % q_heads);
    int b;
    if (a.q_starts) {
        int lo = 0, hi = a.seqs;               // the last sequence that starts at or before t
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (a.q_starts[mid] <= t)
                lo = mid;
            else
                hi = mid;
        }
        b = lo;
    } else {
        b = (int)(t / (a.T / a.seqs));
    }
    const Seq seq = sequence(c, a, b);
    const int row = (int)(t - seq.q0) * a.group + h % a.group;
    const int used = min(sp.splits, chunks_of(seq, row / tile_rows, tile_rows, a, sp.chunk));
    if (used <= 1)
        return;                                // its workgroup wrote the output
    const int64_t stride = a.T * q_heads * (D + 4);
    const float *p = sp.part + out_row * (D + 4);
    float m = -INFINITY;
    for (int s = threadIdx.x & 63; s < used; s += 64)
        m = fmaxf(m, p[s * stride + D]);
#pragma unroll
    for (int d = 32; d; d >>= 1)
        m = fmaxf(m, __shfl_xor(m, d));
    const float base = m == -INFINITY ? 0.0f : m;
    const int way = threadIdx.x / PER, d = threadIdx.x % PER * 4;
    f32x4 v = {};
    float l = 0.0f;
    if (way < WAYS)
        for (int s = way; s < used; s += WAYS) {
            const float w = __builtin_amdgcn_exp2f(p[s * stride + D] - base);
            l += w * p[s * stride + D + 1];
            const f32x4 x = *reinterpret_cast<const f32x4 *>(p + s * stride + d);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = __builtin_fmaf(w, x[e], v[e]);
        }
    if (way < WAYS) {
        *reinterpret_cast<f32x4 *>(&red[way][d]) = v;
        if (d == 0)
            red[way][D] = l;
    }
    __syncthreads();
    if (way == 0) {
#pragma unroll
        for (int w = 1; w < WAYS; ++w) {
            v += *reinterpret_cast<const f32x4 *>(&red[w][d]);
            l += red[w][D];
        }
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        *reinterpret_cast<u32x2 *>(a.out + out_row * D + d) =
            u32x2{pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv)};
    }
}

// Chunks: long enough that a partial result (4 (dim + 4) bytes a row) is little beside the
// keys and values it stands for, short enough to fill the card.
Split split_of(const KvShape &c, int64_t T, int seqs, int group, int max_q, int max_kv) {
    const int64_t tiles = ((int64_t)max_q * group + kSplitRows - 1) / kSplitRows;
    const int64_t total = (int64_t)seqs * c.heads * tiles * max_kv;
    int64_t chunk = (total / 4096 + 127) / 128 * 128;
    chunk = chunk < 512 ? 512 : chunk > kMaxChunk ? kMaxChunk : chunk;
    Split sp;
    sp.chunk = (int)chunk;
    sp.splits = (int)((max_kv + chunk - 1) / chunk);
    if (sp.splits < 1)
        sp.splits = 1;
    sp.part = nullptr;
    sp.magic = 0;
    return sp;
}

}  // namespace

size_t kv_attention_workspace_bytes(const KvShape &c, int64_t T, int seqs, int group, int max_q,
                                    int max_kv) {
    const Split sp = split_of(c, T, seqs, group, max_q, max_kv);
    return sp.splits == 1 ? 0 : (size_t)sp.splits * T * c.heads * group * (c.dim + 4) * 4;
}

hipError_t launch_kv_attention(const KvShape &c, const KvAttnArgs &a, void *ws, size_t,
                               hipStream_t s) {
    Split sp = split_of(c, a.T, a.seqs, a.group, a.max_q, a.max_kv);
    sp.part = static_cast<float *>(ws);
    const uint32_t pb = (uint32_t)c.page / 16;
    sp.magic = (((uint64_t)1 << 32) + pb - 1) / pb;
    const int64_t tiles = ((int64_t)a.max_q * a.group + kSplitRows - 1) / kSplitRows;
    const int64_t x = (int64_t)sp.splits * c.heads * a.seqs, rows = a.T * c.heads * a.group;
    if (x > 0x7FFFFFFF || rows > 0x7FFFFFFF)
        return hipErrorInvalidValue;
    const dim3 grid((unsigned)x, (unsigned)(tiles > 65535 ? 65535 : tiles));
    const auto go = [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        if (c.fmt == KV_FP8)
            hipLaunchKernelGGL((kv_attention_split_kernel<KV_FP8, D>), grid, dim3(256), 0, s, c, a, sp);
        else
            hipLaunchKernelGGL((kv_attention_split_kernel<KV_FP4, D>), grid, dim3(256), 0, s, c, a, sp);
        if (sp.splits > 1)
            hipLaunchKernelGGL((kv_attention_join_kernel<D>), dim3((unsigned)rows), dim3(256), 0, s, c,
                               a, sp, kSplitRows);
        return hipGetLastError();
    };
    switch (c.dim) {
    case 64: return go(std::integral_constant<int, 64>{});
    case 128: return go(std::integral_constant<int, 128>{});
    case 192: return go(std::integral_constant<int, 192>{});
    default: return go(std::integral_constant<int, 256>{});
    }
}

}  // namespace w8a8
