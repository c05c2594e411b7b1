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
// weights are rounded for the second product: to two bf16 terms (2^-16 of each at most) in sequences
// of few rows, to one (2^-8) in those of many, whose products bind. Each sequence gets the kernel
// for its own rows, so that its rounding does not hang on the batch or on the caller's bounds.
#include "../../include/w8a8.h"
#include "mx_internal.hpp"
#include "mx_math.hpp"
#include "quant_math.hpp"

#include <algorithm>

namespace w8a8 {
namespace {

using namespace mx;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// How the keys of a launch are divided: a workgroup's share is `share` tokens (a multiple of
// 128), or what the lengths make of `target` if that is more, or what divides a sequence's tokens
// among `splits` workgroups, the most that a head and row tile of it can have, if that is more.
struct Split {
    int rows_from, rows_to;   // sequences of this many rows (queries x group) are this kernel's
    int share, splits;
    int target;      // workgroups that the tokens of all sequences are spread over, 0: share holds
    float *part;     // joined: [splits][T * q heads][dim + 4]: O, m, l; in split 0 the number
                     // of splits the row has (1: its output is written already)
    bool joined;     // a launch that joins partial results follows
    uint64_t magic;  // n / (page / 16) = n * magic >> 32 for n < 2^22 (kMaxTokens / 16)
};

// The maximum that exponents are taken from may lag behind by this much: O and l are rescaled
// only when a row's maximum rises further. Weights up to 2^8 instead of 1 lose nothing, as
// float32 sums and bf16 roundings are relative; a rescaling costs as much as a product. 4 x 1000
// queries on 6000 keys, 18 heads of 256: 783 us rescaling at every rise, 670 so.
constexpr float kSlack = 8.0f;
constexpr int kMaxChunk = 4096;
constexpr int kSplitRows = 16, kTileRows = 128, kTileTokens = 64;
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

__device__ __forceinline__ bool mine(const Split &sp, int rows) {
    return rows >= sp.rows_from && rows <= sp.rows_to;
}

// The share for this call's lengths: their tokens (once a head and row tile) spread evenly,
// whatever each sequence has of them. A wavefront sums them by itself, in the same order in
// every workgroup.
__device__ __forceinline__ int share_of(const KvShape &c, const KvAttnArgs &a, const Split &sp, int rows) {
    if (sp.target == 0)
        return sp.share;
    float sum = 0.0f;
    for (int i = threadIdx.x & 63; i < a.seqs; i += 64) {
        const Seq s = sequence(c, a, i);
        if (mine(sp, s.lq * a.group))
            sum += (float)max(s.kv, 0) * (float)((s.lq * a.group + rows - 1) / rows);
    }
#pragma unroll
    for (int d = 32; d > 0; d /= 2)
        sum += __shfl_xor(sum, d);
    const float even = fminf(sum * (float)c.heads / (float)sp.target, (float)W8A8_KV_MAX_TOKENS);
    return __builtin_amdgcn_readfirstlane(max(((int)even + 127) & ~127, sp.share));
}

// Its equal pieces, for which Places has room.
__device__ __forceinline__ int chunk_of(int share) {
    const int pieces = (share + kMaxChunk - 1) / kMaxChunk;
    return ((share + pieces - 1) / pieces + 127) & ~127;
}

// A row's maximum before its first key: minus infinity where it sees none, else the least finite
// number. A sum of zero then tells a row without keys (zeros) from one all of whose scores are
// minus infinity, as a query with an infinity has them (NaN, as exp(-inf - -inf) is).
__device__ __forceinline__ float start_of(int limit) { return limit > 0 ? -__FLT_MAX__ : -INFINITY; }

__device__ __forceinline__ float inverse(float l, float m) {
    return l == 0.0f ? (m == -INFINITY ? 0.0f : NAN) : 1.0f / l;
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

// An operand of ones: products with it sum the weights on the matrix cores.
__device__ __forceinline__ bf16x8 ones() {
    return __builtin_bit_cast(bf16x8, u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
}

// In a branch that few tiles take: without it the compiler computes both sides in every tile.
__device__ __forceinline__ void keep_branch() { asm volatile(""); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)lo, (__bf16)hi});
}

// Four neighbouring outputs: v times inv. bf16 tensors may begin at any element.
__device__ __forceinline__ void store_outputs(uint16_t *out, const f32x4 &v, float inv) {
    *reinterpret_cast<Bytes8 *>(out) =
        Bytes8{{pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv)}};
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

// Where the tokens of a chunk lie, 16 at a time: the first one's place in its page, and the
// page's keys of the head, from which its codes, scales and values follow.
struct Places {
    int64_t page[kMaxChunk / 16];
    int at[kMaxChunk / 16];
};

// Fills `count` entries from token j_first on; those past token j_end - 1 repeat its block.
__device__ __forceinline__ void fill_places(Places &pl, const KvShape &c, const KvAttnArgs &a,
                                            const Split &sp, int b, int head, int j_first, int j_end,
                                            int count) {
    const uint32_t last = (uint32_t)(j_end - 1) / 16;
    const int32_t *table = a.table + b * a.table_stride;
    for (int i = threadIdx.x; i < count; i += 256) {
        const uint32_t blk = min((uint32_t)(j_first / 16 + i), last);
        const uint32_t entry = (uint32_t)(blk * sp.magic >> 32);
        const int64_t page = min((int64_t)max(table[entry], 0), c.pages - 1);
        pl.page[i] = (page * 2 * c.heads + head) * c.head_bytes();
        pl.at[i] = (int)(blk - entry * (uint32_t)(c.page / 16)) * 16;
    }
}

// Few rows (16 a workgroup): the keys are divided among workgroups, and among the four
// wavefronts of each in tiles of 32 tokens; every wavefront keeps its own m, l and O, joined
// in LDS at the end. Keys go from memory to the matrix registers as they are: lane (t, g) =
// (lane % 16, lane / 16) holds of token t the elements whose unit number is g modulo 4, and Q
// is loaded in the same order. Values pass through the wavefront's own piece of LDS, decoded,
// and come back transposed. The next tile's codes are loaded while this one is worked on.
//
// Bound by reading the cache: 4 sequences of 100000 tokens (8 heads of 128, e4m3, 4 queries a
// head) at 5.4 TB/s, 16 of 8000 with 18 heads of 256 at 5.6; one of 200000 in e2m1, 8 queries a
// head, at 4.6 (about 370 instructions for 32 tokens of 4.3 KB); 48 sequences of very different
// lengths at 4.0 (unequal shares, more workgroups that start).
template <int FMT, int D>
__global__ void __launch_bounds__(256, D <= 128 ? 3 : 2)
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
    __shared__ Places places;
    __shared__ float row_m[4][16], row_l[4][16], all_l[16], all_m[16];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, g = lane >> 4;
    // Heads fastest, splits slowest: every 8th workgroup goes to one XCD, and the last splits
    // of short sequences are empty; with splits fastest one XCD can get all the full ones.
    const int pairs = c.heads * a.seqs;
    const int split = __builtin_amdgcn_readfirstlane(blockIdx.x / pairs);
    const int pair = blockIdx.x - split * pairs;
    const int b = __builtin_amdgcn_readfirstlane(pair / c.heads), head = pair - b * c.heads;
    const Seq seq = sequence(c, a, b);
    const int rows = seq.lq * a.group, q_heads = c.heads * a.group;
    if (!mine(sp, rows) || (split > 0 && (int64_t)split * sp.share >= seq.kv))
        return;                            // shares are this long or longer
    const int even = share_of(c, a, sp, kSplitRows);
    const int64_t v_offset = c.heads * c.head_bytes();     // from a page's keys to its values
    const int scales_at = c.page * CB;                     // from codes to scales
    uint8_t *const vt = lds[wave];

    for (int rt = blockIdx.y; rt * kSplitRows < rows; rt += gridDim.y) {
        const int some_see =
            seen(seq, (min(rt * kSplitRows + kSplitRows, rows) - 1) / a.group, a.causal);   // some row
        const int share = max(even, ((some_see + sp.splits - 1) / sp.splits + 127) & ~127);
        const int used = (some_see + share - 1) / share;
        if (split >= max(used, 1))
            continue;
        const int chunk = chunk_of(share), nch = (some_see + chunk - 1) / chunk;
        const int row = rt * kSplitRows + r16;
        const bool live = row < rows;
        const int qi = live ? row / a.group : 0;
        const int qh = head * a.group + (live ? row % a.group : 0);
        const int limit = live ? seen(seq, qi, a.causal) : 0;
        const int all_see = seen(seq, rt * kSplitRows / a.group, a.causal);   // every live row
        u32x4 q[NK][KU / 8];
        {
            const uint16_t *src = a.q + (seq.q0 + qi) * a.q_token + qh * a.q_head;
#pragma unroll
            for (int s = 0; s < NK; ++s)
#pragma unroll
                for (int e = 0; e < KU / 8; ++e) {
                    const Bytes16 v =
                        *reinterpret_cast<const Bytes16 *>(src + (4 * s + g) * KU + 8 * e);
                    q[s][e] = live ? u32x4{v.w[0], v.w[1], v.w[2], v.w[3]} ^ a.q_sign : u32x4{};
                }
        }
        f32x4 o[F];
#pragma unroll
        for (int f = 0; f < F; ++f)
            o[f] = f32x4{};
        float m = start_of(limit);
        f32x4 sums = {};           // in each element: the sum of a row's weights
        uint32_t row_nan = 0;      // blocks of the row's output that a seen NaN value reaches

        for (int ch = split; ch < nch; ch += used) {
            const int j_first = ch * chunk;
            const int j_end = min(j_first + chunk, some_see);
            const int ntile = (j_end - j_first + 31) / 32;
            __syncthreads();       // the places and the LDS rows of what came before are read
            fill_places(places, c, a, sp, b, head, j_first, j_end, 2 * ntile);
            __syncthreads();

            u32x4 kc[2][NK], vc[NV];
            uint32_t ks[2][NK], vs[NV];
            const auto load = [&](int tile) {
                const uint8_t *page[2];
                int at[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint64_t p = places.page[2 * tile + h];
                    page[h] = a.cache + (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)p) +
                              ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(p >> 32)) << 32);
                    at[h] = __builtin_amdgcn_readfirstlane(places.at[2 * tile + h]);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int s = 0; s < NK; ++s) {
                        kc[h][s] =
                            Unit<KB>::load(page[h] + (uint32_t)((at[h] + r16) * CB + (4 * s + g) * KB));
                        ks[h][s] = page[h][(uint32_t)(scales_at + (at[h] + r16) * (D / 32) +
                                                      (4 * s + g) * KU / 32)];
                    }
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int unit = i * 64 + lane, tok = unit / VT, part = unit % VT;
                    // NV even: an instruction's tokens lie in one half of the tile
                    constexpr bool EVEN = NV % 2 == 0;
                    const int h = EVEN ? 2 * i / NV : 0;
                    const uint8_t *p = EVEN || tok < 16 ? page[h] : page[1];
                    const int in = EVEN ? at[h] + tok - 16 * h
                                        : tok < 16 ? at[0] + tok : at[1] + tok - 16;
                    p += v_offset;
                    vc[i] = Unit<16>::load(p + (uint32_t)(in * CB + part * 16));
                    vs[i] = p[(uint32_t)(scales_at + in * (D / 32) + part * VU / 32)];
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
                        keep_branch();
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

                if (part_seen) {
                    const int left = limit - j0 - 4 * g;
                    keep_branch();
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            s[h][e] = 16 * h + e < left ? s[h][e] : -INFINITY;
                }
                float top = -INFINITY;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        top = fmaxf(top, s[h][e]);
                top = fmaxf(max_of_row(top) * a.scale, m);
                if (__any(top > m + kSlack)) {
                    keep_branch();
                    const float keep =
                        __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.0f : top));
                    sums[0] *= keep;           // the only one that is used
#pragma unroll
                    for (int f = 0; f < F; ++f)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            o[f][e] *= keep;
                    m = top;
                }
                const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s[h][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][e], a.scale, -base));
                // The weights in two bf16 terms, 16 bits in all: the products are few here.
                u32x4 p, p2;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = s[i / 2][i % 2 * 2], y = s[i / 2][i % 2 * 2 + 1];
                    p[i] = pack_bf16(x, y);
                    p2[i] = pack_bf16(x - __uint_as_float(p[i] << 16),
                                      y - __uint_as_float(p[i] & 0xFFFF0000u));
                }
                sums = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    ones(), __builtin_bit_cast(bf16x8, p), sums, 0, 0, 0);
                sums = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    ones(), __builtin_bit_cast(bf16x8, p2), sums, 0, 0, 0);
#pragma unroll
                for (int f = 0; f < F; ++f) {
                    typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
                    const uint8_t *src = vt + (4 * g + (r16 >> 2)) * RS + f * 32 + (r16 & 3) * 8;
                    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)src);
                    const i16x4 hi =
                        __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(src + 16 * RS));
                    const u32x2 x = __builtin_bit_cast(u32x2, lo), y = __builtin_bit_cast(u32x2, hi);
                    const bf16x8 v = __builtin_bit_cast(bf16x8, u32x4{x[0], x[1], y[0], y[1]});
                    o[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8, p), o[f],
                                                                   0, 0, 0);
                    o[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8, p2), o[f],
                                                                   0, 0, 0);
                }
            }
        }

        // Join the four wavefronts: row r16, outputs 16 f + 4 g + e.
        const float l = sums[0];
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
                const float inv = inverse(all_l[r], all_m[r]);
                store_outputs(a.out + out_row * D + d, v, inv);
            } else {
                float *p = sp.part + (split * a.T * q_heads + out_row) * (D + 4);
                *reinterpret_cast<f32x4 *>(p + d) = v;
                if (d == 0) {
                    p[D] = all_m[r];
                    p[D + 1] = all_l[r];
                }
            }
            if (d == 0 && split == 0 && sp.joined)
                sp.part[out_row * (D + 4) + D + 2] = (float)used;
        }
        __syncthreads();           // the next row tile writes the same LDS
    }
}

// Barrier that orders LDS only: loads from memory stay in flight across it.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The other half's value beside this one's: lanes l and l ^ 32 hold the same row.
__device__ __forceinline__ u32x2 both_halves(float v) {
    return __builtin_bit_cast(
        u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
}

// Many rows (128 a workgroup, 32 a wavefront): 64 tokens at a time are decoded once into LDS
// for all four wavefronts, between the products of the 64 before; 32x32x16 products with the
// rows as columns, as above. Keys lie in rows of 2 D + 16 bytes, values in rows of 2 D + 64, which
// spreads the fragment reads (32 keys x 16 bytes; 4 values x 64 bytes) over the banks. Still a
// quarter of the LDS cycles at heads of 256 are conflicts, by the counters: the likely ones are the
// staging's 16-byte stores, whose neighbouring lanes write 32 bytes apart.
//
// Bound by instructions: per row and 64 tokens 64 exponentials and some 350 other vector
// instructions a wavefront beside 64 (heads of 256) or 32 (128) products, two wavefronts a SIMD
// for heads of up to 128, one above (O and Q alone take 192 registers). 4 x 1000 queries on
// 6000 keys, causal: 32 heads of 128 at 950 TFLOP/s, 18 heads of 256 at 610; 8 x 512 on 4000,
// 32 heads of 64 at 720. Staging whole tiles between barriers, before it was spread over the
// products, cost a third of the time at heads of 256.
//
// Workgroup -> problem: every 8th workgroup goes to one XCD; a split of a key/value head of a
// sequence is given to one XCD with all its row tiles, the last ones (which see the most keys)
// first, so that its L2 holds the keys. Fewer than kSpreadUnits of them would leave XCDs idle:
// their row tiles go to all XCDs. 4 x 1000 queries on 6000 keys take 713 us at 18 heads of 256
// and 405 at 8 of 128 (4 queries a head) where neighbours in the grid are neighbouring row
// tiles, 670 and 382 so.
constexpr int kSpreadUnits = 32;

template <int FMT, int D>
__global__ void __launch_bounds__(256, D <= 128 ? 2 : 1)
kv_attention_tile_kernel(KvShape c, KvAttnArgs a, Split sp, int tiles) {
    constexpr int TT = kTileTokens;
    constexpr int VU = FMT == KV_FP8 ? 16 : 32;        // a unit: 16 bytes of codes
    constexpr int VT = D / VU, UNITS = TT * VT, NU = (UNITS + 255) / 256;
    constexpr int CB = FMT == KV_FP8 ? D : D / 2;
    constexpr int RSK = 2 * D + 16, RSV = 2 * D + 64;
    constexpr int KS = D / 16, F = D / 32;
    // Two stages: a tile is staged while the one before it is multiplied.
    __shared__ __attribute__((aligned(16))) uint8_t keys[2][TT * RSK];
    __shared__ __attribute__((aligned(16))) uint8_t values[2][TT * RSV];
    __shared__ Places places;
    __shared__ uint8_t nan_unit[2][UNITS];
    __shared__ int nan_any;

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r32 = lane & 31, h = lane >> 5;
    const int pairs = a.seqs * c.heads, units = pairs * sp.splits;
    int unit, in;                          // head of a sequence and split; row tile from the end
    if (units >= kSpreadUnits) {
        const int slot = blockIdx.x >> 3;
        unit = __builtin_amdgcn_readfirstlane(slot / tiles);
        in = slot - unit * tiles;
        unit = unit * 8 + (blockIdx.x & 7);
        if (unit >= units)
            return;
    } else {
        unit = __builtin_amdgcn_readfirstlane(blockIdx.x / tiles);
        in = blockIdx.x - unit * tiles;
    }
    const int split = __builtin_amdgcn_readfirstlane(unit / pairs), pair = unit - split * pairs;
    const int b = __builtin_amdgcn_readfirstlane(pair / c.heads), head = pair - b * c.heads;
    const Seq seq = sequence(c, a, b);
    const int rows = seq.lq * a.group, q_heads = c.heads * a.group;
    if (!mine(sp, rows) || (split > 0 && (int64_t)split * sp.share >= seq.kv))
        return;                            // shares are this long or longer
    const int even = share_of(c, a, sp, kTileRows);
    const int64_t v_offset = c.heads * c.head_bytes();

    const int first_rt = tiles - 1 - in;
    const int last_rt = (rows + kTileRows - 1) / kTileRows - 1;
    // Row tiles first_rt, first_rt + tiles, ...: more than one only where the grid has fewer.
    for (int rt = first_rt; rt <= last_rt; rt += tiles) {
        const int some_see =
            seen(seq, (min(rt * kTileRows + kTileRows, rows) - 1) / a.group, a.causal);   // some row
        const int share = max(even, ((some_see + sp.splits - 1) / sp.splits + 127) & ~127);
        const int used = (some_see + share - 1) / share;
        if (split >= max(used, 1))
            continue;
        const int chunk = chunk_of(share), nch = (some_see + chunk - 1) / chunk;
        const int row = rt * kTileRows + wave * 32 + r32;
        const bool live = row < rows;
        const int qi = live ? row / a.group : 0;
        const int qh = head * a.group + (live ? row - qi * a.group : 0);
        const int limit = live ? seen(seq, qi, a.causal) : 0;
        const int all_see = seen(seq, rt * kTileRows / a.group, a.causal);
        // what some row of this wavefront sees
        const int wave_first = rt * kTileRows + wave * 32;
        const int wave_sees =
            wave_first < rows ? seen(seq, (min(wave_first + 32, rows) - 1) / a.group, a.causal) : 0;
        u32x4 q[KS];
        {
            const uint16_t *src = a.q + (seq.q0 + qi) * a.q_token + qh * a.q_head + 8 * h;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const Bytes16 v = *reinterpret_cast<const Bytes16 *>(src + 16 * s);
                q[s] = live ? u32x4{v.w[0], v.w[1], v.w[2], v.w[3]} ^ a.q_sign : u32x4{};
            }
        }
        f32x16 o[F];
#pragma unroll
        for (int f = 0; f < F; ++f)
            o[f] = f32x16{};
        float m = start_of(limit), l = 0.0f;
        uint32_t row_nan = 0;

        for (int ch = split; ch < nch; ch += used) {
            const int j_first = ch * chunk;
            const int j_end = min(j_first + chunk, some_see);
            const int ntile = (j_end - j_first + TT - 1) / TT;
            __syncthreads();
            if (threadIdx.x == 0)
                nan_any = 0;
            fill_places(places, c, a, sp, b, head, j_first, j_end, ntile * (TT / 16));
            __syncthreads();

            u32x4 kc[NU], vc[NU];
            uint32_t ks[NU], vs[NU];
            const auto load = [&](auto ic, int tile) __attribute__((always_inline)) {
                constexpr int i = decltype(ic)::value;
                const int unit = min(i * 256 + (int)threadIdx.x, UNITS - 1);
                const int tok = unit / VT, part = unit % VT;
                const int blk = tile * (TT / 16) + tok / 16;
                const int at = places.at[blk] + tok % 16;
                const uint8_t *p = a.cache + places.page[blk];
                const uint32_t code = at * CB + part * 16;
                const uint32_t scale = c.page * CB + at * (D / 32) + part * VU / 32;
                kc[i] = Unit<16>::load(p + code);
                ks[i] = p[scale];
                vc[i] = Unit<16>::load(p + v_offset + code);
                vs[i] = p[v_offset + scale];
            };
            const auto load_all = [&](int tile) {
                [&]<int... i>(std::integer_sequence<int, i...>) __attribute__((always_inline)) {
                    (load(std::integral_constant<int, i>{}, tile), ...);
                }(std::make_integer_sequence<int, NU>{});
            };
            // Values past the end, and NaN blocks in tiles that only some rows see whole, become
            // zeros before they are staged (a zero weight would not silence them).
            const auto mark = [&](int j0, int st) {
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    const int unit = min(i * 256 + (int)threadIdx.x, UNITS - 1);
                    const bool past = j0 + unit / VT >= seq.kv;
                    const bool nan = vs[i] == kNaNScale && !past;
                    nan_unit[st][unit] = nan;
                    if (nan)
                        nan_any = 1;
                    if (past || nan) {
                        vc[i] = u32x4{};
                        vs[i] = 0;
                    }
                }
            };
            // Half z of 4 NU half units into stage st: keys, then values.
            const auto stage = [&](auto zc, int st) __attribute__((always_inline)) {
                constexpr int z = decltype(zc)::value / 2, half = decltype(zc)::value % 2, i = z % NU;
                const int unit = i * 256 + threadIdx.x, tok = unit / VT, part = unit % VT;
                if (UNITS % 256 != 0 && unit >= UNITS)
                    return;
                const u32x4 codes = z < NU ? kc[i] : vc[i];
                const float sc = scale_operand(z < NU ? ks[i] : vs[i]);
                u32x4 *d = reinterpret_cast<u32x4 *>(
                    (z < NU ? keys[st] + tok * RSK : values[st] + tok * RSV) + part * VU * 2);
                if constexpr (VU == 16) {
                    d[half] = decode_part<FMT, half>(codes, sc);
                } else {
                    d[2 * half] = decode_part<FMT, 2 * half>(codes, sc);
                    d[2 * half + 1] = decode_part<FMT, 2 * half + 1>(codes, sc);
                }
            };
            const auto partly_seen = [&](int j0) { return j0 + TT > all_see; };
            load_all(0);
            if (partly_seen(j_first))
                mark(j_first, 0);
            [&]<int... z>(std::integer_sequence<int, z...>) __attribute__((always_inline)) {
                (stage(std::integral_constant<int, z>{}, 0), ...);
            }(std::make_integer_sequence<int, 4 * NU>{});
            load_all(min(1, ntile - 1));
            for (int tile = 0; tile < ntile; ++tile) {
                const int j0 = j_first + tile * TT, st = tile & 1;
                const bool part_seen = partly_seen(j0);
                lds_barrier();       // this tile is staged, the other stage's last one is read
                if (partly_seen(j0 + TT) && tile + 1 < ntile)
                    mark(j0 + TT, st ^ 1);
                if (part_seen && nan_any)      // rare: which rows see a NaN block
                    for (int unit = 0; unit < UNITS; ++unit)
                        if (nan_unit[st][unit] && j0 + unit / VT < limit)
                            row_nan |= 1u << (unit % VT * VU / 32);
                // Scores: token 32 t + 8 (i / 4) + 4 h + i % 4 in s[t][i]. Between the products
                // the next tile is staged (after the last tile: itself again, unread).
                f32x16 s[2] = {f32x16{}, f32x16{}};
                const uint8_t *kp = keys[st] + r32 * RSK + h * 16;
                bf16x8 fk[2][2];
                const auto read_keys = [&](int k) __attribute__((always_inline)) {
                    fk[k & 1][0] = *reinterpret_cast<const bf16x8 *>(kp + k * 32);
                    fk[k & 1][1] = *reinterpret_cast<const bf16x8 *>(kp + 32 * RSK + k * 32);
                };
                read_keys(0);
                [&]<int... k>(std::integer_sequence<int, k...>) __attribute__((always_inline)) {
                    ([&]() __attribute__((always_inline)) {
                        if constexpr (k + 1 < KS)
                            read_keys(k + 1);
                        constexpr int z0 = k * 4 * NU / KS, z1 = (k + 1) * 4 * NU / KS;
                        if constexpr (z0 < z1)
                            stage(std::integral_constant<int, z0>{}, st ^ 1);
                        static_assert(z1 - z0 <= 1, "half units of a step");
                        __builtin_amdgcn_sched_barrier(0);
                        s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            fk[k & 1][0], __builtin_bit_cast(bf16x8, q[k]), s[0], 0, 0, 0);
                        s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            fk[k & 1][1], __builtin_bit_cast(bf16x8, q[k]), s[1], 0, 0, 0);
                        __builtin_amdgcn_sched_barrier(0);
                    }(), ...);
                }(std::make_integer_sequence<int, KS>{});
                // The next loads go out between the products with the values.
                if (j0 >= wave_sees) {
                    load_all(min(tile + 2, ntile - 1));
                    continue;
                }

                if (part_seen) {
                    const int left = limit - j0 - 4 * h;
                    keep_branch();
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            s[t][i] = 32 * t + 8 * (i / 4) + i % 4 < left ? s[t][i] : -INFINITY;
                }
                float top = -INFINITY;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        top = fmaxf(top, s[t][i]);
                const u32x2 tops = both_halves(top);
                top = fmaxf(fmaxf(__uint_as_float(tops[0]), __uint_as_float(tops[1])) * a.scale, m);
                if (__any(top > m + kSlack)) {
                    keep_branch();
                    const float keep =
                        __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.0f : top));
                    l *= keep;
#pragma unroll
                    for (int f = 0; f < F; ++f)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            o[f][i] *= keep;
                    m = top;
                }
                const float base = m == -INFINITY ? 0.0f : m;
                // Values: step u of 16 tokens, half h takes tokens 4h + 0 .. 3 and 8 + 4h +
                // 0 .. 3. The weights of step u + 1 are computed between the products of step u.
                typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
                const uint8_t *vp = values[st] + (4 * h + ((lane & 15) >> 2)) * RSV +
                                    ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
                u32x2 fv[2][2];
                const auto read_values = [&](int z) __attribute__((always_inline)) {
                    const uint8_t *src = vp + 16 * (z / F) * RSV + z % F * 64;
                    fv[z & 1][0] = __builtin_bit_cast(
                        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)src));
                    fv[z & 1][1] = __builtin_bit_cast(
                        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(src + 8 * RSV)));
                };
                u32x4 p[4];
                const auto weight = [&](auto qc) __attribute__((always_inline)) {
                    constexpr int w = decltype(qc)::value;     // of 16 pairs
                    const float x = __builtin_amdgcn_exp2f(
                        __builtin_fmaf(s[w / 8][w % 8 * 2], a.scale, -base));
                    const float y = __builtin_amdgcn_exp2f(
                        __builtin_fmaf(s[w / 8][w % 8 * 2 + 1], a.scale, -base));
                    l += x + y;
                    p[w / 4][w % 4] = pack_bf16(x, y);
                };
                weight(std::integral_constant<int, 0>{});
                weight(std::integral_constant<int, 1>{});
                weight(std::integral_constant<int, 2>{});
                weight(std::integral_constant<int, 3>{});
                read_values(0);
                [&]<int... z>(std::integer_sequence<int, z...>) __attribute__((always_inline)) {
                    ([&]() __attribute__((always_inline)) {
                        constexpr int u = z / F, f = z % F;
                        if constexpr (z + 1 < 4 * F)
                            read_values(z + 1);
                        if constexpr (u < 3) {
                            constexpr int w0 = 4 * (u + 1) + f * 4 / F, w1 = 4 * (u + 1) + (f + 1) * 4 / F;
                            if constexpr (w0 < w1)
                                weight(std::integral_constant<int, w0>{});
                            if constexpr (w0 + 1 < w1)
                                weight(std::integral_constant<int, w0 + 1>{});
                        }
                        if constexpr (z < 2 * NU && z % 2 == 1)
                            load(std::integral_constant<int, z / 2>{}, min(tile + 2, ntile - 1));
                        static_assert(2 * NU <= 4 * F, "loads between the products");
                        __builtin_amdgcn_sched_barrier(0);
                        o[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            __builtin_bit_cast(bf16x8, u32x4{fv[z & 1][0][0], fv[z & 1][0][1],
                                                             fv[z & 1][1][0], fv[z & 1][1][1]}),
                            __builtin_bit_cast(bf16x8, p[u]), o[f], 0, 0, 0);
                        __builtin_amdgcn_sched_barrier(0);
                    }(), ...);
                }(std::make_integer_sequence<int, 4 * F>{});
            }
        }

        const u32x2 ls = both_halves(l);
        l = __uint_as_float(ls[0]) + __uint_as_float(ls[1]);
        if (!live)
            continue;        // the next row tile's barriers are reached all the same
        const int64_t out_row = (seq.q0 + qi) * q_heads + qh;
        const float inv = inverse(l, m);
        float *const part = sp.part + (split * a.T * q_heads + out_row) * (D + 4);
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const bool nan = row_nan >> f & 1;
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int d = 32 * f + 2 * i + 4 * h;
                f32x4 v = {o[f][i], o[f][i + 1], o[f][i + 2], o[f][i + 3]};
                if (nan)
                    v = f32x4{NAN, NAN, NAN, NAN};
                if (used <= 1)
                    store_outputs(a.out + out_row * D + d, v, inv);
                else
                    *reinterpret_cast<f32x4 *>(part + d) = v;
            }
        }
        if (used > 1 && h == 0) {
            part[D] = m;
            part[D + 1] = l;
        }
        if (split == 0 && sp.joined && h == 0)
            part[D + 2] = (float)used;
    }
}

// Joins the splits of each row with weights 2^(m_s - max m): LANES lanes hold 4 outputs each of
// a row (or of 4 LANES of its outputs), WAYS groups of them take the splits in turn.
template <int D, int LANES, int WAYS>
__global__ void __launch_bounds__(256)
kv_attention_join_kernel(const float *part, int splits, int64_t rows, uint16_t *out) {
    constexpr int PIECES = D / (4 * LANES), PER = LANES * WAYS, JOBS = 256 / PER;
    __shared__ f32x4 red[JOBS][WAYS][LANES];
    __shared__ float red_l[JOBS][WAYS], red_m[JOBS][WAYS];
    const int job = threadIdx.x / PER, in = threadIdx.x % PER, way = in / LANES;
    const int64_t id = (int64_t)blockIdx.x * JOBS + job, row = id / PIECES;
    const int d = (int)(id % PIECES) * (4 * LANES) + in % LANES * 4;
    const bool live = job < JOBS && row < rows;
    const float *p = part + (live ? row : 0) * (D + 4);
    const int64_t stride = rows * (D + 4);
    const int used = live ? min((int)p[D + 2], splits) : 0;
    float m = -INFINITY, l = 0.0f;
    f32x4 v = {};
    if (used > 1) {
        for (int s = way; s < used; s += WAYS) {
            const float mm = p[s * stride + D], ll = p[s * stride + D + 1];
            const f32x4 x = *reinterpret_cast<const f32x4 *>(p + s * stride + d);
            const float top = fmaxf(m, mm), base = top == -INFINITY ? 0.0f : top;
            const float keep = __builtin_amdgcn_exp2f(m - base), w = __builtin_amdgcn_exp2f(mm - base);
            m = top;
            l = l * keep + ll * w;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = v[e] * keep + x[e] * w;
        }
    }
    if constexpr (WAYS > 1) {
        if (live) {
            red[job][way][in % LANES] = v;
            if (in % LANES == 0) {
                red_l[job][way] = l;
                red_m[job][way] = m;
            }
        }
        __syncthreads();
        if (way > 0 || used <= 1)
            return;
        float top = m;
#pragma unroll
        for (int w = 1; w < WAYS; ++w)
            top = fmaxf(top, red_m[job][w]);
        const float base = top == -INFINITY ? 0.0f : top, mine = __builtin_amdgcn_exp2f(m - base);
        l *= mine;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] *= mine;
#pragma unroll
        for (int w = 1; w < WAYS; ++w) {
            const float f = __builtin_amdgcn_exp2f(red_m[job][w] - base);
            const f32x4 x = red[job][w][in % LANES];
            l += red_l[job][w] * f;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] += x[e] * f;
        }
    }
    if (used > 1) {
        const float inv = inverse(l, m);
        store_outputs(out + row * D + d, v, inv);
    }
}

template <int D, int LANES, int WAYS>
hipError_t launch_join(const float *part, int splits, int64_t rows, uint16_t *out, hipStream_t s) {
    constexpr int jobs = 256 / (LANES * WAYS), pieces = D / (4 * LANES);
    const int64_t blocks = (rows * pieces + jobs - 1) / jobs;
    if (!launchable(blocks, 256))
        return hipErrorInvalidValue;
    hipLaunchKernelGGL((kv_attention_join_kernel<D, LANES, WAYS>), dim3((unsigned)blocks), dim3(256), 0, s,
                       part, splits, rows, out);
    return hipGetLastError();
}

// Up to this many rows of a sequence are few: the split kernel's, whose weights have two terms. The
// tile kernel decodes keys and values once for 128 rows, that one once for 16. Its time by the
// tile kernel's, 1800 random shapes of a sequence and head, e4m3 and e2m1: 17 to 32 rows 0.86,
// 0.75; 33 to 48 0.96, 0.82; 49 to 64 1.04, 0.94. Where heads and sequences alone fill the card its
// instructions bind and the tile kernel, with its one term, would be faster from 33 rows on (32 x
// 8 heads of 128, 16000 keys: e4m3, 48 rows 493 and 270 us, 56 rows 671 and 270; e2m1, 56 rows
// 342 and 243); a query's rounding is not to hang on the batch that it comes in.
constexpr int kFewRows = 64;

// Most rows of a sequence that each kernel gets, 0: not launched. Where sequences may be of both
// kinds both run, one after the other, and each takes those of its own. 8 heads of 128, 4 queries a
// head, 100 queries on 4000 keys with 63 sequences of one on up to 8000: 202 us, all by the tile
// kernel 441; 2000 with 15 of one 158 and 278. The one without sequences takes 1 to 2 us where the
// call is small and 12 at 4 x 1000 queries of 18 heads of 256 (660).
struct Rows {
    int64_t few, many;
};

Rows rows_of(int64_t T, int seqs, int group, int max_q) {
    const int64_t rows = (seqs == 1 ? T : std::min<int64_t>(max_q, T)) * group;
    if (rows <= kFewRows)
        return {rows, 0};
    return {seqs == 1 || (int64_t)max_q * seqs == T ? 0 : kFewRows, rows};
}

// Up to here one workgroup takes all keys: a second launch costs as much. us divided and whole, 8
// heads of 128, 4 queries a head: 300 keys 9.7, 8.6; 500 9.8, 9.8; 700 10.0, 11.9.
constexpr int kWholeTokens = 512;
// Workgroups of a launch of many rows. Most are empty where max_q is loose or one sequence long,
// and an empty one still takes its turn; too few, and a long sequence's row tiles queue up. us with
// 2^16, 2^18 and 2^20, 8 heads of 128, 4 queries a head: 64 x 1000 queries, max_q left out 820, 1004,
// 1772 (809 with it); 4000 queries beside 2000 sequences of one 1622, 608, 1340.
constexpr int64_t kMostGroups = 1 << 18;
// Sequences whose lengths a wavefront sums, 64 at a time, at the start of every workgroup.
constexpr int kSummed = 512;

// How the keys are divided. A partial result is 4 (dim + 4) bytes a row to write and to read, and
// a workgroup takes some microseconds to start, so only as many as fill the card: 512 workgroups
// of few rows, one of many rows a CU (1.5 up to 128 wide heads, where two share one); on 1055
// random shapes of many rows and 3077 of few, twice as many took 4% and 1% longer, half as many 4%
// and none. With several sequences the kernels spread the tokens that there are over them, and a
// long sequence may take 1.5 and 8 times its part of the workgroups. With twice its part 48
// sequences of up to 16384 tokens, a quarter of that in the mean, took 128 us, with 4 times 104,
// 8 times 98; many rows, in whose launches empty and small workgroups cost more, take as long
// with 2 and with 4 times on average, and 216 row tiles of 256 wide heads had better stay whole
// (227 us, in two parts 250).
Split split_of(const KvShape &c, int64_t T, int seqs, int group, bool many, const Rows &of, int max_kv) {
    const int tile_rows = many ? kTileRows : kSplitRows;
    // Row tiles: of the most rows of a sequence, and no more than T queries in all make.
    const int64_t tiles = std::min(seqs * (((many ? of.many : of.few) + tile_rows - 1) / tile_rows),
                                   T * group / tile_rows + seqs);
    const int64_t blocks = c.heads * tiles;
    Split sp;
    sp.rows_from = many && of.few > 0 ? (int)of.few + 1 : 0;
    sp.rows_to = many || of.many == 0 ? INT32_MAX : (int)of.few;
    const int64_t target = many ? (c.dim <= 128 ? 384 : 256) : 512;
    const int64_t most = target * (seqs == 1 ? 2 : many ? 3 : 16) / 2 / blocks;
    const int64_t least = blocks <= 16 ? 256 : blocks < 512 ? 512 : 1024;
    const int64_t splits = max_kv <= kWholeTokens ? 1 : std::min(most, (max_kv + least - 1) / least);
    sp.splits = (int)std::max<int64_t>(splits, 1);
    sp.target = seqs == 1 || seqs > kSummed || sp.splits == 1 ? 0 : (int)target;
    sp.share = (int)(sp.target ? least : std::max<int64_t>((max_kv + sp.splits - 1) / sp.splits, 1) + 127) / 128 * 128;
    const uint32_t pb = (uint32_t)c.page / 16;
    sp.magic = (((uint64_t)1 << 32) + pb - 1) / pb;
    sp.part = nullptr;
    sp.joined = false;
    return sp;
}

// The launches of a call.
struct Plan {
    Rows rows;
    Split few, many;
    int splits;      // the most of them; 1: nothing to join
};

Plan plan_of(const KvShape &c, int64_t T, int seqs, int group, int max_q, int max_kv) {
    Plan p;
    p.rows = rows_of(T, seqs, group, max_q);
    p.splits = 1;
    if (p.rows.few > 0) {
        p.few = split_of(c, T, seqs, group, false, p.rows, max_kv);
        p.splits = p.few.splits;
    }
    if (p.rows.many > 0) {
        p.many = split_of(c, T, seqs, group, true, p.rows, max_kv);
        p.splits = std::max(p.splits, p.many.splits);
    }
    return p;
}

template <int FMT, int D>
hipError_t run_plan(const KvShape &c, const KvAttnArgs &a, Plan &p, float *ws, hipStream_t s) {
    const int64_t rows = a.T * c.heads * a.group;
    const auto run = [&](bool many, Split &sp, int64_t most_rows) {
        sp.part = ws;
        sp.joined = p.splits > 1;
        const int64_t units = (int64_t)c.heads * a.seqs * sp.splits;
        if (!many) {
            if (!launchable(units, 256))
                return hipErrorInvalidValue;
            const dim3 grid((unsigned)units, (unsigned)((most_rows + kSplitRows - 1) / kSplitRows));
            hipLaunchKernelGGL((kv_attention_split_kernel<FMT, D>), grid, dim3(256), 0, s, c, a, sp);
            return hipGetLastError();
        }
        // A workgroup goes on to every tiles-th row tile, so that a loose max_q costs empty
        // workgroups but never more than kMostGroups of them.
        const int64_t columns = units >= kSpreadUnits ? (units + 7) / 8 * 8 : units;
        const int64_t tiles = std::min((most_rows + kTileRows - 1) / kTileRows,
                                       std::max<int64_t>(kMostGroups / columns, 1));
        if (!launchable(columns * tiles, 256))
            return hipErrorInvalidValue;
        hipLaunchKernelGGL((kv_attention_tile_kernel<FMT, D>), dim3((unsigned)(columns * tiles)),
                           dim3(256), 0, s, c, a, sp, (int)tiles);
        return hipGetLastError();
    };
    hipError_t e = hipSuccess;
    if (p.rows.few > 0)
        e = run(false, p.few, p.rows.few);
    if (e == hipSuccess && p.rows.many > 0)
        e = run(true, p.many, p.rows.many);
    if (e != hipSuccess || p.splits == 1)
        return e;
    // Few splits: a row by D / 4 lanes. Many: 32 outputs of a row by 32 groups of 8 lanes.
    return p.splits <= 16 || rows * (D / 4) >= 65536
               ? launch_join<D, D / 4, 1>(ws, p.splits, rows, a.out, s)
               : launch_join<D, 8, 32>(ws, p.splits, rows, a.out, s);
}

}  // namespace

size_t kv_attention_workspace_bytes(const KvShape &c, int64_t T, int seqs, int group, int max_q,
                                    int max_kv) {
    const Plan p = plan_of(c, T, seqs, group, max_q, max_kv);
    return p.splits == 1 ? 0 : (size_t)p.splits * T * c.heads * group * (c.dim + 4) * 4;
}

hipError_t launch_kv_attention(const KvShape &c, const KvAttnArgs &a, void *ws, hipStream_t s) {
    if (a.T * c.heads * a.group > INT32_MAX)
        return hipErrorInvalidValue;
    Plan p = plan_of(c, a.T, a.seqs, a.group, a.max_q, a.max_kv);
    const auto run = [&](auto dim, auto format) {
        return run_plan<decltype(format)::value, decltype(dim)::value>(c, a, p, static_cast<float *>(ws), s);
    };
    const auto go = [&](auto dim) {
        return c.fmt == KV_FP8 ? run(dim, std::integral_constant<int, KV_FP8>{})
                               : run(dim, std::integral_constant<int, KV_FP4>{});
    };
    switch (c.dim) {
    case 64: return go(std::integral_constant<int, 64>{});
    case 128: return go(std::integral_constant<int, 128>{});
    case 192: return go(std::integral_constant<int, 192>{});
    default: return go(std::integral_constant<int, 256>{});
    }
}

}  // namespace w8a8
