// Attention of drafted token trees over the quantized cache.
//
// The last lq cached tokens of a sequence are the nodes of a tree, its lq queries their own; query
// i sees all tokens in front of the tree and the nodes whose bits its mask has set, itself and its
// ancestors. The mathematics is that of kv_attention.hip: the queries of all the heads that share a
// key/value head are the rows of one problem, one pass over the keys keeps a running maximum m and
// sum l a row in float32, S^T = K Q^T and O^T = V^T P^T on the bf16 matrix instructions, and the
// weights are rounded to one bf16 term (2^-8 of each) for the second product.
//
// A step of a sequence has some tens of nodes, so a row tile of 128 rows is seldom full, and the
// lengths of a batch differ: the work is divided by what there is. The pieces of a call (a row tile
// of a head and sequence, and a part of its keys) are numbered one after the other, about as many
// as the card runs at once, each of about the same cost; a workgroup finds the piece of its own
// number by a scan over the sequences. Partial results lie in the pieces' own slots of the workspace,
// and a second launch joins those of a row tile, found by the same scan. So everything follows from
// the lengths on the device, no row outside the sequences is read or written, and sums have a fixed
// order.
#include "kv_attention.hpp"

#include <algorithm>

namespace w8a8 {
namespace {

constexpr int kRows = 128, kTokens = 64;       // of a row tile, and staged at a time
// Sequences over whose tokens a wavefront sums, 64 at a time; with more of them keys stay whole.
constexpr int kSummed = 512;

struct TreePlan {
    int target;        // pieces that the keys are divided for, 0: every row tile is one
    int least;         // tokens of a piece at least (a multiple of 64)
    int grid;          // pieces there can be
    float *part;       // [grid][kRows][dim + 4]: O, m, l of a piece
    uint64_t magic;    // n / (page / 16) = n * magic >> 32 for n < 2^22
};

// What a row of a tree sees: the tokens in front of it, and nodes by its bits.
struct TreeRow {
    const uint32_t *bits;     // nullptr: no row, sees nothing
    int words, prefix, kv;    // the tree's first token (below 0: its first nodes are not cached)
    __device__ __forceinline__ TreeRow(const KvAttnArgs &a, const Seq &s, int qi, bool live)
        : bits(live ? a.tree + (s.q0 + qi) * a.tree_words : nullptr), words(a.tree_words),
          prefix(s.kv - s.lq), kv(s.kv) {}
    __device__ __forceinline__ uint32_t word(int i) const { return i < words ? bits[i] : 0; }
    // Tokens j .. j + 31, the first in the lowest bit.
    __device__ __forceinline__ uint32_t window(int j) const {
        if (!bits || j >= kv)
            return 0;
        const int node = j - prefix;
        uint32_t w;
        if (node <= -32)
            w = ~0u;
        else if (node < 0)
            w = word(0) << -node | ((1u << -node) - 1);
        else
            w = (uint32_t)((word(node / 32) | (uint64_t)word(node / 32 + 1) << 32) >> node % 32);
        return kv - j < 32 ? w & ((1u << (kv - j)) - 1) : w;
    }
    __device__ __forceinline__ bool any() const {
        uint32_t w = 0;
        for (int j = 0; w == 0 && j < kv; j += 32)
            w = window(j);
        return w != 0;
    }
};

// A piece, or a row tile with all of its pieces.
struct Job {
    bool found;
    Seq seq;
    int b, head, tile, split;
    int used;          // pieces of a row tile of this sequence
    int slot, stride;  // of the tile's first piece, and from one to the next
};

// Eighths of the cost of a full row tile: up to half as many rows take products of half the size,
// but the same staging (measured).
__device__ __forceinline__ int eighths(int rows) { return rows <= kRows / 2 ? 5 : 8; }

// Job number `index` of the call's pieces, or (WHOLE) of its row tiles.
template <bool WHOLE>
__device__ __forceinline__ Job find_job(const KvShape &c, const KvAttnArgs &a, const TreePlan &plan,
                                        int index) {
    const int lane = threadIdx.x & 63;
    const auto rows_of = [&](const Seq &s) { return max(s.lq, 0) * a.group; };
    const auto tiles_of = [&](int rows) { return (rows + kRows - 1) / kRows; };
    // The share of a piece, in eighths of a token of a full tile. Float32 in a fixed order: the same
    // in every workgroup.
    float share = 0.0f;
    if (plan.target > 0) {
        for (int i = lane; i < a.seqs; i += 64) {
            const Seq s = sequence(c, a, i);
            const int rows = rows_of(s);
            share += (float)max(s.kv, 0) * (float)(tiles_of(rows) * eighths(rows));
        }
#pragma unroll
        for (int d = 32; d > 0; d /= 2)
            share += __shfl_xor(share, d);
        share *= (float)c.heads / (float)plan.target;
    }
    Job job;
    job.found = false;
    int pieces = 0, jobs = 0;              // in front of the 64 sequences at hand
    for (int i0 = 0; i0 < a.seqs; i0 += 64) {
        const int i = i0 + lane;
        int used = 0, tiles = 0;
        if (i < a.seqs) {
            const Seq s = sequence(c, a, i);
            const int rows = rows_of(s);
            tiles = tiles_of(rows);
            used = 1;
            if (plan.target > 0 && s.kv > plan.least) {
                const float tokens = fmaxf(share / (float)eighths(rows), (float)plan.least);
                used = min((int)ceilf((float)s.kv / tokens), (s.kv + plan.least - 1) / plan.least);
            }
        }
        // what comes to more than a grid is some malformed array's: counted as one past it
        const int most = plan.grid + 1;
        const int own = (int)min((int64_t)c.heads * tiles * used, (int64_t)most);
        const int own_jobs = WHOLE ? (int)min((int64_t)c.heads * tiles, (int64_t)most) : own;
        int sum = own, sum_jobs = own_jobs;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int x = __shfl_up(sum, d), y = __shfl_up(sum_jobs, d);
            if (lane >= d) {
                sum += x;
                sum_jobs += y;
            }
        }
        const uint64_t past = __ballot(jobs + sum_jobs > index);
        if (past) {
            const int at = __builtin_ctzll(past);
            const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
            job.found = true;
            job.b = i0 + at;
            job.seq = sequence(c, a, job.b);
            job.used = of(used);
            job.stride = c.heads * of(tiles);
            int in = index - jobs - of(sum_jobs - own_jobs);
            job.split = 0;
            if constexpr (!WHOLE) {
                job.split = in / job.stride;
                in -= job.split * job.stride;
            }
            // heads fastest: the row tiles of a head go to one XCD where heads come in eights
            job.tile = in / c.heads;
            job.head = in - job.tile * c.heads;
            job.slot = pieces + of(sum - own) + in;
            return job;
        }
        pieces = min(pieces + __builtin_amdgcn_readlane(sum, 63), most);
        jobs = min(jobs + __builtin_amdgcn_readlane(sum_jobs, 63), most);
    }
    return job;
}

// The other half's value beside this one's: lanes l and l ^ 32 hold the same row.
__device__ __forceinline__ u32x2 halves_of(float v) {
    return __builtin_bit_cast(
        u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
}

// A piece: 64 tokens at a time are decoded once into LDS for all four wavefronts, between the
// products of the 64 before. A wavefront has 32 rows and all 64 tokens of each step, or, in tiles
// of up to 64 rows, 32 rows and 32 of the tokens; then two wavefronts' results are joined in LDS.
// Rows in LDS and fragments as in kv_attention.hip's kernel for many rows.
template <int FMT, int D>
__global__ void __launch_bounds__(256, D <= 128 ? 2 : 1)
kv_tree_kernel(KvShape c, KvAttnArgs a, TreePlan plan) {
    constexpr int TT = kTokens;
    constexpr int VU = FMT == KV_FP8 ? 16 : 32;        // a unit: 16 bytes of codes
    constexpr int VT = D / VU, UNITS = TT * VT, NU = (UNITS + 255) / 256;
    constexpr int CB = FMT == KV_FP8 ? D : D / 2;
    constexpr int RSK = 2 * D + 16, RSV = 2 * D + 64;
    constexpr int KS = D / 16, F = D / 32;
    __shared__ __attribute__((aligned(16))) uint8_t keys[2][TT * RSK];
    __shared__ __attribute__((aligned(16))) uint8_t values[2][TT * RSV];
    __shared__ Places places;
    __shared__ uint8_t nan_unit[2][UNITS];
    __shared__ int nan_any;
    __shared__ float other_m[2][64], other_l[2][64];
    __shared__ uint32_t other_nan[2][64];
    static_assert(sizeof(keys) >= 2 * 64 * (D / 2) * sizeof(float), "O of two wavefronts");

    const Job job = find_job<false>(c, a, plan, blockIdx.x);
    if (!job.found)
        return;
    const Seq seq = job.seq;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r32 = lane & 31, h = lane >> 5;
    const int rows = seq.lq * a.group, q_heads = c.heads * a.group, head = job.head;
    const int64_t v_offset = c.heads * c.head_bytes();
    const int kv = max(seq.kv, 0);
    const int per = ((kv + job.used - 1) / job.used + TT - 1) / TT * TT;
    const int piece_first = min(job.split * per, kv), piece_end = min(piece_first + per, kv);
    const int all_see = max(0, seq.kv - seq.lq);       // tokens that every row sees

    const auto run = [&](auto groups) __attribute__((always_inline)) {
        constexpr int RG = decltype(groups)::value, TG = 4 / RG;      // of rows, of tokens
        constexpr int NS = 2 / TG, US = 4 / TG;        // fragments of 32 keys, steps of 16 values
        const int rg = wave % RG, tg = wave / RG;
        const int first_row = job.tile * kRows + rg * 32, row = first_row + r32;
        const bool live = row < rows, wave_live = first_row < rows;
        const int qi = live ? row / a.group : 0;
        const int qh = head * a.group + (live ? row - qi * a.group : 0);
        const TreeRow tree(a, seq, qi, live);
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
        float m = start_of(tree.any()), l = 0.0f;
        uint32_t row_nan = 0;

        for (int j_first = piece_first; j_first < piece_end; j_first += kMaxChunk) {
            const int j_end = min(j_first + kMaxChunk, piece_end);
            const int ntile = (j_end - j_first + TT - 1) / TT;
            __syncthreads();
            if (threadIdx.x == 0)
                nan_any = 0;
            fill_places(places, c, a, plan.magic, job.b, head, j_first, j_end, ntile * (TT / 16));
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
                const int mine = j0 + 32 * tg;         // this wavefront's first token
                const bool part_seen = partly_seen(j0);
                lds_barrier();       // this tile is staged, the other stage's last one is read
                if (partly_seen(j0 + TT) && tile + 1 < ntile)
                    mark(j0 + TT, st ^ 1);
                if (part_seen && nan_any) {    // rare: which rows see a NaN block
                    const uint64_t visible = tree.window(j0) | (uint64_t)tree.window(j0 + 32) << 32;
                    for (int unit = 0; unit < UNITS; ++unit)
                        if (nan_unit[st][unit] && visible >> (unit / VT) & 1)
                            row_nan |= 1u << (unit % VT * VU / 32);
                }
                // Scores: token 32 t + 8 (i / 4) + 4 h + i % 4 in s[t][i]. Between the products
                // the next tile is staged (after the last tile: itself again, unread).
                f32x16 s[NS];
#pragma unroll
                for (int t = 0; t < NS; ++t)
                    s[t] = f32x16{};
                const uint8_t *kp = keys[st] + (32 * tg + r32) * RSK + h * 16;
                bf16x8 fk[2][NS];
                const auto read_keys = [&](int k) __attribute__((always_inline)) {
#pragma unroll
                    for (int t = 0; t < NS; ++t)
                        fk[k & 1][t] = *reinterpret_cast<const bf16x8 *>(kp + t * 32 * RSK + k * 32);
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
#pragma unroll
                        for (int t = 0; t < NS; ++t)
                            s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                                fk[k & 1][t], __builtin_bit_cast(bf16x8, q[k]), s[t], 0, 0, 0);
                        __builtin_amdgcn_sched_barrier(0);
                    }(), ...);
                }(std::make_integer_sequence<int, KS>{});
                // The next loads go out between the products with the values.
                if (!wave_live || mine >= seq.kv) {
                    load_all(min(tile + 2, ntile - 1));
                    continue;
                }

                if (part_seen) {
                    uint32_t visible[NS];
#pragma unroll
                    for (int t = 0; t < NS; ++t)
                        visible[t] = tree.window(mine + 32 * t) >> 4 * h;
                    keep_branch();
#pragma unroll
                    for (int t = 0; t < NS; ++t)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            s[t][i] = visible[t] >> (8 * (i / 4) + i % 4) & 1 ? s[t][i] : -INFINITY;
                }
                float top = -INFINITY;
#pragma unroll
                for (int t = 0; t < NS; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        top = fmaxf(top, s[t][i]);
                const u32x2 tops = halves_of(top);
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
                const uint8_t *vp = values[st] + (32 * tg + 4 * h + ((lane & 15) >> 2)) * RSV +
                                    ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
                u32x2 fv[2][2];
                const auto read_values = [&](int z) __attribute__((always_inline)) {
                    const uint8_t *src = vp + 16 * (z / F) * RSV + z % F * 64;
                    fv[z & 1][0] = __builtin_bit_cast(
                        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)src));
                    fv[z & 1][1] = __builtin_bit_cast(
                        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(src + 8 * RSV)));
                };
                u32x4 p[US];
                const auto weight = [&](auto qc) __attribute__((always_inline)) {
                    constexpr int w = decltype(qc)::value;     // of 8 NS pairs
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
                        if constexpr (z + 1 < US * F)
                            read_values(z + 1);
                        if constexpr (u < US - 1) {
                            constexpr int w0 = 4 * (u + 1) + f * 4 / F, w1 = 4 * (u + 1) + (f + 1) * 4 / F;
                            if constexpr (w0 < w1)
                                weight(std::integral_constant<int, w0>{});
                            if constexpr (w0 + 1 < w1)
                                weight(std::integral_constant<int, w0 + 1>{});
                        }
                        if constexpr (z < 2 * NU && z % 2 == 1)
                            load(std::integral_constant<int, z / 2>{}, min(tile + 2, ntile - 1));
                        static_assert(2 * NU <= US * F, "loads between the products");
                        __builtin_amdgcn_sched_barrier(0);
                        o[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            __builtin_bit_cast(bf16x8, u32x4{fv[z & 1][0][0], fv[z & 1][0][1],
                                                             fv[z & 1][1][0], fv[z & 1][1][1]}),
                            __builtin_bit_cast(bf16x8, p[u]), o[f], 0, 0, 0);
                        __builtin_amdgcn_sched_barrier(0);
                    }(), ...);
                }(std::make_integer_sequence<int, US * F>{});
            }
        }

        const u32x2 ls = halves_of(l);
        l = __uint_as_float(ls[0]) + __uint_as_float(ls[1]);
        if constexpr (TG > 1) {
            // The other tokens' m, l and O of the same rows, lane by lane.
            f32x4 *const os = reinterpret_cast<f32x4 *>(&keys[0][0]) + rg * (F * 4 * 64) + lane;
            __syncthreads();           // the stages are read
            if (tg == 1) {
                other_m[rg][lane] = m;
                other_l[rg][lane] = l;
                other_nan[rg][lane] = row_nan;
#pragma unroll
                for (int f = 0; f < F; ++f)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        os[(f * 4 + i) * 64] =
                            f32x4{o[f][4 * i], o[f][4 * i + 1], o[f][4 * i + 2], o[f][4 * i + 3]};
            }
            __syncthreads();
            if (tg == 1)
                return;
            const float m2 = other_m[rg][lane], mm = fmaxf(m, m2), base = mm == -INFINITY ? 0.0f : mm;
            const float f1 = __builtin_amdgcn_exp2f(m - base), f2 = __builtin_amdgcn_exp2f(m2 - base);
            l = l * f1 + other_l[rg][lane] * f2;
            m = mm;
            row_nan |= other_nan[rg][lane];
#pragma unroll
            for (int f = 0; f < F; ++f)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 x = os[(f * 4 + i) * 64];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[f][4 * i + e] = o[f][4 * i + e] * f1 + x[e] * f2;
                }
        }
        if (!live)
            return;
        const int64_t out_row = (seq.q0 + qi) * q_heads + qh;
        const float inv = inverse(l, m);
        const int64_t slot = job.slot + (int64_t)job.split * job.stride;
        float *const part = plan.part + (slot * kRows + row - job.tile * kRows) * (D + 4);
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const bool nan = row_nan >> f & 1;
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int d = 32 * f + 2 * i + 4 * h;
                f32x4 v = {o[f][i], o[f][i + 1], o[f][i + 2], o[f][i + 3]};
                if (nan)
                    v = f32x4{NAN, NAN, NAN, NAN};
                if (job.used == 1)
                    store_outputs(a.out + out_row * D + d, v, inv);
                else
                    *reinterpret_cast<f32x4 *>(part + d) = v;
            }
        }
        if (job.used > 1 && h == 0) {
            part[D] = m;
            part[D + 1] = l;
        }
    };
    if (rows - job.tile * kRows <= kRows / 2)
        run(std::integral_constant<int, 2>{});
    else
        run(std::integral_constant<int, 4>{});
}

// Joins the pieces of a row tile with weights 2^(m_s - max m): D / 4 lanes a row, blockIdx.y a
// quarter of the tile.
constexpr int kJoinParts = 4;

template <int D>
__global__ void __launch_bounds__(256)
kv_tree_join_kernel(KvShape c, KvAttnArgs a, TreePlan plan) {
    constexpr int LANES = D / 4, ROWS = 256 / LANES;
    const Job job = find_job<true>(c, a, plan, blockIdx.x);
    if (!job.found || job.used == 1)
        return;
    const int lane = threadIdx.x % LANES, first = threadIdx.x / LANES, d = 4 * lane;
    const int rows = min(job.seq.lq * a.group - job.tile * kRows, kRows), q_heads = c.heads * a.group;
    const int used = job.slot + (int64_t)(job.used - 1) * job.stride < plan.grid ? job.used : 0;
    if (first >= ROWS)
        return;
    for (int r = blockIdx.y * ROWS + first; r < rows; r += kJoinParts * ROWS) {
        const float *p = plan.part + ((int64_t)job.slot * kRows + r) * (D + 4);
        const int64_t stride = (int64_t)job.stride * kRows * (D + 4);
        float m = -INFINITY, l = 0.0f;
        f32x4 v = {};
#pragma unroll 4
        for (int s = 0; s < used; ++s) {
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
        const int row = job.tile * kRows + r, qi = row / a.group;
        const int64_t out_row = (job.seq.q0 + qi) * q_heads + job.head * a.group + row - qi * a.group;
        store_outputs(a.out + out_row * D + d, v, inverse(l, m));
    }
}

// Row tiles that T queries in sequences can make, whatever each has of them.
int64_t blocks_of(const KvShape &c, int64_t T, int seqs, int group) {
    return c.heads * (T * group / kRows + std::min<int64_t>(seqs, T));
}

constexpr int kWholeTokens = 512;

TreePlan plan_of(const KvShape &c, int64_t T, int seqs, int group, int max_kv) {
    TreePlan p;
    const int64_t blocks = blocks_of(c, T, seqs, group);
    const bool divided = max_kv > kWholeTokens && seqs <= kSummed;
    p.target = divided ? (c.dim <= 128 ? 512 : 256) : 0;
    p.least = 256;
    // pieces: a share less than their number for each row tile, and the target in all
    p.grid = (int)std::min<int64_t>(blocks + p.target + p.target / 16, INT32_MAX / 2);
    const uint32_t pb = (uint32_t)c.page / 16;
    p.magic = (((uint64_t)1 << 32) + pb - 1) / pb;
    p.part = nullptr;
    return p;
}

}  // namespace

size_t kv_tree_workspace_bytes(const KvShape &c, int64_t T, int seqs, int group, int max_kv) {
    const TreePlan p = plan_of(c, T, seqs, group, max_kv);
    return p.target == 0 ? 0 : (size_t)p.grid * kRows * (c.dim + 4) * 4;
}

hipError_t launch_kv_tree(const KvShape &c, const KvAttnArgs &a, void *ws, hipStream_t s) {
    if (a.T * c.heads * a.group > INT32_MAX)
        return hipErrorInvalidValue;
    TreePlan plan = plan_of(c, a.T, a.seqs, a.group, a.max_kv);
    plan.part = static_cast<float *>(ws);
    const int64_t blocks = blocks_of(c, a.T, a.seqs, a.group);
    if (!launchable(plan.grid, 256) || !launchable(blocks, 256))
        return hipErrorInvalidValue;
    const auto run = [&](auto dim, auto format) {
        constexpr int F = decltype(format)::value, D = decltype(dim)::value;
        hipLaunchKernelGGL((kv_tree_kernel<F, D>), dim3((unsigned)plan.grid), dim3(256), 0, s, c, a, plan);
        if (plan.target > 0 && hipPeekAtLastError() == hipSuccess)
            hipLaunchKernelGGL((kv_tree_join_kernel<D>), dim3((unsigned)blocks, kJoinParts), dim3(256), 0,
                               s, c, a, plan);
        return hipGetLastError();
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
