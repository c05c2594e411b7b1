// Attention of drafted token trees over the quantized cache.
//
// The last lq cached tokens of a sequence are the nodes of a tree, its lq queries their own; query
// i sees all tokens in front of the tree and the nodes whose bits its mask has set, itself and its
// ancestors. The mathematics is that of kv_attention.hip: the queries of all the heads that share a
// key/value head are the rows of one problem, one pass over the keys keeps a running maximum m and
// sum l a row in float32, S^T = K Q^T and O^T = V^T P^T on the bf16 matrix instructions. The weights
// are rounded for the second product: to two bf16 terms (2^-16 of each at most) in row tiles of up to
// 64 rows, to one (2^-8) in others, whose products bind. There l sums the rounded weights: what a
// weight's rounding by d does to an output is then d (v - o) / l and not d v / l, less where a few
// weights are most of the sum. Two terms everywhere take 414 us where one takes 324 (32 trees of 60 nodes on
// 8192 tokens, 8 heads of 128, 4 queries a head), 220 where it takes 173 (201 nodes on 40001). Rounding is
// relative to a piece's running maximum (the largest weight, 1, stays as it is), so one term's hangs on
// where the pieces end: on all lengths of a call.
//
// A step of a sequence has some tens of nodes, so a row tile of 128 rows is seldom full, and the
// lengths of a batch differ: the work is divided by what there is. The pieces of a call (a row tile
// of a head and sequence, and a part of its keys) are numbered one after the other, about as many
// as the card runs at once, each of about the same cost; a workgroup finds the piece of its own
// number by a scan over the sequences (where keys stay whole, by a search among their starts). Pieces of
// row tiles that are divided have a slot each in the workspace for their partial results, and a second
// launch joins those of each such tile, whose first piece has left a note where they are. So everything
// follows from the lengths on the device, no row outside the sequences is read or written, and sums have
// a fixed order.
//
// 32 trees of 60 nodes on 8192 tokens each, 8 heads of 128, 4 queries a head, take 315 us (800 TFLOP/s, 880
// where no row tile is partly filled), 16 nodes on the same 167 (3.3 TB/s). No unit binds alone: of the
// SIMDs' cycles 47% are matrix and 43% vector instructions (16 nodes: 35% and 43%), which the two
// wavefronts of each overlap only in part, and 12% of the CUs' cycles are conflicts in LDS. 32 trees of up to
// 60 nodes on up to 8192 tokens, all different: 235 us where a sequence's keys were divided as the causal
// kernel divides them, 91 to 99 so.
#include "kv_attention.hpp"

#include <algorithm>

namespace w8a8 {
namespace {

constexpr int kRows = 128, kTokens = 64;       // of a row tile, and staged at a time
constexpr int kMostTiles = 1 << 20;            // counted of a sequence: far more than run at once
// Sequences over whose tokens a wavefront sums, 64 at a time; with more of them keys stay whole, however
// long: a sequence of 100000 tokens among ones of 500, 8 nodes each, 8 heads of 128, 4 queries a head: 290 us
// with 512 sequences, 1919 with 513, 1942 with 1024 (355 without the long one).
constexpr int kSummed = 512;

// Where the pieces of a divided row tile are.
struct Note {
    int b, head, tile;
    int used;          // pieces; of the first note: the divided row tiles of the call
    int slot, stride;  // of the tile's first piece, and from one to the next
    int pad[2];
};

struct TreePlan {
    int target;        // pieces that the keys are divided for, 0: every row tile is one (find_tile)
    int least;         // tokens of a piece at least (a multiple of 64)
    int grid;          // pieces there can be
    int tiles, slots;  // divided row tiles there can be, and their pieces
    struct Note *notes;   // [1 + tiles]: the number of divided row tiles, then each of them
    float *part;       // [slots][kRows][dim + 4]: O, m, l of a piece
    uint64_t magic;    // n / (page / 16) = n * magic >> 32 for n < 2^22
};

struct Job {
    bool found;
    Note note;
    int number, split; // of its row tile among the divided ones, and of the piece in that
    Seq seq;
};

// Eighths of the cost of a full row tile: up to half as many rows take products of half the size, but
// the same staging: 1.17 and 1.5 us a step of 64 tokens, two workgroups a CU, heads of 128.
__device__ __forceinline__ int eighths(int rows) { return rows <= kRows / 2 ? 6 : 8; }

__device__ __forceinline__ int rows_of(const KvAttnArgs &a, const Seq &s) { return max(s.lq, 0) * a.group; }
__device__ __forceinline__ int tiles_of(int rows) { return (rows + kRows - 1) / kRows; }

// Pieces of a row tile of a sequence. share: their cost, in eighths of a token of a full tile.
__device__ __forceinline__ int used_of(const TreePlan &plan, int kv, int rows, float share) {
    if (kv <= plan.least)
        return 1;
    const float tokens = fmaxf(share * (rows <= kRows / 2 ? 1.0f / 6.0f : 0.125f), (float)plan.least);
    return min((int)ceilf((float)kv * __builtin_amdgcn_rcpf(tokens)), (kv + plan.least - 1) / plan.least);
}

// Sums over the lanes up to each, in DPP operands (a shuffle goes through LDS).
template <typename V>
__device__ __forceinline__ V lanes_scan(V v) {
    const auto step = [&](auto ctrl, auto rows) {
        const int x = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value,
                                                  decltype(rows)::value, 0xF, true);
        v += __builtin_bit_cast(V, x);
    };
    using std::integral_constant;
    step(integral_constant<int, 0x111>{}, integral_constant<int, 0xF>{});   // row_shr:1
    step(integral_constant<int, 0x112>{}, integral_constant<int, 0xF>{});   // row_shr:2
    step(integral_constant<int, 0x114>{}, integral_constant<int, 0xF>{});   // row_shr:4
    step(integral_constant<int, 0x118>{}, integral_constant<int, 0xF>{});   // row_shr:8
    step(integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});   // row_bcast:15, rows 1, 3
    step(integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});   // row_bcast:31, rows 2, 3
    return v;
}

__device__ __forceinline__ float last_lane(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}

// The cost of a piece: the call's divided by the target, rounded up to the least that makes no more
// pieces than the target (what runs at once), up to half as much again: one sequence of 9.1 shares
// makes 10 pieces a row tile, and the last of them a second round. Where none does, as with many
// row tiles of very different lengths, three quarters of it: the rounds then even out. With up to 64
// sequences, a lane each. Sums have a fixed order: the same result in every workgroup.
__device__ __forceinline__ float share_of(const KvShape &c, const TreePlan &plan, int seqs, float sum,
                                          int kv, int rows) {
    const float even = last_lane(lanes_scan(sum)) * (float)c.heads * __builtin_amdgcn_rcpf((float)plan.target);
    if (seqs <= 64) {
        const int tiles = tiles_of(rows), most = plan.target / c.heads;
        if (qmath::wave_sum(min(tiles, kMostTiles)) <= most)
            for (int n = 8; n <= 12; ++n) {
                const float share = even * (float)n * 0.125f;
                if (qmath::wave_sum(min(tiles * used_of(plan, kv, rows, share), kMostTiles)) <= most)
                    return share;
            }
    }
    return even * 0.75f;
}

// Row tile `index` of a call whose keys stay whole. Tiles are numbered with gaps: those of a sequence
// from (its first row in the call) / kRows + (its number) on, which lies behind all tiles of those
// before it. So the sequence is found among the starts, 64 at a time, and not by a sum over all of
// them: 8192 sequences of up to 16 nodes on up to 512 tokens, 8 heads of 128, 7357 us by sums, 1850 so.
__device__ __forceinline__ Job find_tile(const KvShape &c, const KvAttnArgs &a, int index) {
    const int lane = threadIdx.x & 63;
    const int64_t number = index / c.heads;
    const auto first_of = [&](int b) {
        const int64_t q0 = a.q_starts ? min(max((int64_t)a.q_starts[b], (int64_t)0), a.T)
                                      : a.T / a.seqs * b;
        return q0 * a.group / kRows + b;
    };
    Job job;
    job.found = false;
    int b = 0;
    for (int step = a.seqs, left; step > 1;) {
        left = min(step, a.seqs - b);              // sequences from b on, one of which it is
        step = (left + 63) / 64;
        const bool before = lane * step < left && first_of(b + lane * step) <= number;
        b += max(__popcll(__ballot(before)) - 1, 0) * step;
    }
    job.seq = sequence(c, a, b);
    const int64_t tile = number - first_of(b);
    if (tile < 0 || tile >= tiles_of(rows_of(a, job.seq)))
        return job;
    job.found = true;
    job.number = job.split = 0;
    job.note.b = b;
    job.note.head = index - (int)number * c.heads;
    job.note.tile = (int)tile;
    job.note.used = job.note.stride = 1;
    job.note.slot = 0;
    return job;
}

// Piece number `index` of the call. For piece 0, `divided` becomes the number of divided row tiles.
__device__ __forceinline__ Job find_job(const KvShape &c, const KvAttnArgs &a, const TreePlan &plan,
                                        int index, int &divided) {
    const int lane = threadIdx.x & 63;
    // the first 64 sequences stay in registers
    int kv = 0, rows = 0;
    const auto fetch = [&](int i) {
        kv = rows = 0;
        if (i < a.seqs) {
            const Seq s = sequence(c, a, i);
            kv = max(s.kv, 0);
            rows = rows_of(a, s);
        }
    };
    float share = 0.0f;
    for (int i0 = (a.seqs - 1) / 64 * 64; i0 >= 0; i0 -= 64) {
        fetch(i0 + lane);
        share += (float)kv * (float)(tiles_of(rows) * eighths(rows));
    }
    share = share_of(c, plan, a.seqs, share, kv, rows);
    Job job;
    job.found = false;
    int pieces = 0, slots = 0, numbers = 0;          // in front of the 64 sequences at hand
    for (int i0 = 0; i0 < a.seqs; i0 += 64) {
        if (i0 > 0)
            fetch(i0 + lane);
        const int tiles = tiles_of(rows), used = tiles > 0 ? used_of(plan, kv, rows, share) : 0;
        // what comes to more than a grid is some malformed array's: counted as one past it
        const int most = plan.grid + 1;
        const int own_tiles = (int)min((int64_t)c.heads * tiles, (int64_t)most);
        const int own = (int)min((int64_t)own_tiles * used, (int64_t)most);
        // what is not divided has no slots and no note
        const int cut = used > 1 ? own : 0, cut_tiles = used > 1 ? own_tiles : 0;
        const int sum = lanes_scan(own), sum_cut = lanes_scan(cut), sum_tiles = lanes_scan(cut_tiles);
        const uint64_t past = __ballot(pieces + sum > index);
        if (past && !job.found) {
            const int at = __builtin_ctzll(past);
            const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
            const int first = pieces + of(sum - own);
            uint32_t in = index - first;
            job.found = true;
            job.note.b = i0 + at;
            job.note.used = of(used);
            job.note.stride = of(own_tiles);
            job.split = in / (uint32_t)job.note.stride;
            in -= job.split * job.note.stride;
            // heads fastest: the row tiles of a head go to one XCD where heads come in eights
            job.note.tile = in / (uint32_t)c.heads;
            job.note.head = in - job.note.tile * c.heads;
            job.note.slot = slots + of(sum_cut - cut) + in;
            job.number = numbers + of(sum_tiles - cut_tiles) + in;
            job.seq = sequence(c, a, job.note.b);
            if (index > 0)
                return job;
        }
        pieces = min(pieces + __builtin_amdgcn_readlane(sum, 63), most);
        slots = min(slots + __builtin_amdgcn_readlane(sum_cut, 63), most);
        numbers = min(numbers + __builtin_amdgcn_readlane(sum_tiles, 63), most);
    }
    divided = numbers;
    return job;
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
    // Tiles whose codes are in registers: two give the loads a step more time (32 trees of 60 nodes on
    // 8192 tokens 320 us with one, 311 with two); above 128 channels there is no room for them.
    constexpr int SETS = D <= 128 ? 2 : 1;
    __shared__ __attribute__((aligned(16))) uint8_t keys[2][TT * RSK];
    __shared__ __attribute__((aligned(16))) uint8_t values[2][TT * RSV];
    __shared__ Places places;
    __shared__ uint8_t nan_unit[2][UNITS];
    __shared__ int nan_any;
    __shared__ float other_m[2][64], other_l[2][64];
    __shared__ uint32_t other_nan[2][64];
    static_assert(sizeof(keys) >= 2 * 64 * (D / 2) * sizeof(float), "O of two wavefronts");

    int divided = 0;
    const Job job = plan.target > 0 ? find_job(c, a, plan, blockIdx.x, divided) : find_tile(c, a, blockIdx.x);
    if (plan.target > 0 && blockIdx.x == 0 && threadIdx.x == 0)
        plan.notes[0].used = min(divided, plan.tiles);
    if (!job.found)
        return;
    const int64_t slot = job.note.slot + (int64_t)job.split * job.note.stride;
    if (job.note.used > 1) {
        if (slot >= plan.slots)        // with lengths that no call may have (sequences that overlap)
            return;
        if (job.split == 0 && threadIdx.x == 0 && job.number < plan.tiles)
            plan.notes[1 + job.number] = job.note;
    }
    const Seq seq = job.seq;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r32 = lane & 31, h = lane >> 5;
    const int rows = seq.lq * a.group, q_heads = c.heads * a.group, head = job.note.head;
    const int64_t v_offset = c.heads * c.head_bytes();
    const int kv = max(seq.kv, 0);
    const int per = ((kv + job.note.used - 1) / job.note.used + TT - 1) / TT * TT;
    const int piece_first = min(job.split * per, kv), piece_end = min(piece_first + per, kv);
    const int all_see = max(0, seq.kv - seq.lq);       // tokens that every row sees

    const auto run = [&](auto groups) __attribute__((always_inline)) {
        constexpr int RG = decltype(groups)::value, TG = 4 / RG;      // of rows, of tokens
        constexpr int NS = 2 / TG, US = 4 / TG;        // fragments of 32 keys, steps of 16 values
        constexpr int TERMS = TG;                      // bf16 terms of a weight
        const int rg = wave % RG, tg = wave / RG;
        const int first_row = job.note.tile * kRows + rg * 32, row = first_row + r32;
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
            fill_places(places, c, a, plan.magic, job.note.b, head, j_first, j_end, ntile * (TT / 16));
            __syncthreads();

            // Codes and scales on their way to the stages.
            u32x4 kc[SETS][NU], vc[SETS][NU];
            uint32_t ks[SETS][NU], vs[SETS][NU];
            const auto load = [&](auto set, auto ic, int tile) __attribute__((always_inline)) {
                constexpr int i = decltype(ic)::value, b = decltype(set)::value % SETS;
                const int unit = min(i * 256 + (int)threadIdx.x, UNITS - 1);
                const int tok = unit / VT, part = unit % VT;
                const int blk = tile * (TT / 16) + tok / 16;
                const int at = places.at[blk] + tok % 16;
                const uint8_t *p = a.cache + places.page[blk];
                const uint32_t code = at * CB + part * 16;
                const uint32_t scale = c.page * CB + at * (D / 32) + part * VU / 32;
                kc[b][i] = Unit<16>::load(p + code);
                ks[b][i] = p[scale];
                vc[b][i] = Unit<16>::load(p + v_offset + code);
                vs[b][i] = p[v_offset + scale];
            };
            const auto load_all = [&](auto set, int tile) __attribute__((always_inline)) {
                [&]<int... i>(std::integer_sequence<int, i...>) __attribute__((always_inline)) {
                    (load(set, std::integral_constant<int, i>{}, tile), ...);
                }(std::make_integer_sequence<int, NU>{});
            };
            // Values past the end, and NaN blocks in tiles that only some rows see whole, become
            // zeros before they are staged (a zero weight would not silence them).
            const auto mark = [&](auto set, int j0) __attribute__((always_inline)) {
                constexpr int st = decltype(set)::value, b = st % SETS;
#pragma unroll
                for (int i = 0; i < NU; ++i) {
                    const int unit = min(i * 256 + (int)threadIdx.x, UNITS - 1);
                    const bool past = j0 + unit / VT >= seq.kv;
                    const bool nan = vs[b][i] == kNaNScale && !past;
                    nan_unit[st][unit] = nan;
                    if (nan)
                        nan_any = 1;
                    if (past || nan) {
                        vc[b][i] = u32x4{};
                        vs[b][i] = 0;
                    }
                }
            };
            // Half z of 4 NU half units of a set into its stage: keys, then values.
            const auto stage = [&](auto set, auto zc) __attribute__((always_inline)) {
                constexpr int z = decltype(zc)::value / 2, half = decltype(zc)::value % 2, i = z % NU;
                constexpr int st = decltype(set)::value, b = st % SETS;
                const int unit = i * 256 + threadIdx.x, tok = unit / VT, part = unit % VT;
                if (UNITS % 256 != 0 && unit >= UNITS)
                    return;
                const u32x4 codes = z < NU ? kc[b][i] : vc[b][i];
                const float sc = scale_operand(z < NU ? ks[b][i] : vs[b][i]);
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
            constexpr std::integral_constant<int, 0> even;
            constexpr std::integral_constant<int, 1> odd;
            load_all(even, 0);
            if constexpr (SETS == 2)
                load_all(odd, min(1, ntile - 1));
            if (partly_seen(j_first))
                mark(even, j_first);
            [&]<int... z>(std::integer_sequence<int, z...>) __attribute__((always_inline)) {
                (stage(even, std::integral_constant<int, z>{}), ...);
            }(std::make_integer_sequence<int, 4 * NU>{});
            load_all(even, min(SETS, ntile - 1));
            // Tile `tile`, of even or odd number: multiplied, the one behind it staged, and the next that
            // has room loaded.
            const auto step = [&](auto number, auto next, int tile) __attribute__((always_inline)) {
                constexpr int st = decltype(number)::value;
                const int j0 = j_first + tile * TT;
                const int mine = j0 + 32 * tg;         // this wavefront's first token
                const bool part_seen = partly_seen(j0);
                lds_barrier();       // this tile is staged, the other stage's last one is read
                if (partly_seen(j0 + TT) && tile + 1 < ntile)
                    mark(next, j0 + TT);
                if (part_seen && nan_any) {    // rare: which rows see a NaN block
                    const uint64_t visible = tree.window(j0) | (uint64_t)tree.window(j0 + 32) << 32;
                    for (int unit = 0; unit < UNITS; ++unit)
                        if (nan_unit[st][unit] && visible >> (unit / VT) & 1)
                            row_nan |= 1u << (unit % VT * VU / 32);
                }
                // Scores: token 32 t + 8 (i / 4) + 4 h + i % 4 in s[t][i]. Between the products
                // the next tile is staged (after the last tile: some tile again, unread).
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
                            stage(next, std::integral_constant<int, z0>{});
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
                    load_all(next, min(tile + SETS + 1, ntile - 1));
                    return;
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
                u32x4 p[US], p2[TERMS == 2 ? US : 1];
                const auto weight = [&](auto qc) __attribute__((always_inline)) {
                    constexpr int w = decltype(qc)::value;     // of 8 NS pairs
                    const float x = __builtin_amdgcn_exp2f(
                        __builtin_fmaf(s[w / 8][w % 8 * 2], a.scale, -base));
                    const float y = __builtin_amdgcn_exp2f(
                        __builtin_fmaf(s[w / 8][w % 8 * 2 + 1], a.scale, -base));
                    const uint32_t both = pack_bf16(x, y);
                    p[w / 4][w % 4] = both;
                    if constexpr (TERMS == 2) {
                        l += x + y;
                        p2[w / 4][w % 4] = pack_bf16(x - __uint_as_float(both << 16),
                                                     y - __uint_as_float(both & 0xFFFF0000u));
                    } else {
                        l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, both),
                                                            bf16x2{1.0f, 1.0f}, l, false);
                    }
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
                            load(next, std::integral_constant<int, z / 2>{}, min(tile + SETS + 1, ntile - 1));
                        static_assert(2 * NU <= US * F, "loads between the products");
                        __builtin_amdgcn_sched_barrier(0);
                        const bf16x8 v = __builtin_bit_cast(
                            bf16x8, u32x4{fv[z & 1][0][0], fv[z & 1][0][1], fv[z & 1][1][0], fv[z & 1][1][1]});
                        o[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, p[u]),
                                                                       o[f], 0, 0, 0);
                        if constexpr (TERMS == 2)
                            o[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                                v, __builtin_bit_cast(bf16x8, p2[u]), o[f], 0, 0, 0);
                        __builtin_amdgcn_sched_barrier(0);
                    }(), ...);
                }(std::make_integer_sequence<int, US * F>{});
            };
            for (int tile = 0; tile < ntile; tile += 2) {
                step(even, odd, tile);
                if (tile + 1 < ntile)
                    step(odd, even, tile + 1);
            }
        }

        const u32x2 ls = both_halves(l);
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
        float *const part = plan.part + (slot * kRows + row - job.note.tile * kRows) * (D + 4);
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const bool nan = row_nan >> f & 1;
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int d = 32 * f + 2 * i + 4 * h;
                f32x4 v = {o[f][i], o[f][i + 1], o[f][i + 2], o[f][i + 3]};
                if (nan)
                    v = f32x4{NAN, NAN, NAN, NAN};
                if (job.note.used == 1)
                    store_outputs(a.out + out_row * D + d, v, inv);
                else
                    *reinterpret_cast<f32x4 *>(part + d) = v;
            }
        }
        if (job.note.used > 1 && h == 0)
            *reinterpret_cast<f32x4 *>(part + D) = f32x4{m, l, 0.0f, 0.0f};
    };
    if (rows - job.note.tile * kRows <= kRows / 2)
        run(std::integral_constant<int, 2>{});
    else
        run(std::integral_constant<int, 4>{});
}

// Joins the pieces of a row tile with weights 2^(m_s - max m): D / 4 lanes hold a row's outputs. Few
// pieces: a row a group of lanes; many: the groups take a row's pieces in turn and meet in LDS.
// gridDim.y workgroups share a tile's rows.
constexpr int kFewPieces = 16;

struct Part {
    float m, l;
    f32x4 v;
    // piece p of a row, outputs d .. d + 3
    __device__ __forceinline__ void add(const float *p, int dim, int d) {
        const f32x4 ml = *reinterpret_cast<const f32x4 *>(p + dim);
        add(ml[0], ml[1], *reinterpret_cast<const f32x4 *>(p + d));
    }
    __device__ __forceinline__ void add(float m2, float l2, const f32x4 &v2) {
        const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top;
        const float keep = __builtin_amdgcn_exp2f(m - base), w = __builtin_amdgcn_exp2f(m2 - base);
        m = top;
        l = l * keep + l2 * w;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = v[e] * keep + v2[e] * w;
    }
};

template <int D>
__global__ void __launch_bounds__(256)
kv_tree_join_kernel(KvShape c, KvAttnArgs a, TreePlan plan) {
    constexpr int LANES = D / 4, GROUPS = 256 / LANES;
    __shared__ f32x4 other_v[GROUPS][LANES];
    __shared__ float other_m[GROUPS], other_l[GROUPS];
    const Note job = plan.notes[1 + blockIdx.x];
    if ((int)blockIdx.x >= plan.notes[0].used || job.used <= 1)
        return;
    // With lengths that no call may have (sequences that overlap) there can be more pieces than a grid
    // has, and notes that nobody wrote: nothing outside the buffers is touched for them either.
    if ((unsigned)job.b >= (unsigned)a.seqs || (unsigned)job.head >= (unsigned)c.heads || job.slot < 0 ||
        job.stride < 1 || job.used > plan.slots ||
        job.slot + (int64_t)(job.used - 1) * job.stride >= plan.slots)
        return;
    const Seq seq = sequence(c, a, job.b);
    if ((unsigned)job.tile >= (unsigned)tiles_of(rows_of(a, seq)))
        return;
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES, d = 4 * lane;
    const int rows = min(seq.lq * a.group - job.tile * kRows, kRows), q_heads = c.heads * a.group;
    const float *first = plan.part + (int64_t)job.slot * kRows * (D + 4);
    const int64_t stride = (int64_t)job.stride * kRows * (D + 4);
    const auto store = [&](int r, const Part &x) {
        const int row = job.tile * kRows + r, qi = row / a.group;
        const int64_t out_row = (seq.q0 + qi) * q_heads + job.head * a.group + row - qi * a.group;
        store_outputs(a.out + out_row * D + d, x.v, inverse(x.l, x.m));
    };
    if (job.used <= kFewPieces) {
        if (group >= GROUPS)
            return;
        for (int r = blockIdx.y * GROUPS + group; r < rows; r += gridDim.y * GROUPS) {
            Part x = {-INFINITY, 0.0f, {}};
            const float *p = first + r * (D + 4);
#pragma unroll 4
            for (int s = 0; s < job.used; ++s)
                x.add(p + s * stride, D, d);
            store(r, x);
        }
        return;
    }
    for (int r = blockIdx.y; r < rows; r += gridDim.y) {
        Part x = {-INFINITY, 0.0f, {}};
        const float *p = first + r * (D + 4);
        if (group < GROUPS) {
#pragma unroll 4
            for (int s = group; s < job.used; s += GROUPS)
                x.add(p + s * stride, D, d);
            other_v[group][lane] = x.v;
            if (lane == 0) {
                other_m[group] = x.m;
                other_l[group] = x.l;
            }
        }
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int g = 1; g < GROUPS; ++g)
                x.add(other_m[g], other_l[g], other_v[g][lane]);
            store(r, x);
        }
        __syncthreads();
    }
}

// Row tiles that T queries in sequences can make, whatever each has of them.
int64_t blocks_of(const KvShape &c, int64_t T, int seqs, int group) {
    return c.heads * (T * group / kRows + std::min<int64_t>(seqs, T));
}

// Up to here keys stay whole: a second launch costs as much as it saves.
constexpr int kWholeTokens = 512;
// And up to here where row tiles alone make four rounds of what runs at once: lengths even out, and parts
// are written and read for nothing. us divided and whole, 4 queries a head, heads of 128, lengths up to
// 2000: 512 x 16 nodes, 8 heads 276, 229; 256 x 16 150, 135; 200 x 60 184, 164; with two rounds 128 x 16
// of up to 8000 187, 248. Longer sequences stay divided: one of them among short ones would run alone.
constexpr int kFullTokens = 4096;

TreePlan plan_of(const KvShape &c, int64_t T, int seqs, int group, int max_kv) {
    TreePlan p;
    const int64_t blocks = blocks_of(c, T, seqs, group);
    const int at_once = c.dim <= 128 ? 512 : 256;
    const bool full = blocks > 4 * at_once && max_kv <= kFullTokens;
    const bool divided = max_kv > kWholeTokens && seqs <= kSummed && !full;
    // What runs at once: two workgroups a CU, one above 128 channels. us with 384, 512 and 768: 32 trees
    // of 60 on 8192 326, 325, 353; 201 nodes on 40001 202, 220, 195 (168 once pieces fit one round).
    p.target = divided ? at_once : 0;
    // 13 nodes on 2001 tokens: pieces of 128, 256 at least 13.6, 18.7.
    p.least = 128;
    // Pieces there can be: a row tile has its cost / share, rounded up, so all have one each and
    // the call's cost / share together, which with a share of three quarters of cost / target is 4 / 3
    // of the target (and some for the roundings of these floats).
    const int64_t numbers = c.heads * (T * group / kRows + seqs);          // as find_tile counts
    p.grid = (int)std::min<int64_t>(divided ? blocks + p.target + p.target / 2 : numbers, INT32_MAX / 2);
    // A divided row tile has a cost of more than one share (x shares make ceil(x) pieces), so there are
    // at most 4 / 3 of the target of them, and as ceil(x) < 2 x above 1, 8 / 3 of it pieces: both rounded up,
    // which is more than the floats are off. So the workspace does not grow with the call: 92 MB at 128
    // channels. With a slot a piece of every row tile 512 trees of 60 nodes took 848 MB.
    p.tiles = (int)std::min<int64_t>(blocks, (4 * p.target + 2) / 3);
    p.slots = std::min(p.grid, (8 * p.target + 2) / 3);
    const uint32_t pb = (uint32_t)c.page / 16;
    p.magic = (((uint64_t)1 << 32) + pb - 1) / pb;
    p.notes = nullptr;
    p.part = nullptr;
    return p;
}

size_t notes_bytes(const TreePlan &p) { return (1 + (size_t)p.tiles) * sizeof(Note); }

// Calls whose sequences have few rows go to kv_attention.hip's kernel that reads keys straight into
// matrix registers, 16 rows a workgroup: up to 16, above 128 channels, where one workgroup of this file's
// fills a CU, up to 32. us there and here: 42 x 6 rows on 1088 tokens, 18 heads of 256, 99 and 159; 32 x
// 16 on up to 8192, 8 heads of 128, 55 and 62, with 32 rows 60 and 60, all 8192 long 212 and 135.
//
// That kernel has a part for every row of the call in each of its splits, 68 MB at most where T is what the
// sequences have, but without end where the call is laid out for more: 4 sequences of 4 nodes on 131072
// tokens in 8192 rows 17.7 GB. Those go to this file's: in 16 rows (there) 204 us, in 1024 (here) 246, on
// 8192 tokens 30 and 30, with heads of 256 43 and 54.
constexpr size_t kFewBytes = size_t(1) << 27;

bool few_rows(const KvShape &c, int64_t T, int seqs, int group, int max_q, int max_kv) {
    return (seqs == 1 ? T : std::min<int64_t>(max_q, T)) * group <= (c.dim <= 128 ? 16 : 32) &&
           kv_attention_workspace_bytes(c, T, seqs, group, max_q, max_kv) <= kFewBytes;
}

}  // namespace

size_t kv_tree_workspace_bytes(const KvShape &c, int64_t T, int seqs, int group, int max_q, int max_kv) {
    if (few_rows(c, T, seqs, group, max_q, max_kv))
        return kv_attention_workspace_bytes(c, T, seqs, group, max_q, max_kv);
    const TreePlan p = plan_of(c, T, seqs, group, max_kv);
    return p.target == 0 ? 0 : notes_bytes(p) + (size_t)p.slots * kRows * (c.dim + 4) * 4;
}

hipError_t launch_kv_tree(const KvShape &c, const KvAttnArgs &a, void *ws, hipStream_t s) {
    if (a.T * c.heads * a.group > INT32_MAX)
        return hipErrorInvalidValue;
    if (few_rows(c, a.T, a.seqs, a.group, a.max_q, a.max_kv))
        return launch_kv_attention(c, a, ws, s);
    TreePlan plan = plan_of(c, a.T, a.seqs, a.group, a.max_kv);
    plan.notes = static_cast<Note *>(ws);
    plan.part = reinterpret_cast<float *>(static_cast<uint8_t *>(ws) + notes_bytes(plan));
    if (!launchable(plan.grid, 256))
        return hipErrorInvalidValue;
    // The join's workgroups a row tile: a row a group of lanes, or, with few tiles, a row each.
    const int join_parts = std::max(16, std::min(128, 8192 / std::max(plan.tiles, 1)));
    const auto run = [&](auto dim, auto format) {
        constexpr int F = decltype(format)::value, D = decltype(dim)::value;
        hipLaunchKernelGGL((kv_tree_kernel<F, D>), dim3((unsigned)plan.grid), dim3(256), 0, s, c, a, plan);
        if (plan.target > 0 && hipPeekAtLastError() == hipSuccess)
            hipLaunchKernelGGL((kv_tree_join_kernel<D>), dim3((unsigned)plan.tiles, (unsigned)join_parts),
                               dim3(256), 0, s, c, a, plan);
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
