// Microscaled 4-bit product: Y[m][n] = bf16(sum_k X[m][k] W[n][k] + b[n]) on the codes and
// scale bytes of mx4_quant.hip, with float32 accumulation in the scaled matrix instructions.
//
// v_mfma_scale_f32_32x32x64 with e2m1 operands takes 16 bytes (a block of 32 elements) of one
// row and its scale byte from every lane: lane l holds row l % 32 and K-half l / 32. A dot
// product is unchanged by a permutation of K that both operands share, so inside a K-panel of
// 256 channels (8 blocks, 128 bytes of codes a row) K-half h takes blocks 4h .. 4h + 3 in
// steps 0 .. 3: the four scale bytes of a lane are then one word of the scales' layout, and
// each step selects its byte of that word.
//
// Many tokens: bound by the matrix cores at the clock that their power leaves (1.6 GHz on
// random codes, 6.4 PFLOP/s from registers; 2.3 GHz and 9.1 on zeros) and by waits for panels.
// 4608 x 4096 x 16384 takes 156 to 166 us on different cards (3.7 to 4.0 PFLOP/s), 4608 x 16384 x
// 4096 in one round of tiles 138 (4.5). Few tokens: bound by reading W; 1 x 4096 x 16384 takes 10 us
// (3.6 TB/s) with its quantizer.
#include "../../include/w8a8.h"
#include "mx_internal.hpp"
#include "mx_quant.hpp"

#include <algorithm>
#include <utility>

namespace w8a8 {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kRsrcWord3 = 0x00020000;     // raw 32-bit buffer
constexpr uint32_t kOOB = 0x7FFFFFF0;      // beyond any buffer: the load gives zero
constexpr int kPanel = 128;                // bytes of codes of a row in a K-panel

// Offset `at` moved on by some rows, forwards or back; from kOOB it stays beyond the buffer, for
// which a sum may pass 2^31 but never 2^32.
__host__ __device__ constexpr uint32_t rows_on(uint32_t at, int rows, int row_bytes) {
    return at + (uint32_t)(rows * row_bytes);
}
constexpr int kMostRowBytes = W8A8_MX4_MAX_K / 32 * 16;

__device__ __forceinline__ i32x8 frag(i32x4 v) {
    return i32x8{v[0], v[1], v[2], v[3], 0, 0, 0, 0};
}

// XOR of the 16-byte chunk index inside an LDS row of 128 bytes: spreads the direct-to-LDS writes
// (8 rows of 8 chunks) and the fragment reads (32 rows, one chunk) over the banks. Not all the way:
// 15% of the LDS cycles of 4608 x 4096 x 16384 are bank conflicts, by the counters; which accesses
// have them they do not tell.
__device__ __forceinline__ int swz(int row) { return (row & 7) ^ ((row >> 3) & 3); }

__host__ __device__ constexpr int waitcnt_vm(int n) {
    return (n & 0xF) | ((n >> 4) << 14) | (0x7 << 4) | (0xF << 8);
}

// Barrier without the fence of __syncthreads(), which would wait for all loads in flight.
__device__ __forceinline__ void barrier_nofence() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
}

struct Mx4Params {
    Mx4Args a;
    int tiles_m, tiles_n, gm;   // tiles, token tiles per raster group
    int splits, split_panels;   // K divided among workgroups: panels of each
    int vec;                    // rows of y 16-byte aligned: N % 8 == 0 and y aligned
    float *part;                // splits > 1: [splits][M][N]
};

// Tile (and K-range) of workgroup `bid`: each XCD takes every 8th workgroup and gets a
// contiguous run of tiles, K-ranges outermost, in groups of gm token tiles.
__device__ __forceinline__ void tile_of(int bid, const Mx4Params &p, int &tm, int &tn, int &split) {
    // Divisions run in vector registers; the results are made scalar again, or the buffer
    // descriptors that they lead to would be taken for different ones in each lane.
    const auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    const int tiles = p.tiles_m * p.tiles_n, total = tiles * p.splits;
    const int xcd = bid & 7, slot = bid >> 3, q = total >> 3, r = total & 7;
    int t = xcd * q + min(xcd, r) + slot;
    split = uniform(t / tiles);
    t -= split * tiles;
    const int per = p.gm * p.tiles_n, group = uniform(t / per), first = group * p.gm;
    const int in = t - group * per, size = min(p.tiles_m - first, p.gm);
    tn = uniform(in / size);
    tm = first + in - tn * size;
}

// One workgroup per TM tokens x TN channels; WM x WN wavefronts, S LDS stages of a K-panel:
// codes of TN weight rows and TM token rows, then their scale words (8 bytes a row). Codes
// and scales go from memory to LDS directly; what lies past a matrix reads as zero codes and
// zero scales. Panel k + S - 1 is requested while panel k is multiplied.
//
// Eight to twelve wavefronts on the large tiles: a product's operands are two LDS reads, and
// with one wavefront a SIMD their latencies show. 256 x 256 by four, whose fragments were read a
// step ahead across four stages of half panels, took 214 us at 4608 x 4096 x 16384 (288 x 256
// by twelve on the same card: 160) and 258 at 4608 x 16384 x 4096 (138).
template <int TM, int TN, int WM, int WN, int S>
__global__ void __launch_bounds__(WM *WN * 64)
mx4_gemm_kernel(Mx4Params p) {
    constexpr int NW = WM * WN;
    constexpr int WTM = TM / WM, WTN = TN / WN, FM = WTM / 32, FN = WTN / 32;
    constexpr int ROWS = TN + TM;
    constexpr int CODES = ROWS * kPanel, STAGE = CODES + ROWS * 8;
    // Loads of a panel, NV to a wavefront: 8 rows of codes each, then SR rows of scales each.
    constexpr int SB = TN % 128 == 0 && TM % 128 == 0 ? 16 : 4, SR = 64 * SB / 8;
    constexpr int IW = TN / 8, IC = ROWS / 8, NI = IC + ROWS / SR, NV = (NI + NW - 1) / NW;
    static_assert(WTM % 32 == 0 && WTN % 32 == 0 && NW % 4 == 0, "tile");
    static_assert(TN % SR == 0 && TM % SR == 0, "scale loads");
    static_assert(S >= 2 && (S - 1) * NV <= 63, "loads in flight");
    // From kOOB, the longest rows: neither the last load of a stage nor the first of its tokens'
    // rows lands in a buffer of TM or TN rows.
    static_assert(rows_on(kOOB, NV * NW * 8, kMostRowBytes) > kOOB &&
                      rows_on(kOOB, -TN, kMostRowBytes) > (uint32_t)(TM > TN ? TM : TN) * kMostRowBytes,
                  "beyond the buffers");
    constexpr int RS = 2 * WTN + 16;       // output staging: bytes of a token's row
    static_assert(NW * 32 * RS <= S * STAGE && S * STAGE + TN * 4 <= 163840, "LDS");
    __shared__ __attribute__((aligned(1024))) uint8_t smem[S * STAGE + TN * 4];
    float *const bias = reinterpret_cast<float *>(smem + S * STAGE);

    const Mx4Args &a = p.a;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    int tm, tn, split;
    tile_of(blockIdx.x, p, tm, tn, split);
    const int64_t m0 = (int64_t)tm * TM, n0 = (int64_t)tn * TN;
    const int rows_x = (int)min(a.M - m0, (int64_t)TM), rows_w = (int)min(a.N - n0, (int64_t)TN);
    const int row_bytes = (int)a.nb * 16;
    const int first_panel = split * p.split_panels;
    const int nk = min((int)((a.nb + 7) / 8) - first_panel, p.split_panels);
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(
        (void *)(a.wq + n0 * row_bytes), (short)0, rows_w * row_bytes, kRsrcWord3);
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(
        (void *)(a.xq + m0 * row_bytes), (short)0, rows_x * row_bytes, kRsrcWord3);

    f32x16 acc[FN][FM];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j)
            acc[i][j] = f32x16{};

    // Load i of this wavefront is number i NW + wave (the last one again past it: the same
    // bytes to the same place). Codes: rows 8n + lane / 8 of the stage, physical chunk lane % 8,
    // and so chunk (lane % 8) ^ swz(row) of the row, the same for all i as NW % 4 == 0.
    const int lrow = wave * 8 + (lane >> 3);
    const int lchunk = ((lane & 7) ^ swz(lrow)) << 4;
    // Where panel kt's codes start for this lane; beyond the buffers past the last panel and
    // past the rows' ends.
    const auto codes_at = [&](int kt) {
        const int k = (first_panel + kt) * kPanel + lchunk;
        return kt < nk && k < row_bytes ? (uint32_t)(lrow * row_bytes + k) : kOOB;
    };
    const auto issue = [&](auto ic, int kt, uint32_t at, int so) __attribute__((always_inline)) {
        constexpr int i = decltype(ic)::value;
        const int n = i * NW + NW <= NI ? i * NW + wave : min(i * NW + wave, NI - 1);
        if (i * NW + NW <= IC || n < IC) {
            const bool w = i * NW + NW <= IW || (i * NW < IW && n < IW);
            uint8_t *dst = smem + so + n * 1024;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                w ? rw : rx, (__attribute__((address_space(3))) void *)dst, 16,
                (int)rows_on(at, i * NW * 8 - (w ? 0 : TN), row_bytes), 0, 0, 0);
        } else {
            const int row = (n - IC) * SR;             // of the stage's scale words
            const bool w = row < TN, in = kt < nk;     // past the last panel: an empty buffer
            const int64_t rows = w ? a.N : a.M, r0 = w ? n0 + row : m0 + row - TN;
            const int left = (w ? rows_w : rows_x + TN) - row;
            const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
                (void *)((w ? a.ws : a.xs) + ((in ? first_panel + kt : 0) * rows + r0) * 8), (short)0,
                in ? max(left, 0) * 8 : 0, kRsrcWord3);
            uint8_t *dst = smem + so + CODES + (n - IC) * 64 * SB;
            if constexpr (SB == 16)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    rs, (__attribute__((address_space(3))) void *)dst, 16, lane * 16, 0, 0, 0);
            else
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    rs, (__attribute__((address_space(3))) void *)dst, 4, lane * 4, 0, 0, 0);
        }
    };

    // Fragment reads: lane (r, h) of step s takes chunk 4h + s of its row.
    int fofs[4];
    {
        const int r = lane & 31, h = lane >> 5;
#pragma unroll
        for (int s = 0; s < 4; ++s)
            fofs[s] = r * kPanel + (((4 * h + s) ^ swz(r)) << 4);
    }
    const int sofs = (lane & 31) * 8 + (lane >> 5) * 4;
    i32x4 fa[2][FN], fb[2][FM];
    int sa[FN], sb[FM];

    // Step s of the panel at so: its MFMAs, between them the reads of step s + 1 and the
    // panel's share of the loads of panel kt + S - 1.
    constexpr int NM = FN * FM, NR = FN + FM;
    const auto read_frag = [&](int q, int so, int s) __attribute__((always_inline)) {
        if (q < FN)
            fa[s & 1][q] = *reinterpret_cast<const i32x4 *>(smem + so + (wn * WTN + q * 32) * kPanel +
                                                            fofs[s]);
        else
            fb[s & 1][q - FN] = *reinterpret_cast<const i32x4 *>(
                smem + so + (TN + wm * WTM + (q - FN) * 32) * kPanel + fofs[s]);
    };
    // With two stages all loads go out in the first step, else a quarter in each.
    constexpr int VPS = S == 2 ? NV : (NV + 3) / 4;
    const auto step = [&](auto sc, int so, int kt, uint32_t at, int so_load) __attribute__((always_inline)) {
        constexpr int s = decltype(sc)::value;
        constexpr int nr = s < 3 ? NR : 0;
        constexpr int va = s * VPS < NV ? s * VPS : NV, vb = va + VPS < NV ? va + VPS : NV;
        constexpr int nops = nr + vb - va, steps = NM > nops ? NM : nops;
        [&]<int... q>(std::integer_sequence<int, q...>) __attribute__((always_inline)) {
            ([&]() __attribute__((always_inline)) {
                if constexpr (q < nr)
                    read_frag(q, so, s + 1);
                else if constexpr (q < nops)
                    issue(std::integral_constant<int, va + q - nr>{}, kt, at, so_load);
                if constexpr (q < NM) {
                    __builtin_amdgcn_sched_barrier(0);
                    acc[q / FM][q % FM] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                        frag(fa[s & 1][q / FM]), frag(fb[s & 1][q % FM]), acc[q / FM][q % FM], 4, 4, s,
                        sa[q / FM], s, sb[q % FM]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }(), ...);
        }(std::make_integer_sequence<int, steps>{});
    };

    // The tile's bias, read behind the first panels.
    constexpr int NB = (TN + NW * 64 - 1) / (NW * 64);
    float tile_bias[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const int n = i * NW * 64 + (int)threadIdx.x;
        tile_bias[i] = a.bias && n < rows_w ? __uint_as_float((uint32_t)a.bias[n0 + n] << 16) : 0.0f;
    }
    const auto park_bias = [&]() {
#pragma unroll
        for (int i = 0; i < NB; ++i)
            if (i * NW * 64 + (int)threadIdx.x < TN)
                bias[i * NW * 64 + threadIdx.x] = tile_bias[i];
    };
    if (nk > 0) {
#pragma unroll
        for (int k = 0; k < S - 1; ++k)
            [&]<int... i>(std::integer_sequence<int, i...>) __attribute__((always_inline)) {
                (issue(std::integral_constant<int, i>{}, k, codes_at(k), k * STAGE), ...);
            }(std::make_integer_sequence<int, NV>{});
        park_bias();
        int st = 0, ld = S - 1;
        for (int kt = 0; kt < nk; ++kt) {
            // Panel kt has landed once at most the S - 2 younger ones are in flight; every
            // wavefront has then read the stage that the next loads go to.
            __builtin_amdgcn_s_waitcnt(waitcnt_vm((S - 2) * NV));
            barrier_nofence();
            const int so = st * STAGE;
#pragma unroll
            for (int i = 0; i < FN; ++i)
                sa[i] = *reinterpret_cast<const int *>(smem + so + CODES + (wn * WTN + i * 32) * 8 + sofs);
#pragma unroll
            for (int j = 0; j < FM; ++j)
                sb[j] = *reinterpret_cast<const int *>(smem + so + CODES +
                                                       (TN + wm * WTM + j * 32) * 8 + sofs);
#pragma unroll
            for (int q = 0; q < NR; ++q)
                read_frag(q, so, 0);
            __builtin_amdgcn_sched_barrier(0);
            const int kl = kt + S - 1, lo = ld * STAGE;
            const uint32_t at = codes_at(kl);
            step(std::integral_constant<int, 0>{}, so, kl, at, lo);
            step(std::integral_constant<int, 1>{}, so, kl, at, lo);
            step(std::integral_constant<int, 2>{}, so, kl, at, lo);
            step(std::integral_constant<int, 3>{}, so, kl, at, lo);
            st = st + 1 == S ? 0 : st + 1;
            ld = ld + 1 == S ? 0 : ld + 1;
        }
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
        __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
    }

    const int64_t mw = m0 + wm * WTM, nw = n0 + wn * WTN;
    const int r = lane & 31, h = lane >> 5;
    if (p.splits > 1) {
        // Lane (r, h) of fragment (i, j): token 32j + r, channels 32i + 8g + 4h + 0 .. 3.
        float *out = p.part + (int64_t)split * a.M * a.N;
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            const int64_t m = mw + j * 32 + r;
            if (m >= a.M)
                continue;
#pragma unroll
            for (int i = 0; i < FN; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int64_t n = nw + i * 32 + g * 8 + h * 4;
                    float *o = out + m * a.N + n;
                    if (n + 4 <= a.N && a.N % 4 == 0) {
                        *reinterpret_cast<f32x4 *>(o) =
                            f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2],
                                  acc[i][j][4 * g + 3]};
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (n + e < a.N)
                                o[e] = acc[i][j][4 * g + e];
                    }
                }
        }
        return;
    }

    // Output: 32 tokens at a time through the wavefront's own piece of LDS (free now), so
    // that stores are whole 16-byte pieces of rows.
    if (nk <= 0)
        park_bias();
    __syncthreads();
    constexpr int CPR = WTN / 8, RPQ = 64 / CPR, NQ = (32 + RPQ - 1) / RPQ;
    constexpr bool EXACT = RPQ * CPR == 64 && NQ * RPQ == 32;
    uint8_t *const region = smem + wave * 32 * RS;
    const int row0 = lane / CPR, ch = lane % CPR;
    const int64_t n_lane = nw + ch * 8;
    uint16_t *const out = a.y + (mw + row0) * a.N + n_lane;
    const bool whole = p.vec && mw + WTM <= a.M && nw + WTN <= a.N;
#pragma unroll
    for (int j = 0; j < FM; ++j) {
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 b =
                    *reinterpret_cast<const f32x4 *>(bias + wn * WTN + i * 32 + g * 8 + h * 4);
                uint16_t v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = __builtin_bit_cast(uint16_t, (__bf16)(acc[i][j][4 * g + e] + b[e]));
                *reinterpret_cast<uint2 *>(region + r * RS + (i * 32 + g * 8 + h * 4) * 2) =
                    make_uint2(v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16);
            }
        u32x4 v[NQ];
        const auto live = [&](int q) { return EXACT || (row0 < RPQ && row0 + q * RPQ < 32); };
#pragma unroll
        for (int q = 0; q < NQ; ++q)
            if (live(q))
                v[q] = *reinterpret_cast<const u32x4 *>(region + (row0 + q * RPQ) * RS + ch * 16);
        if (whole) {
#pragma unroll
            for (int q = 0; q < NQ; ++q)
                if (live(q))
                    __builtin_nontemporal_store(
                        v[q], reinterpret_cast<u32x4 *>(out + (int64_t)(j * 32 + q * RPQ) * a.N));
            continue;
        }
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            if (!live(q) || mw + j * 32 + row0 + q * RPQ >= a.M || n_lane >= a.N)
                continue;
            uint16_t *o = out + (int64_t)(j * 32 + q * RPQ) * a.N;
            if (n_lane + 8 <= a.N) {
                *reinterpret_cast<Bytes16 *>(o) = __builtin_bit_cast(Bytes16, v[q]);
            } else {
                for (int e = 0; e < 7; ++e)
                    if (n_lane + e < a.N)
                        o[e] = (uint16_t)(v[q][e >> 1] >> (16 * (e & 1)));
            }
        }
    }
}

// Sums the K-ranges in order and adds the bias: four outputs a thread where rows allow.
template <bool VEC>
__global__ void __launch_bounds__(256)
mx4_reduce_kernel(Mx4Params p) {
    const Mx4Args &a = p.a;
    const int64_t MN = a.M * a.N, t = ((int64_t)blockIdx.x * 256 + threadIdx.x) * (VEC ? 4 : 1);
    if (t >= MN)
        return;
    const int64_t n = t % a.N;
    if constexpr (VEC) {
        f32x4 v = *reinterpret_cast<const f32x4 *>(p.part + t);
        for (int s = 1; s < p.splits; ++s)
            v += *reinterpret_cast<const f32x4 *>(p.part + s * MN + t);
        uint16_t y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float b = a.bias ? __uint_as_float((uint32_t)a.bias[n + e] << 16) : 0.0f;
            y[e] = __builtin_bit_cast(uint16_t, (__bf16)(v[e] + b));
        }
        Bytes8 o;
        o.w[0] = y[0] | (uint32_t)y[1] << 16;
        o.w[1] = y[2] | (uint32_t)y[3] << 16;
        *reinterpret_cast<Bytes8 *>(a.y + t) = o;
    } else {
        float v = p.part[t];
        for (int s = 1; s < p.splits; ++s)
            v += p.part[s * MN + t];
        const float b = a.bias ? __uint_as_float((uint32_t)a.bias[n] << 16) : 0.0f;
        a.y[t] = __builtin_bit_cast(uint16_t, (__bf16)(v + b));
    }
}

// Few tokens (16 FMB): bound by reading W once, so nothing of it is staged. A workgroup owns
// 16 FNB channels; its NW wavefronts take K in turn, 512 channels (256 bytes, 16 blocks) at a
// time, with the next 512 channels' loads in flight. v_mfma_scale_f32_16x16x128: lane (r, g) =
// (lane % 16, lane / 16) holds row r; in step s of four it takes block 4s + g, so that a load
// instruction reads whole 64-byte pieces of rows, and byte g of a scale word. The wavefronts'
// sums meet in LDS, added in their order.
//
// QX: the tokens are bf16 rows (transformed as in the quantizer), which the workgroup quantizes
// into LDS while its first weights are on their way; the whole linear is then this one launch.
// Every workgroup quantizes them again, so the host allows it for few tokens x channels only.
// LDS rows are an odd number of 16-byte blocks apart: the 16 rows of a read then lie in
// different banks.
template <int FMB, int FNB, int NW, bool QX, int ACT, bool CM>
__global__ void __launch_bounds__(NW * 64)
mx4_stream_kernel(Mx4Args a, const uint16_t *x, int64_t K, const float *col_mul) {
    using namespace mx;
    static_assert(!QX || FMB == 1);
    __shared__ f32x4 red[NW][FNB * FMB][64];
    extern __shared__ __attribute__((aligned(16))) uint8_t tokens[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * (16 * FNB);
    const int M = (int)a.M, nb = (int)a.nb, panels = (nb + 7) / 8;

    // Rows past the matrices repeat the last one; their results are not stored.
    const uint8_t *wrow[FNB], *wscale[FNB];
#pragma unroll
    for (int c = 0; c < FNB; ++c) {
        const int64_t n = min(n0 + c * 16 + r, a.N - 1);
        wrow[c] = a.wq + n * nb * 16;
        wscale[c] = a.ws + n * 8;
    }
    f32x4 acc[FNB][FMB];
#pragma unroll
    for (int c = 0; c < FNB; ++c)
#pragma unroll
        for (int f = 0; f < FMB; ++f)
            acc[c][f] = f32x4{};

    i32x4 w[FNB][4], fx[FMB][4];
    uint2 sw[FNB][2], sx[FMB][2];
    int token_scale[4];
    const auto load = [&](int j) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < FNB; ++c) {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int blk = 16 * j + 4 * s + g;
                w[c][s] = blk < nb ? *reinterpret_cast<const i32x4 *>(wrow[c] + (int64_t)blk * 16)
                                   : i32x4{};
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
                sw[c][h] = 2 * j + h < panels
                               ? *reinterpret_cast<const uint2 *>(wscale[c] + (2 * j + h) * a.N * 8)
                               : make_uint2(0, 0);
        }
        if constexpr (!QX) {
#pragma unroll
            for (int f = 0; f < FMB; ++f) {
                const int m = min(f * 16 + r, M - 1);
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const int blk = min(16 * j + 4 * s + g, nb - 1);   // against zero weights past nb
                    fx[f][s] = *reinterpret_cast<const i32x4 *>(a.xq + ((int64_t)m * nb + blk) * 16);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    sx[f][h] = 2 * j + h < panels ? *reinterpret_cast<const uint2 *>(
                                                        a.xs + ((int64_t)(2 * j + h) * M + m) * 8)
                                                  : make_uint2(0, 0);
            }
        }
    };
    const int steps = (nb + 15) / 16;
    if (wave < steps)
        load(wave);
    const int stride = (nb | 1) * 16;
    uint8_t *const token_scales = tokens + M * stride;
    if constexpr (QX) {
        __shared__ __attribute__((aligned(16))) float gelu[ACT == ACT_GELU ? sizeof(GeluTable) / 4 : 1];
        if constexpr (ACT == ACT_GELU) {
            for (int i = threadIdx.x; i < (int)(sizeof(GeluTable) / 16); i += NW * 64)
                reinterpret_cast<float4 *>(gelu)[i] = reinterpret_cast<const float4 *>(&kGeluTable)[i];
            __syncthreads();
        }
        // A lane quantizes 8 channels, four lanes a block.
        for (int u = threadIdx.x; u < M * nb * 4; u += NW * 64) {
            const int row = u / (nb * 4), q = u - row * (nb * 4);
            float c[8];
            if constexpr (CM)
                load_multipliers(col_mul, 8 * q, K, c);
            uint32_t v[4], byte;
            load8(x + row * K, 8 * q, K, v);
            const uint32_t codes = quantize_quad<ACT, CM>(v, c, gelu, byte);
            *reinterpret_cast<uint32_t *>(tokens + row * stride + q * 4) = codes;
            if (q % 4 == 0)
                token_scales[row * nb + q / 4] = (uint8_t)byte;
        }
        __syncthreads();
    }
    for (int j = wave; j < steps; j += NW) {
        if constexpr (QX) {
            const int m = min(r, M - 1);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int blk = min(16 * j + 4 * s + g, nb - 1);
                fx[0][s] = *reinterpret_cast<const i32x4 *>(tokens + m * stride + blk * 16);
                token_scale[s] = token_scales[m * nb + blk];
            }
        }
        i32x4 wc[FNB][4], xc[FMB][4];
        int sc[FNB][4], xsc[FMB][4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
#pragma unroll
            for (int f = 0; f < FMB; ++f) {
                xc[f][s] = fx[f][s];
                xsc[f][s] = QX ? token_scale[s] : (int)((s & 1 ? sx[f][s / 2].y : sx[f][s / 2].x) >> (8 * g));
            }
#pragma unroll
            for (int c = 0; c < FNB; ++c) {
                wc[c][s] = w[c][s];
                sc[c][s] = (int)((s & 1 ? sw[c][s / 2].y : sw[c][s / 2].x) >> (8 * g));
            }
        }
        if (j + NW < steps)
            load(j + NW);
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int f = 0; f < FMB; ++f)
#pragma unroll
                for (int c = 0; c < FNB; ++c)
                    acc[c][f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        frag(wc[c][s]), frag(xc[f][s]), acc[c][f], 4, 4, 0, sc[c][s], 0, xsc[f][s]);
    }
#pragma unroll
    for (int c = 0; c < FNB; ++c)
#pragma unroll
        for (int f = 0; f < FMB; ++f)
            red[wave][f * FNB + c][lane] = acc[c][f];
    __syncthreads();
    // Lane (r, g) of a fragment holds token r, channels 4g .. 4g + 3.
    for (int i = threadIdx.x; i < FNB * FMB * 64; i += NW * 64) {
        const int l = i & 63, c = (i >> 6) % FNB, t = i / (FNB * 64) * 16 + (l & 15);
        f32x4 v = red[0][i >> 6][l];
#pragma unroll
        for (int k = 1; k < NW; ++k)
            v += red[k][i >> 6][l];
        const int64_t n = n0 + c * 16 + (l >> 4) * 4;
        if (t >= M)
            continue;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < a.N) {
                const float bias = a.bias ? __uint_as_float((uint32_t)a.bias[n + e] << 16) : 0.0f;
                a.y[t * a.N + n + e] = __builtin_bit_cast(uint16_t, (__bf16)(v[e] + bias));
            }
    }
}

// ---------------------------------------------------------------- what runs for a shape

// A workgroup of tile t takes start + panel * (its K-panels) microseconds alone. Each full round
// of 256 workgroups costs `more` of that (under 1 where two share a CU), the last one's share of
// the CUs `fill` (the clock falls as more of them work). Fitted to 245 random shapes (M 17 ..
// 8192, N 64 .. 20480, K 64 .. 24576) with every tile and 1 to 16 K-ranges: the choice is 1%
// slower than the best measured one in the geometric mean, 15% at most.
struct TileCost {
    int tm, tn;
    float start, panel, more, fill;
};
constexpr TileCost kTiles[] = {
    {288, 256, 5.36f, 1.48f, 1.30f, 0.35f}, {256, 256, 5.10f, 1.30f, 1.22f, 0.32f},
    {192, 256, 4.02f, 1.10f, 1.17f, 0.29f}, {128, 256, 3.14f, 0.70f, 1.21f, 0.54f},
    {128, 128, 2.90f, 0.475f, 1.07f, 0.43f}, {64, 128, 1.52f, 0.367f, 0.87f, 0.46f},
    {64, 64, 1.19f, 0.26f, 0.79f, 0.39f},
};
constexpr float kReduce = 4.4f, kReducePerMega = 1.33f;   // joining K-ranges: + per 10^6 partials
constexpr int kCus = 256;

// Fragments of 16 tokens for the streaming kernel, 0: a tile. It has no workgroups' partial sums
// to join, but reads every token from the L2 in each workgroup: it wins where one round of
// workgroups covers N, and where K is short for the second fragment. us, streaming and the best
// tile, K x N: 16 tokens 4096 x 4096 5.4, 7.7; 4096 x 8192 about 6.6, 8.0; 8192 x 8192 11.9,
// 15.2; 4096 x 16384 10.3, 9.4. 32 tokens 4096 x 4096 6.5, 7.8; 8192 x 1024 9.1, 8.1; 4096 x
// 6144 8.5, 8.2; 48 tokens 4096 x 4096 8.0, 8.1.
int stream_fragments(int64_t M, int64_t N, int64_t nb) {
    if (M <= 16)
        return N <= 8192 ? 1 : 0;
    return M <= 32 && N <= 4096 && nb <= 128 ? 2 : 0;
}

struct Plan {
    int tile, splits;
};

Plan plan_of(int64_t M, int64_t N, int64_t nb) {
    thread_local struct {
        int64_t M = -1, N, nb;
        Plan plan;
    } last;      // a pure function of the sizes: asked for several times in a call
    if (last.M == M && last.N == N && last.nb == nb)
        return last.plan;
    const int64_t panels = (nb + 7) / 8;
    Plan best = {0, 1};
    float least = INFINITY;
    for (int t = 0; t < (int)(sizeof(kTiles) / sizeof(kTiles[0])); ++t) {
        const TileCost &c = kTiles[t];
        const int64_t tiles = ((M + c.tm - 1) / c.tm) * ((N + c.tn - 1) / c.tn);
        for (int splits = 1; splits <= 16; splits *= 2) {
            if (splits > 1 && (tiles * splits > 2 * kCus || panels < 3 * splits))
                break;
            const int64_t blocks = tiles * splits, full = (blocks - 1) / kCus;
            const float last = (float)(blocks - full * kCus) / (float)kCus;
            float us = (c.start + c.panel * (float)((panels + splits - 1) / splits)) *
                       (1.0f + (float)full * c.more + last * c.fill);
            if (splits > 1)
                us += kReduce + kReducePerMega * (float)splits * (float)M * (float)N / 1e6f;
            if (us < least) {
                least = us;
                best = {t, splits};
            }
        }
    }
    last.M = M;
    last.N = N;
    last.nb = nb;
    last.plan = best;
    return best;
}

template <int TM, int TN, int WM, int WN, int S>
hipError_t run_tile(Mx4Params p, hipStream_t s) {
    p.tiles_m = (int)((p.a.M + TM - 1) / TM);
    p.tiles_n = (int)((p.a.N + TN - 1) / TN);
    p.gm = 8;
    const int64_t blocks = (int64_t)p.tiles_m * p.tiles_n * p.splits;
    if (!launchable(blocks, WM * WN * 64))
        return hipErrorInvalidValue;
    hipLaunchKernelGGL((mx4_gemm_kernel<TM, TN, WM, WN, S>), dim3((unsigned)blocks), dim3(WM * WN * 64), 0,
                       s, p);
    return hipGetLastError();
}

template <int FMB, bool QX, int ACT, bool CM>
hipError_t run_stream(const Mx4Args &a, const uint16_t *x, int64_t K, const float *cm, hipStream_t s) {
    const auto go = [&](auto kernel, int64_t channels, int waves) {
        const int64_t blocks = (a.N + channels - 1) / channels;
        if (!launchable(blocks, waves * 64))
            return hipErrorInvalidValue;
        const size_t lds = QX ? (size_t)(a.M * ((a.nb | 1) * 16 + a.nb)) : 0;
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(waves * 64), lds, s, a, x, K, cm);
        return hipGetLastError();
    };
    // A workgroup a CU. us for 16 tokens, K x N: 4096 x 4096 5.4 by 16 channels (32: 6.2), 4096 x
    // 6144 6.6 by 32 (7.6 by 16); one token through 4096 x 16384 9.9 with 4 wavefronts (8: 10.7).
    if (a.N <= 4096)
        return go(mx4_stream_kernel<FMB, 1, 8, QX, ACT, CM>, 16, 8);
    if constexpr (FMB == 1) {
        if (a.N <= 8192)
            return go(mx4_stream_kernel<1, 2, 8, QX, ACT, CM>, 32, 8);
        if constexpr (QX)
            return go(mx4_stream_kernel<1, 2, 4, QX, ACT, CM>, 32, 4);
    }
    return hipErrorInvalidValue;
}

}  // namespace

size_t mx4_gemm_workspace_bytes(int64_t M, int64_t N, int64_t nb) {
    if (stream_fragments(M, N, nb) != 0)
        return 0;
    const Plan p = plan_of(M, N, nb);
    return p.splits > 1 ? (size_t)p.splits * M * N * 4 : 0;
}

hipError_t launch_mx4_gemm(const Mx4Args &a, void *ws, hipStream_t s) {
    switch (stream_fragments(a.M, a.N, a.nb)) {
    case 1: return run_stream<1, false, ACT_NONE, false>(a, nullptr, 0, nullptr, s);
    case 2: return run_stream<2, false, ACT_NONE, false>(a, nullptr, 0, nullptr, s);
    default: break;
    }
    const Plan plan = plan_of(a.M, a.N, a.nb);
    const int64_t panels = (a.nb + 7) / 8;
    Mx4Params p;
    p.a = a;
    p.split_panels = (int)((panels + plan.splits - 1) / plan.splits);
    p.splits = p.split_panels > 0 ? (int)((panels + p.split_panels - 1) / p.split_panels) : 1;
    p.vec = a.N % 8 == 0 && reinterpret_cast<uintptr_t>(a.y) % 16 == 0;
    p.part = static_cast<float *>(ws);
    hipError_t e;
    switch (plan.tile) {
    case 0: e = run_tile<288, 256, 3, 4, 2>(p, s); break;
    case 1: e = run_tile<256, 256, 4, 2, 2>(p, s); break;
    case 2: e = run_tile<192, 256, 2, 4, 2>(p, s); break;
    case 3: e = run_tile<128, 256, 2, 4, 3>(p, s); break;
    case 4: e = run_tile<128, 128, 2, 2, 4>(p, s); break;
    case 5: e = run_tile<64, 128, 1, 4, 3>(p, s); break;
    default: e = run_tile<64, 64, 2, 2, 4>(p, s); break;
    }
    if (e != hipSuccess || p.splits <= 1)
        return e;
    const bool vec = a.N % 4 == 0;
    const int64_t blocks = (a.M * a.N / (vec ? 4 : 1) + 255) / 256;
    if (!launchable(blocks, 256))
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(vec ? mx4_reduce_kernel<true> : mx4_reduce_kernel<false>, dim3((unsigned)blocks),
                       dim3(256), 0, s, p);
    return hipGetLastError();
}

// The streaming kernel's workgroups each quantize all tokens again, 2 us for 16384 values on top
// of the product, as much as a launch of its own; past 8192 channels they do so in two rounds. us
// in one launch and in two, tokens x K x N: 4 x 4096 x 4096 6.0, 7.0; 6 x 4096 x 4096 7.0, 7.1;
// 6 x 2048 x 8192 6.3, 6.7; 2 x 4096 x 16384 10.7, 11.5; 4 x 4096 x 16384 12.2, 11.5.
bool mx4_linear_one_launch(int64_t M, int64_t N, int64_t K) {
    return M <= 16 && M * K <= (N <= 8192 ? 16384 : 8192);
}

hipError_t launch_mx4_linear(const Mx4Args &a, const uint16_t *x, int64_t K, int act,
                             const float *col_mul, hipStream_t s) {
    if (act == ACT_GELU)
        return col_mul ? run_stream<1, true, ACT_GELU, true>(a, x, K, col_mul, s)
                       : run_stream<1, true, ACT_GELU, false>(a, x, K, nullptr, s);
    return col_mul ? run_stream<1, true, ACT_NONE, true>(a, x, K, col_mul, s)
                   : run_stream<1, true, ACT_NONE, false>(a, x, K, nullptr, s);
}

}  // namespace w8a8
