// Root-mean-square norm of rows, with the residual's addition in front of it and the row's
// quantization behind it: what stands before every linear of a transformer, in one pass.
//   h = bf16(x + residual), or x itself
//   r = float32(1 / sqrt(sum_k h[k]^2 / K + eps)), the sum and the root in 64 bits
//   v[k] = (h[k] * r) * w[k], float32, each product rounded (w absent: v = h * r)
// then v by the int8 rule of quant_math.hpp (codes and one scale a row) or in 4-bit blocks of
// mx_math.hpp. The squares are exact in 32 bits and their sum is held in 64, so that r does not
// hang on the order of the sum: codes are determined bit by bit, but for sums that lie within
// 2^-50 of a rounding border of r.
//
// Bound by memory: 2 (4 with a residual) bytes read and 1 or 17/32 (+ 2) written an element. 4608 x
// 4096 with a residual takes 22.7 us in int8 (5.8 TB/s; a large copy reaches 5.1), 22.9 in 4 bits (5.4),
// 4608 x 16384 101 and 97, 2001 x 1000 in 4 bits 4.1, one token of 4096 channels 2.4, two barriers and
// 64-bit root included. The sum in 64 bits costs a conversion and a product an element, which the loads hide.
#include "lm_internal.hpp"
#include "mx_quant.hpp"

namespace w8a8 {
namespace {

using namespace qmath;
using namespace mx;

typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2v __attribute__((ext_vector_type(2)));

constexpr int kRsrcWord3 = 0x00020000;     // gfx9 raw buffer

// Sum over the wavefront, the same in every lane: both halves of a double move through DPP
// operands; lanes that a step leaves out add zero.
__device__ __forceinline__ double wave_sum64(double v) {
    const auto step = [&](auto ctrl, auto rows) {
        const uint64_t b = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(
            0, (int)(uint32_t)b, decltype(ctrl)::value, decltype(rows)::value, 0xF, true);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(
            0, (int)(uint32_t)(b >> 32), decltype(ctrl)::value, decltype(rows)::value, 0xF, true);
        v += __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    };
    using std::integral_constant;
    step(integral_constant<int, 0x111>{}, integral_constant<int, 0xF>{});   // row_shr:1
    step(integral_constant<int, 0x112>{}, integral_constant<int, 0xF>{});   // row_shr:2
    step(integral_constant<int, 0x114>{}, integral_constant<int, 0xF>{});   // row_shr:4
    step(integral_constant<int, 0x118>{}, integral_constant<int, 0xF>{});   // row_shr:8
    step(integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});   // row_bcast:15
    step(integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});   // row_bcast:31
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, 63);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), 63);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

__device__ __forceinline__ float lo_f32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f32(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// bf16(a + b) of two pairs.
__device__ __forceinline__ uint32_t add_pairs(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)(lo_f32(a) + lo_f32(b)),
                                               (__bf16)(hi_f32(a) + hi_f32(b))});
}

__device__ __forceinline__ double squares(const uint32_t (&w)[4], double sum) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const double a = lo_f32(w[i]), b = hi_f32(w[i]);
        sum = __builtin_fma(a, a, sum);
        sum = __builtin_fma(b, b, sum);
    }
    return sum;
}

__device__ __forceinline__ float inverse_rms(double sum, int64_t K, double eps) {
    return (float)(1.0 / __builtin_sqrt(sum / (double)K + eps));
}

// v of a unit of 8 channels.
__device__ __forceinline__ void scaled8(const uint32_t (&w)[4], float r, const float (&c)[8],
                                        float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = lo_f32(w[i]) * r * c[2 * i];
        v[2 * i + 1] = hi_f32(w[i]) * r * c[2 * i + 1];
    }
}

__device__ __forceinline__ uint32_t magnitude8(const float (&v)[8]) {
    float m = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        m = fmaxf(m, __builtin_fabsf(v[e]));
    return __float_as_uint(m);             // |v| >= 0: its bits order like the value
}

// The 4-bit codes of a lane's 8 values and their block's scale byte; the block's four lanes call
// it together. The largest magnitude by bits, so that infinities and NaN mark the block.
__device__ __forceinline__ uint32_t block_codes(const float (&v)[8], uint32_t &byte) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        m = max(m, __float_as_uint(v[e]) & 0x7FFFFFFFu);
    byte = scale_byte<kTop4>(quad_max(m) >> 23);
    const uint32_t q = encode4_f32(v, scale_operand(byte));
    return byte == kNaNScale ? 0 : q;
}

// Weights of channels k .. k + 7, zeros behind K (nothing is stored there), ones where there are
// none. WIDE: 16-byte aligned, and K a multiple of 8.
template <bool WIDE>
__device__ __forceinline__ void weights8(const NormArgs &a, int64_t k, float (&c)[8]) {
    const __amdgpu_buffer_rsrc_t src = __builtin_amdgcn_make_buffer_rsrc(
        (void *)a.weight, (short)0, a.weight ? (int)(4 * a.K) : 0, kRsrcWord3);
    uint32_t w[8];
    if constexpr (WIDE) {
        const u32x4v lo = __builtin_amdgcn_raw_buffer_load_b128(src, (int)(4 * k), 0, 0);
        const u32x4v hi = __builtin_amdgcn_raw_buffer_load_b128(src, (int)(4 * k) + 16, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            w[e] = lo[e];
            w[e + 4] = hi[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            w[e] = __builtin_amdgcn_raw_buffer_load_b32(src, (int)(4 * k) + 4 * e, 0, 0);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        c[e] = __uint_as_float(a.weight ? w[e] : 0x3F800000u);
}

// Stores n (1 .. 8) values of a unit at any alignment.
__device__ __forceinline__ void store_sum(uint16_t *p, const uint32_t (&w)[4], int64_t n) {
    if (n >= 8) {
        *reinterpret_cast<Bytes16 *>(p) = Bytes16{{w[0], w[1], w[2], w[3]}};
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n)
                p[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
    }
}

__device__ __forceinline__ void store_codes8(int8_t *p, uint2 c, int64_t n) {
    if (n >= 8) {
        *reinterpret_cast<Bytes8 *>(p) = Bytes8{{c.x, c.y}};
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n)
                p[e] = (int8_t)((e < 4 ? c.x : c.y) >> (8 * (e & 3)));
    }
}

__device__ __forceinline__ uint2 codes8(const float (&v)[8], float inv) {
    return make_uint2(code4(v[0], v[1], v[2], v[3], inv), code4(v[4], v[5], v[6], v[7], inv));
}

// A row by TPR threads, NV units of 8 channels each, in registers from its load to its codes; the
// next row is loaded while this one is worked on. Without ANY rows are 16-byte aligned and go
// through buffer descriptors, whose bounds replace the branches at a row's end (a branch around a
// load makes the compiler wait for all loads in flight, the next row's included).
template <int TPR>
constexpr int norm_threads() { return TPR > 256 ? TPR : 256; }

template <int FMT, int TPR, int NV, bool RES, bool ANY>
__global__ void __launch_bounds__(norm_threads<TPR>())
norm_rows_kernel(NormArgs a) {
    constexpr int BS = norm_threads<TPR>(), RPB = BS / TPR, WPR = TPR / 64;
    __shared__ double part_sum[2][RPB][WPR];       // in turn: one barrier a row and exchange
    __shared__ uint32_t part_max[2][RPB][WPR];
    const int t = threadIdx.x % TPR;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int sub = wave / WPR;
    const int64_t groups = (a.R + RPB - 1) / RPB;
    const int64_t row_bytes = (a.K + 31) / 32 * 16;        // of 4-bit codes

    float c[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j)
        weights8<!ANY>(a, ((int64_t)j * TPR + t) * 8, c[j]);

    struct Loaded {
        uint32_t x[NV][4], r[RES ? NV : 1][4];
    };
    const auto load = [&](Loaded &d, int64_t grp) __attribute__((always_inline)) {
        const int64_t row = grp * RPB + sub;
        const bool live = row < a.R;
        const int64_t at = (live ? row : 0) * a.K;
        if constexpr (ANY) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int64_t k = live ? ((int64_t)j * TPR + t) * 8 : a.K;
                load8(a.x + at, k, a.K, d.x[j]);
                if constexpr (RES)
                    load8(a.residual + at, k, a.K, d.r[j]);
            }
        } else {
            const int bytes = live ? (int)(2 * a.K) : 0;
            const auto fetch = [&](const uint16_t *p, uint32_t (&w)[4], int j) {
                const __amdgpu_buffer_rsrc_t src =
                    __builtin_amdgcn_make_buffer_rsrc((void *)(p + at), (short)0, bytes, kRsrcWord3);
                const u32x4v v = __builtin_amdgcn_raw_buffer_load_b128(src, (j * TPR + t) * 16, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    w[i] = v[i];
            };
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                fetch(a.x, d.x[j], j);
                if constexpr (RES)
                    fetch(a.residual, d.r[j], j);
            }
        }
    };

    int turn = 0;
    const auto process = [&](Loaded &d, int64_t grp) __attribute__((always_inline)) {
        const int64_t row = grp * RPB + sub;
        const bool live = row < a.R;
        const int64_t at = (live ? row : 0) * a.K;
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if constexpr (RES) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    d.x[j][i] = add_pairs(d.x[j][i], d.r[j][i]);
            }
            sum = squares(d.x[j], sum);
        }
        if constexpr (RES) {
            if constexpr (ANY) {
                if (live) {
#pragma unroll
                    for (int j = 0; j < NV; ++j) {
                        const int64_t k = ((int64_t)j * TPR + t) * 8;
                        if (k < a.K)
                            store_sum(a.sum + at + k, d.x[j], a.K - k);
                    }
                }
            } else {
                const __amdgpu_buffer_rsrc_t dst = __builtin_amdgcn_make_buffer_rsrc(
                    (void *)(a.sum + at), (short)0, live ? (int)(2 * a.K) : 0, kRsrcWord3);
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    __builtin_amdgcn_raw_buffer_store_b128(
                        u32x4v{d.x[j][0], d.x[j][1], d.x[j][2], d.x[j][3]}, dst, (j * TPR + t) * 16,
                        0, 0);
            }
        }
        sum = wave_sum64(sum);
        if constexpr (WPR > 1) {
            if ((threadIdx.x & 63) == 0)
                part_sum[turn][sub][wave % WPR] = sum;
            __syncthreads();
            sum = 0.0;
#pragma unroll
            for (int w = 0; w < WPR; ++w)
                sum += part_sum[turn][sub][w];
        }
        const float r = inverse_rms(sum, a.K, a.eps);
        if constexpr (FMT == NORM_INT8) {
            float v[NV][8];
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                scaled8(d.x[j], r, c[j], v[j]);
                m = max(m, magnitude8(v[j]));
            }
            m = wave_max(m);
            if constexpr (WPR > 1) {
                if ((threadIdx.x & 63) == 0)
                    part_max[turn][sub][wave % WPR] = m;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < WPR; ++w)
                    m = max(m, part_max[turn][sub][w]);
            }
            const RowScale rs = row_scale_f(__uint_as_float(m));
            if constexpr (ANY) {
                if (live) {
                    if (t == 0)
                        a.scale[row] = rs.scale;
#pragma unroll
                    for (int j = 0; j < NV; ++j) {
                        const int64_t k = ((int64_t)j * TPR + t) * 8;
                        if (k < a.K)
                            store_codes8(reinterpret_cast<int8_t *>(a.codes) + at + k,
                                         codes8(v[j], rs.inv), a.K - k);
                    }
                }
            } else {
                const __amdgpu_buffer_rsrc_t sdst = __builtin_amdgcn_make_buffer_rsrc(
                    (void *)(a.scale + (live ? row : 0)), (short)0, live ? 4 : 0, kRsrcWord3);
                __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(rs.scale), sdst, t * 4, 0, 0);
                const __amdgpu_buffer_rsrc_t dst = __builtin_amdgcn_make_buffer_rsrc(
                    (void *)(a.codes + at), (short)0, live ? (int)a.K : 0, kRsrcWord3);
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const uint2 q = codes8(v[j], rs.inv);
                    __builtin_amdgcn_raw_buffer_store_b64(u32x2v{q.x, q.y}, dst, (j * TPR + t) * 8, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int64_t u = (int64_t)j * TPR + t;
                float v[8];
                uint32_t byte;
                scaled8(d.x[j], r, c[j], v);
                const uint32_t q = block_codes(v, byte);
                if (live && u * 4 < row_bytes)
                    *reinterpret_cast<uint32_t *>(a.codes + row * row_bytes + u * 4) = q;
                if (live && u * 8 < (a.K + 255) / 256 * 256 && t % 4 == 0)
                    a.scales[((u >> 5) * a.R + row) * 8 + (u >> 2) % 8] = (uint8_t)byte;
            }
        }
        turn ^= 1;
    };

    Loaded p, q;
    int64_t grp = blockIdx.x;
    load(p, grp);
    for (;;) {
        load(q, grp + gridDim.x);          // past the last row: nothing is read
        __builtin_amdgcn_sched_barrier(0);
        process(p, grp);
        grp += gridDim.x;
        if (grp >= groups)
            break;
        load(p, grp + gridDim.x);
        __builtin_amdgcn_sched_barrier(0);
        process(q, grp);
        grp += gridDim.x;
        if (grp >= groups)
            break;
    }
}

// Rows too long for registers (or of no channels): 1024 threads read a row twice (4 bits) or
// three times, the sum from where the first pass stored it (each thread what it wrote itself).
template <int FMT, bool RES>
__global__ void __launch_bounds__(1024)
norm_loop_kernel(NormArgs a) {
    __shared__ double part_sum[16];
    __shared__ uint32_t part_max[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t units = (a.K + 255) / 256 * 32, row_bytes = (a.K + 31) / 32 * 16;
    for (int64_t row = blockIdx.x; row < a.R; row += gridDim.x) {
        const uint16_t *x = a.x + row * a.K, *h = RES ? a.sum + row * a.K : x;
        double sum = 0.0;
        for (int64_t u = threadIdx.x; u * 8 < a.K; u += 1024) {
            uint32_t w[4], s[4];
            load8(x, u * 8, a.K, w);
            if constexpr (RES) {
                load8(a.residual + row * a.K, u * 8, a.K, s);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    w[i] = add_pairs(w[i], s[i]);
                store_sum(a.sum + row * a.K + u * 8, w, a.K - u * 8);
            }
            sum = squares(w, sum);
        }
        sum = wave_sum64(sum);
        if (lane == 0)
            part_sum[wave] = sum;
        __syncthreads();
        sum = 0.0;
        for (int w = 0; w < 16; ++w)
            sum += part_sum[w];
        const float r = inverse_rms(sum, a.K, a.eps);
        const auto values = [&](int64_t u, float (&v)[8]) {
            uint32_t w[4];
            float c[8];
            load8(h, u * 8, a.K, w);
            weights8<false>(a, u * 8, c);
            scaled8(w, r, c, v);
        };
        if constexpr (FMT == NORM_INT8) {
            uint32_t m = 0;
            for (int64_t u = threadIdx.x; u * 8 < a.K; u += 1024) {
                float v[8];
                values(u, v);
                m = max(m, magnitude8(v));
            }
            m = wave_max(m);
            if (lane == 0)
                part_max[wave] = m;
            __syncthreads();
            for (int w = 0; w < 16; ++w)
                m = max(m, part_max[w]);
            const RowScale rs = row_scale_f(__uint_as_float(m));
            if (threadIdx.x == 0)
                a.scale[row] = rs.scale;
            for (int64_t u = threadIdx.x; u * 8 < a.K; u += 1024) {
                float v[8];
                values(u, v);
                store_codes8(reinterpret_cast<int8_t *>(a.codes) + row * a.K + u * 8,
                             codes8(v, rs.inv), a.K - u * 8);
            }
        } else {
            // whole blocks: the four lanes of one leave the loop together
            for (int64_t u = threadIdx.x; u < units; u += 1024) {
                float v[8];
                uint32_t byte;
                values(u, v);
                const uint32_t q = block_codes(v, byte);
                if (u * 4 < row_bytes)
                    *reinterpret_cast<uint32_t *>(a.codes + row * row_bytes + u * 4) = q;
                if (u % 4 == 0)
                    a.scales[((u >> 5) * a.R + row) * 8 + (u >> 2) % 8] = (uint8_t)byte;
            }
        }
        __syncthreads();           // the next row's sums go where this one's were
    }
}

bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

template <int FMT, int TPR, int NV, bool RES>
hipError_t run_rows(const NormArgs &a, hipStream_t s) {
    constexpr int BS = norm_threads<TPR>(), RPB = BS / TPR;
    const int64_t groups = (a.R + RPB - 1) / RPB;
    // A grid of at most 2048 threads a CU, whose workgroups get equally many row groups: weights stay
    // in registers from one to the next.
    const int64_t most = 256 * 2048 / BS, turns = (groups + most - 1) / most;
    const dim3 grid((unsigned)((groups + turns - 1) / turns)), block(BS);
    const bool whole = a.K % 8 == 0 && aligned(a.x, 16) && aligned(a.weight, 16) &&
                       (!RES || (aligned(a.residual, 16) && aligned(a.sum, 16))) &&
                       (FMT != NORM_INT8 || aligned(a.codes, 8));
    if (whole)
        hipLaunchKernelGGL((norm_rows_kernel<FMT, TPR, NV, RES, false>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((norm_rows_kernel<FMT, TPR, NV, RES, true>), grid, block, 0, s, a);
    return hipGetLastError();
}

template <int FMT, bool RES>
hipError_t run_norm(const NormArgs &a, hipStream_t s) {
    // Units that a row's threads have to cover: 4-bit rows write the scales of whole panels.
    const int64_t units = FMT == NORM_INT8 ? (a.K + 7) / 8 : (a.K + 255) / 256 * 32;
    if (a.K > 0 && units <= 64)
        return run_rows<FMT, 64, 1, RES>(a, s);
    if (a.K > 0 && units <= 128)
        return run_rows<FMT, 64, 2, RES>(a, s);
    if (a.K > 0 && units <= 256)
        return run_rows<FMT, 256, 1, RES>(a, s);
    if (a.K > 0 && units <= 512)
        return run_rows<FMT, 256, 2, RES>(a, s);
    if (a.K > 0 && units <= 1024)
        return run_rows<FMT, 512, 2, RES>(a, s);
    if (a.K > 0 && units <= 2048)
        return run_rows<FMT, 1024, 2, RES>(a, s);
    if (a.K > 0 && units <= 4096)
        return run_rows<FMT, 1024, 4, RES>(a, s);
    const dim3 grid((unsigned)(a.R < 65536 ? a.R : 65536));
    hipLaunchKernelGGL((norm_loop_kernel<FMT, RES>), grid, dim3(1024), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_quant(const NormArgs &a, int fmt, hipStream_t s) {
    if (a.R == 0)
        return hipSuccess;
    if (fmt == NORM_INT8)
        return a.residual ? run_norm<NORM_INT8, true>(a, s) : run_norm<NORM_INT8, false>(a, s);
    return a.residual ? run_norm<NORM_MX4, true>(a, s) : run_norm<NORM_MX4, false>(a, s);
}

}  // namespace w8a8
