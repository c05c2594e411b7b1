// Microscaled 4-bit quantization of a matrix and back.
//
// mx4_quantize: v[r][k] = T(x[r][k]) * c[k] (T the identity or GELU, c the SmoothQuant
// multiplier or absent; float32, or the bf16 inputs themselves where neither is there) in
// blocks of 32 channels by the rule of mx_math.hpp. Codes [R, 16 ceil(K/32)], scales
// [ceil(K/256), R, 8]: the scale bytes of 256 channels of neighbouring rows side by side, so
// that the product reads a tile's scales of one K-panel as one piece of memory.
//
// Bound by memory: 2 bytes read and 17/32 written per element. 4608 x 4096 with a multiplier
// takes 10.3 us (4.6 TB/s; 13.9 before all of a wavefront's rows were loaded at once). 4608 x 16384
// on matrices in turn takes 33 us (5.7 TB/s), 41 with GELU (its table's LDS reads), and 51 right
// behind the 151 MB that its decoder has written (75 with GELU evaluated); on one matrix again
// and again, which then comes from the last cache, 29 and 39. That matrix decoded again 27.9 us
// (6.8 TB/s, the codes still in the cache).
#include "mx_internal.hpp"
#include "mx_quant.hpp"

namespace w8a8 {
namespace {

using namespace mx;

// A lane holds 8 neighbouring channels, four lanes a block, a wavefront 512 channels (two
// scale panels) of one row at a time; it takes ROWS rows one below the other, whose scale
// bytes are neighbours in memory, and has all their loads in flight at once. No value outside a
// block matters to it, so nothing is exchanged but the block's maximum inside its four lanes.
// GELU comes from the table of all bf16 magnitudes, copied to LDS while the rows arrive.
constexpr int kWaves = 4;

template <int ACT, bool CM, int ROWS>
__global__ void __launch_bounds__(kWaves * 64)
mx4_quant_kernel(const uint16_t *x, int64_t R, int64_t K, const float *col_mul, uint8_t *codes,
                 uint8_t *scales, unsigned chunks) {
    constexpr bool GELU = ACT == ACT_GELU;
    __shared__ __attribute__((aligned(16))) float gelu[GELU ? sizeof(GeluTable) / 4 : 1];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned group = blockIdx.x / chunks;
    const int64_t chunk = blockIdx.x - group * chunks;          // 512 channels
    const int64_t r0 = ((int64_t)group * kWaves + wave) * ROWS;
    const int64_t k = chunk * 512 + lane * 8;
    const int64_t row_bytes = (K + 31) / 32 * 16;
    const int64_t panel = chunk * 2 + (lane >> 5);
    const bool store_codes = k / 2 < row_bytes, store_scale = panel * 256 < K && lane % 4 == 0;
    uint32_t w[ROWS][4];
    if (chunk * 512 + 512 <= K) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const Bytes16 b = *reinterpret_cast<const Bytes16 *>(x + min(r0 + i, R - 1) * K + k);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                w[i][e] = b.w[e];
        }
    } else {
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
            load8(x + min(r0 + i, R - 1) * K, k, K, w[i]);
    }
    float c[8];
    if constexpr (CM)
        load_multipliers(col_mul, k, K, c);
    if constexpr (GELU) {
        for (int i = threadIdx.x; i < (int)(sizeof(GeluTable) / 16); i += kWaves * 64)
            reinterpret_cast<float4 *>(gelu)[i] = reinterpret_cast<const float4 *>(&kGeluTable)[i];
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t r = r0 + i;
        if (r >= R)
            return;
        uint32_t byte;
        const uint32_t q = quantize_quad<ACT, CM>(w[i], c, gelu, byte);
        if (store_codes)
            *reinterpret_cast<uint32_t *>(codes + r * row_bytes + k / 2) = q;
        if (store_scale)
            scales[(panel * R + r) * 8 + (lane >> 2) % 8] = (uint8_t)byte;
    }
}

// One lane decodes 8 channels.
__global__ void __launch_bounds__(256)
mx4_dequant_kernel(const uint8_t *codes, const uint8_t *scales, int64_t R, int64_t K, uint16_t *y) {
    const int64_t r = blockIdx.y + (int64_t)blockIdx.z * 65535;
    const int64_t k = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (r >= R || k >= K)
        return;
    const uint32_t q = *reinterpret_cast<const uint32_t *>(codes + r * ((K + 31) / 32 * 16) + k / 2);
    const float s = scale_operand(scales[((k >> 8) * R + r) * 8 + ((k >> 5) & 7)]);
    const uint32_t w[4] = {decode4<0>(q, s), decode4<1>(q, s), decode4<2>(q, s), decode4<3>(q, s)};
    uint16_t *o = y + r * K + k;
    if (k + 8 <= K) {
        Bytes16 b;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            b.w[i] = w[i];
        *reinterpret_cast<Bytes16 *>(o) = b;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (k + e < K)
                o[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
    }
}

}  // namespace

hipError_t launch_mx4_quant(const uint16_t *x, int64_t R, int64_t K, int act,
                            const float *col_mul, uint8_t *codes, uint8_t *scales,
                            hipStream_t s) {
    if (R == 0 || K == 0)
        return hipSuccess;
    const int64_t chunks = (K + 511) / 512;
    // Eight rows a wavefront where that leaves 4096 wavefronts, 16 a CU; else a row each, as a
    // short call's time is one row's latency. us by one and by eight, calls on one input in a
    // graph: 64 x 256 2.4, 5.0; 1024 x 4096 with GELU and multiplier 4.7, 5.9; 2048 x 4096 4.5,
    // 4.3; 1152 x 16384 and 4608 x 16384 with both 16.0, 15.2 and 52.7, 40.1.
    const int rows = R * chunks >= 8 * 4096 ? 8 : 1;
    const int64_t blocks = chunks * ((R + kWaves * rows - 1) / (kWaves * rows));
    if (!launchable(blocks, kWaves * 64))
        return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks), block(kWaves * 64);
    const auto go = [&](auto act_c, auto cm) {
        constexpr int A = decltype(act_c)::value;
        constexpr bool CM = decltype(cm)::value;
        if (rows == 8)
            hipLaunchKernelGGL((mx4_quant_kernel<A, CM, 8>), grid, block, 0, s, x, R, K, col_mul, codes,
                               scales, (unsigned)chunks);
        else
            hipLaunchKernelGGL((mx4_quant_kernel<A, CM, 1>), grid, block, 0, s, x, R, K, col_mul, codes,
                               scales, (unsigned)chunks);
        return hipGetLastError();
    };
    const auto with_act = [&](auto act_c) {
        return col_mul ? go(act_c, std::true_type{}) : go(act_c, std::false_type{});
    };
    return act == ACT_GELU ? with_act(std::integral_constant<int, ACT_GELU>{})
                           : with_act(std::integral_constant<int, ACT_NONE>{});
}

hipError_t launch_mx4_dequant(const uint8_t *codes, const uint8_t *scales, int64_t R, int64_t K,
                              uint16_t *y, hipStream_t s) {
    if (R == 0 || K == 0)
        return hipSuccess;
    const int64_t tall = (R + 65534) / 65535;
    if (tall > 65535)
        return hipErrorInvalidValue;
    const dim3 grid((unsigned)((K + 2047) / 2048), (unsigned)(R < 65535 ? R : 65535), (unsigned)tall);
    hipLaunchKernelGGL(mx4_dequant_kernel, grid, dim3(256), 0, s, codes, scales, R, K, y);
    return hipGetLastError();
}

}  // namespace w8a8
