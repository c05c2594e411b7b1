// Microscaled 4-bit product: Y[m][n] = bf16(sum_k X[m][k] W[n][k] + b[n]) on the codes and
// scale bytes of mx4_quant.hip, with float32 accumulation in the scaled matrix instructions.
#include "mx_internal.hpp"
#include "mx_math.hpp"

namespace w8a8 {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ i32x8 frag(i32x4 v) {
    return i32x8{v[0], v[1], v[2], v[3], 0, 0, 0, 0};
}

// One wavefront per 32 x 32 outputs, operands straight from memory.
__global__ void __launch_bounds__(256)
mx4_gemm_simple_kernel(Mx4Args a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t tiles_n = (a.N + 63) / 64;
    const int64_t m0 = blockIdx.x / tiles_n * 64 + (wave & 1) * 32;
    const int64_t n0 = blockIdx.x % tiles_n * 64 + (wave >> 1) * 32;
    const int64_t m = m0 + (lane & 31), n = n0 + (lane & 31);
    const int64_t mr = min(m, a.M - 1), nr = min(n, a.N - 1);
    f32x16 acc = {};
    for (int64_t b = lane >> 5; b - (lane >> 5) < a.nb; b += 2) {
        i32x4 x = {}, w = {};
        int sx = 0, sw = 0;
        if (b < a.nb) {
            x = *reinterpret_cast<const i32x4 *>(a.xq + (mr * a.nb + b) * 16);
            w = *reinterpret_cast<const i32x4 *>(a.wq + (nr * a.nb + b) * 16);
            sx = a.xs[((b >> 3) * a.M + mr) * 8 + (b & 7)];
            sw = a.ws[((b >> 3) * a.N + nr) * 8 + (b & 7)];
        }
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(frag(w), frag(x), acc, 4, 4, 0, sw, 0,
                                                              sx);
    }
    if (m >= a.M)
        return;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int64_t c = n0 + 8 * (i / 4) + 4 * (lane >> 5) + i % 4;
        if (c < a.N) {
            const float b = a.bias ? __uint_as_float((uint32_t)a.bias[c] << 16) : 0.0f;
            a.y[m * a.N + c] = __builtin_bit_cast(uint16_t, (__bf16)(acc[i] + b));
        }
    }
}

}  // namespace

size_t mx4_gemm_workspace_bytes(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_mx4_gemm(const Mx4Args &a, void *, size_t, hipStream_t s) {
    const int64_t blocks = ((a.M + 63) / 64) * ((a.N + 63) / 64);
    if (blocks > 0x7FFFFFFF)
        return hipErrorInvalidValue;
    hipLaunchKernelGGL(mx4_gemm_simple_kernel, dim3((unsigned)blocks), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace w8a8
