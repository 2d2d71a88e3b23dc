// Products in 8-bit integers with a scale for each token and each output channel, for gfx950.
//
//   y[m, n] = act( xs[m] ws[n] sum_k x[m, k] w[n, k] + bias[n] (+ res[m, n]) )
//
// The sum is an int32 of v_mfma_i32_32x32x32_i8 and exact; the epilogue is fp32, rounded once.
#include "activation.hpp"
#include "decoder.hpp"

namespace strait {

typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx16 __attribute__((ext_vector_type(16)));

// One output of a sum: the same operations in the same order in every kernel, so that a row has the same bits whatever launch it is part of.
__device__ __forceinline__ float finish(int sum, float xs, float ws, float bias, float res, int act) {
    return apply_act(__builtin_fmaf((float)sum, xs * ws, bias) + res, act);
}

__global__ void __launch_bounds__(256) gemm_i8_kernel(const GemmI8 p, int tiles_n) {
    if (p.hp) __builtin_amdgcn_s_setprio(3);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, lh = lane >> 5;
    const int tm = (int)blockIdx.x / tiles_n, tn = (int)blockIdx.x - tm * tiles_n;
    const int m = tm * 64 + (wave >> 1) * 32 + l32, n0 = tn * 64 + (wave & 1) * 32, n = n0 + l32;
    const int8_t* xr = p.x + (long long)(m < p.M ? m : p.M - 1) * p.K + lh * 16;
    const int8_t* wr = p.w + (long long)(n < p.N ? n : p.N - 1) * p.K + lh * 16;
    intx16 acc = {};
    for (int k = 0; k < p.K; k += 32) {
        const bool there = k + lh * 16 < p.K;
        const intx4 a = there ? *(const intx4*)(wr + k) : intx4{}, b = there ? *(const intx4*)(xr + k) : intx4{};
        acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, acc, 0, 0, 0);
    }
    if (m >= p.M) return;
    // lane holds y[m][n0 + 8 g + 4 lh + j], v = 4 g + j
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const int c = n0 + 8 * (v >> 2) + 4 * lh + (v & 3);
        if (c >= p.N) continue;
        const long long at = (long long)m * p.N + c;
        const float y = finish(acc[v], p.xs[m], p.ws[c], p.bias ? p.bias[c] : 0.f, p.res ? (float)p.res[at] : 0.f, p.act);
        if (p.out_f32) ((float*)p.y)[at] = y;
        else ((half_t*)p.y)[at] = (half_t)y;
    }
}

int launch_gemm_i8(const GemmI8& p, hipStream_t stream) {
    const long long tiles_m = (p.M + 63LL) / 64, tiles_n = (p.N + 63LL) / 64;
    if (tiles_m * tiles_n > 0x7fffffffLL) { set_error("gemm_i8: grid too large"); return STRAIT_E_SHAPE; }
    hipLaunchKernelGGL(gemm_i8_kernel, dim3((unsigned)(tiles_m * tiles_n)), dim3(256), 0, stream, p, (int)tiles_n);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("gemm_i8 launch: %s", hipGetErrorString(e)); return -2; }
    return 0;
}

}  // namespace strait
