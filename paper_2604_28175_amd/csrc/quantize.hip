// Rows of activations as 8-bit integers with a scale each, the left operand of gemm_i8.hip, for gfx950.
//
//   s = max_k |x_k| (1 / 127),   q_k = rint(x_k (1 / s))
//
// A row is read once and stays in registers between its maximum and its codes where it has at most 32 numbers per thread; 2 + 1 bytes per number, so
// the memory bounds it: 65536 x 4096 134 us (6.0 TB/s), 8192 x 4096 19 us (5.3 TB/s); a single row is a launch's latency, 3.0 us.  A wavefront per row up to 2048 numbers
// (no barrier), four of them beyond: 8192 x 1024 7.8 and 12.3 us, 65536 x 2048 72 and 90, 8192 x 4096 23.5 and 18.8, 1 x 4096 4.6 and 2.9.
#include "decoder.hpp"

namespace strait {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef unsigned short ushort8 __attribute__((ext_vector_type(8)));
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));

constexpr int QUANTIZE_KEPT = 4;         // chunks of 8 numbers that a thread keeps

template <int TPR>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const half_t* __restrict__ x, int M, int chunks, long long pitch, int8_t* __restrict__ q,
                                                            float* __restrict__ scale, int hp) {
    __shared__ unsigned part[4];
    if (hp) __builtin_amdgcn_s_setprio(3);
    const int t = TPR == 64 ? threadIdx.x & 63 : threadIdx.x;
    const int m = TPR == 64 ? (int)blockIdx.x * 4 + (int)(threadIdx.x >> 6) : (int)blockIdx.x;
    if (TPR == 64 && m >= M) return;
    const half8* row = (const half8*)(x + (long long)m * pitch);
    uintx2* out = (uintx2*)(q + (long long)m * chunks * 8);
    half8 kept[QUANTIZE_KEPT];
    // magnitudes compare like the 16-bit numbers that hold them, infinities above all numbers and NaN above these
    ushort8 top = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < QUANTIZE_KEPT; ++i)
        if (t + i * TPR < chunks) kept[i] = row[t + i * TPR];
#pragma unroll
    for (int i = 0; i < QUANTIZE_KEPT; ++i)
        if (t + i * TPR < chunks) top = __builtin_elementwise_max(top, __builtin_bit_cast(ushort8, kept[i]) & (unsigned short)0x7fff);
    for (int c = t + QUANTIZE_KEPT * TPR; c < chunks; c += TPR) top = __builtin_elementwise_max(top, __builtin_bit_cast(ushort8, row[c]) & (unsigned short)0x7fff);
    unsigned a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = top[i] > a ? top[i] : a;
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const unsigned b = (unsigned)__shfl_xor((int)a, d);
        a = a > b ? a : b;
    }
    if (TPR > 64) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = a;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) a = part[i] > a ? part[i] : a;
    }
    const bool finite = a < 0x7c00;
    const float s = (float)__builtin_bit_cast(half_t, (unsigned short)a) * (1.f / 127.f);
    const float inv = finite && a ? 1.f / s : 0.f;
    if (t == 0) scale[m] = finite ? s : __builtin_nanf("");
    auto store = [&](int c, half8 v) __attribute__((always_inline)) {
        uintx2 w = {0, 0};
        if (finite) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i >> 2] |= ((unsigned)(int)__builtin_rintf((float)v[i] * inv) & 0xffu) << (8 * (i & 3));
        }
        out[c] = w;
    };
#pragma unroll
    for (int i = 0; i < QUANTIZE_KEPT; ++i)
        if (t + i * TPR < chunks) store(t + i * TPR, kept[i]);
    for (int c = t + QUANTIZE_KEPT * TPR; c < chunks; c += TPR) store(c, row[c]);
}

int launch_quantize_rows(const half_t* x, int M, int K, long long pitch, int8_t* q, float* scale, int hp, hipStream_t stream) {
    if (M > MOST_WORKGROUPS) { set_error("quantize_rows: grid too large"); return STRAIT_E_SHAPE; }
    if (K <= 64 * 8 * QUANTIZE_KEPT) hipLaunchKernelGGL((quantize_rows_kernel<64>), dim3((unsigned)((M + 3LL) / 4)), dim3(256), 0, stream, x, M, K / 8, pitch, q, scale, hp);
    else hipLaunchKernelGGL((quantize_rows_kernel<256>), dim3((unsigned)M), dim3(256), 0, stream, x, M, K / 8, pitch, q, scale, hp);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("quantize_rows launch: %s", hipGetErrorString(e)); return -2; }
    return 0;
}

}  // namespace strait
