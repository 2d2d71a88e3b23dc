// Attention of a step's tokens over a paged cache, with a causal mask, an optional sliding window and a few first tokens that stay visible, for gfx950.
//
//   out[t, h] = sum_j softmax_j( scale q[t, h] . k_j ) v_j  over the keys j <= p  with  window == 0  or  p - j < window  or  j < sinks
//
// The rows of a tile are 16 (token, head of the group) pairs of one kv head: all of them read the same keys.  A wavefront walks over the keys in
// blocks of 32, which lie on one page each:
//   - scores^T = K Q^T with v_mfma_f32_16x16x32_f16: a lane names 16 bytes of a key, as they lie in memory, and Q is enumerated in the same order; it then holds
//     8 of the block's keys for ONE row;
//   - an int8 code becomes fp16 by way of the number 2^-24 (code + 128), a subnormal whose bits are the code's: one fused multiply-add makes
//     code 2^-9 of it, exactly.  The scale of the block's page multiplies the scores and the block's share of the output, in fp32;
//   - the probabilities, rounded to fp16, are the "B" operand of out^T = V^T P^T as they are, keys enumerated in the order that the scores came in; V^T's lanes
//     read 8 keys at D / 16 dimensions each and exchange bytes within a lane;
//   - one pass with a running maximum, which follows the true one only where that is more than 8 (in log2) ahead: probabilities stay below 2^8, and the
//     output is rescaled a few times in all.
#include "decoder.hpp"

namespace strait {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));

constexpr int KEYS = 32;                 // of a block

// Two of the 8-bit codes in `a` and `b` (biased by 128: codes ^ 0x80) as fp16 code 2^-9; sel: v_perm_b32's selector of the two bytes
__device__ __forceinline__ half2_t two_codes(unsigned a, unsigned b, unsigned sel) {
    const half2_t u = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(b, a, sel));
    const half2_t by = {(half_t)32768.f, (half_t)32768.f}, off = {(half_t)-0.25f, (half_t)-0.25f};
    return __builtin_elementwise_fma(u, by, off);
}

// The blocks of keys that any of the positions lo .. hi sees, in order: the first `sink` ones, then those from `from` on, `count` in all.
struct Blocks {
    int sink, from, count;
    __device__ __forceinline__ int at(int i) const { return i < sink ? i : from + i - sink; }
};
__device__ __forceinline__ Blocks visible_blocks(int lo, int hi, int window, int sinks) {
    if (hi < 0) return {0, 0, 0};
    if (lo < 0) lo = 0;
    const int last = hi / KEYS + 1, first = window && lo >= window ? (lo - window + 1) / KEYS : 0;
    const int sink = window ? (sinks + KEYS - 1) / KEYS : 0;
    if (sink >= first) return {0, 0, last};            // one piece
    return {sink, first, sink + last - first};
}

template <int D, bool I8>
__global__ void __launch_bounds__(64) paged_attention_kernel(const PagedAttention p, int tiles) {
    if (p.hp) __builtin_amdgcn_s_setprio(3);
    const int lane = threadIdx.x, l16 = lane & 15, g4 = lane >> 4;
    const int H = p.cache.kv_heads, P = p.cache.page_tokens, group = p.heads / H;
    const int tile = (int)blockIdx.x % tiles, bh = (int)blockIdx.x / tiles, h = bh % H, b = bh / H;
    const Sequence s = sequence(p.batch, b);
    const int r0 = tile * 16;
    if (r0 >= s.n * group) return;
    const int r = r0 + l16, i = r / group;
    const bool real = i < s.n;
    const int pos = s.past + i;                        // of this lane's row
    const int lo = s.past + r0 / group, hi_row = (r0 + 15) / group, hi = s.past + (hi_row < s.n ? hi_row : s.n - 1);
    const Blocks blocks = visible_blocks(lo, hi, p.window, p.sinks);
    const half_t* qrow = p.q + (long long)(s.first + (real ? i : 0)) * p.pitch_q + (h * group + (real ? r - i * group : 0)) * D;

    // Q: dimension of element e of step t: int8 16 g4 + 64 (t / 2) + 8 (t % 2) + e, fp16 8 g4 + 32 t + e
    half8 qf[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t) qf[t] = *(const half8*)(qrow + (I8 ? 16 * g4 + 64 * (t >> 1) + 8 * (t & 1) : 8 * g4 + 32 * t));

    constexpr int J = D / 16;
    floatx4 o[J];
#pragma unroll
    for (int j = 0; j < J; ++j) o[j] = floatx4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    const float c = p.scale * 1.44269504088896340736f * (I8 ? 512.f : 1.f);

    for (int n = 0; n < blocks.count; ++n) {
        const int k0 = blocks.at(n) * KEYS;
        const int page = p.batch.page_table[(long long)b * p.batch.table_pitch + k0 / P];
        if ((unsigned)page >= (unsigned)p.cache.pages) continue;
        const long long place = (long long)page * H + h;
        const long long row0 = place * P + (k0 & (P - 1));
        half8 kf[2][D / 32];
        half8 vf[J];
        if (I8) {
            const int8_t* kp = (const int8_t*)p.cache.k + row0 * D;
            const int8_t* vp = (const int8_t*)p.cache.v + row0 * D;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int u = 0; u < D / 64; ++u) {
                    const uintx4 w = *(const uintx4*)(kp + (kb * 16 + l16) * D + 16 * g4 + 64 * u) ^ 0x80808080u;
#pragma unroll
                    for (int e = 0; e < 16; e += 2) {
                        const half2_t x = two_codes(w[e >> 2], 0, e & 2 ? 0x0c030c02u : 0x0c010c00u);
                        kf[kb][2 * u + (e >> 3)][e & 7] = x[0];
                        kf[kb][2 * u + (e >> 3)][(e & 7) + 1] = x[1];
                    }
                }
            unsigned w[8][J / 4];
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int u = 0; u < J / 4; ++u) w[e][u] = *(const unsigned*)(vp + (16 * (e >> 2) + 4 * g4 + (e & 3)) * D + J * l16 + 4 * u) ^ 0x80808080u;
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const half2_t x = two_codes(w[e][j >> 2], w[e + 1][j >> 2], 0x0c040c00u + 0x00010001u * (j & 3));
                    vf[j][e] = x[0];
                    vf[j][e + 1] = x[1];
                }
        } else {
            const half_t* kp = (const half_t*)p.cache.k + row0 * D;
            const half_t* vp = (const half_t*)p.cache.v + row0 * D;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int t = 0; t < D / 32; ++t) kf[kb][t] = *(const half8*)(kp + (kb * 16 + l16) * D + 8 * g4 + 32 * t);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int key = 16 * (e >> 2) + 4 * g4 + (e & 3);
                // (a value that no row sees may be anything: 0 times an infinity is none of its business)
                const bool seen = k0 + key <= hi && (!p.window || lo - (k0 + key) < p.window || k0 + key < p.sinks);
                half_t v[J];
#pragma unroll
                for (int j = 0; j < J; ++j) v[j] = seen ? vp[key * D + J * l16 + j] : (half_t)0.f;
#pragma unroll
                for (int j = 0; j < J; ++j) vf[j][e] = v[j];
            }
        }
        const float kc = I8 ? p.cache.k_scale[place] * c : c, vs = I8 ? p.cache.v_scale[place] * 512.f : 1.f;
        float sc[8];                                   // keys k0 + 16 kb + 4 g4 + v, at e = 4 kb + v
        float top = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            floatx4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < D / 32; ++t) a = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[kb][t], qf[t], a, 0, 0, 0);
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int key = k0 + 16 * kb + 4 * g4 + v;
                const bool seen = key <= pos && (!p.window || pos - key < p.window || key < p.sinks);
                sc[4 * kb + v] = seen ? a[v] * kc : -INFINITY;
                top = fmaxf(top, sc[4 * kb + v]);
            }
        }
        if (__any(top > m + 8.f)) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float now = fmaxf(m, top), alpha = now > -INFINITY ? __builtin_amdgcn_exp2f(m - now) : 1.f;
            m = now;
            l *= alpha;
#pragma unroll
            for (int j = 0; j < J; ++j) o[j] *= alpha;
        }
        const float ref = m > -INFINITY ? m : 0.f;
        half8 pf;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = __builtin_amdgcn_exp2f(sc[e] - ref);
            l += v;
            pf[e] = (half_t)v;
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (I8) {
                const floatx4 a = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[j], pf, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                for (int v = 0; v < 4; ++v) o[j][v] = __builtin_fmaf(a[v], vs, o[j][v]);
            } else o[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[j], pf, o[j], 0, 0, 0);
        }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    const float inv = l == 0.f ? 0.f : 1.f / l;        // nothing seen: zeros
    if (!real) return;
    half_t* orow = p.out + ((long long)(s.first + i) * p.heads + h * group + r - i * group) * D;
    // lane holds row l16's dimensions J (4 g4 + v) + j
#pragma unroll
    for (int v = 0; v < 4; ++v)
#pragma unroll
        for (int j = 0; j < J; ++j) orow[J * (4 * g4 + v) + j] = (half_t)(o[j][v] * inv);
}

size_t paged_attention_workspace(const PagedAttention&) { return 0; }

int launch_paged_attention(const PagedAttention& p, hipStream_t stream) {
    const int H = p.cache.kv_heads, group = p.heads / H;
    const int tiles = (int)(((long long)p.batch.max_q * group + 15) / 16);
    const long long grid = (long long)p.batch.seqs * H * tiles;
    if (grid > 0x7fffffffLL) { set_error("attention_paged: grid too large"); return STRAIT_E_SHAPE; }
    const bool i8 = p.cache.type == STRAIT_KV_I8;
    auto kernel = p.cache.head_dim == 64 ? (i8 ? paged_attention_kernel<64, true> : paged_attention_kernel<64, false>)
                                         : (i8 ? paged_attention_kernel<128, true> : paged_attention_kernel<128, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64), 0, stream, p, tiles);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("attention_paged launch: %s", hipGetErrorString(e)); return -2; }
    return 0;
}

}  // namespace strait
