// A step's keys and values into a paged cache, rotated by their positions on the way, and the queries rotated with them, for gfx950.
//
//   dimensions (a, b) of a head at position p become (a cos - b sin, b cos + a sin), cos and sin from row p of a table; pairs (j, j + R/2) or (2j, 2j + 1)
//
// One launch.  Queries, and keys and values on their way into an fp16 cache, are worked on token by token: a wavefront has a token, a lane 8 numbers of a head at a
// time, the other halves of its pairs from the cache lines that the lanes beside it read anyway.  An int8 cache has a scale for each page and head, so there a
// wavefront has what a step brings of one page and head (of K or of V): the largest magnitude first, then the page's older codes where the scale grows,
// then the new codes; nothing is shared between wavefronts, and no order changes a result.
// Every number moves once, 2 bytes in and 1 or 2 out: the memory bounds it, and a step of single tokens is a launch's latency.
#include "decoder.hpp"

namespace strait {

// The definition of an int8 cache's codes names every rounding: products and sums are not contracted here.
#pragma clang fp contract(off)

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));

struct Eight { float v[8]; };

// Dimensions d .. d + 7 of the head at `x`, rotated with the table's row `rope` (nullptr: as they are).  SANE: infinities as 65504, NaN as 0.
template <bool SANE>
__device__ __forceinline__ Eight rotated(const half_t* x, int d, const float* rope, int R, int interleaved) {
    auto load = [](const half_t* at) __attribute__((always_inline)) {
        const half8 h = *(const half8*)at;
        Eight e;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float f = (float)h[i];
            e.v[i] = SANE ? (f != f ? 0.f : __builtin_fminf(__builtin_fmaxf(f, -65504.f), 65504.f)) : f;
        }
        return e;
    };
    Eight e = load(x + d);
    if (!rope || d >= R) return e;
    const int half = R / 2;
    if (interleaved) {
        const floatx4 c = *(const floatx4*)(rope + d / 2), s = *(const floatx4*)(rope + half + d / 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = e.v[2 * i], b = e.v[2 * i + 1];
            e.v[2 * i] = a * c[i] - b * s[i];
            e.v[2 * i + 1] = b * c[i] + a * s[i];
        }
        return e;
    }
    const bool low = d < half;
    const int j = low ? d : d - half;
    const Eight o = load(x + (low ? d + half : j));
    floatx4 c[2], s[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        c[i] = *(const floatx4*)(rope + j + 4 * i);
        s[i] = *(const floatx4*)(rope + half + j + 4 * i);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float ci = c[i >> 2][i & 3], si = s[i >> 2][i & 3];
        e.v[i] = low ? e.v[i] * ci - o.v[i] * si : e.v[i] * ci + o.v[i] * si;
    }
    return e;
}
__device__ __forceinline__ void store_half8(half_t* at, const Eight& e) {
    half8 h;
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = (half_t)e.v[i];
    *(half8*)at = h;
}
__device__ __forceinline__ uintx2 codes_of(const float (&v)[8], float by) {
    uintx2 w = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i >> 2] |= ((unsigned)(int)__builtin_rintf(v[i] * by) & 0xffu) << (8 * (i & 3));
    return w;
}
// The sequence that token t belongs to, found by the whole wavefront: the number of sequences that end at or before it (-1: none; the last with tokens wins no tie,
// since q_start does not decrease).
__device__ __forceinline__ int sequence_of(const strait_kv_batch& b, int t) {
    const int lane = threadIdx.x & 63;
    int ended = 0;
    for (int s = 0; s < b.seqs; s += 64) ended += __popcll(__ballot(s + lane < b.seqs && b.q_start[s + lane + 1] <= t));
    return ended < b.seqs && b.q_start[ended] <= t ? ended : -1;
}

// Items: first the int8 cache's (sequence, page of the step, head, K or V), then tokens; a wavefront each.
template <bool I8>
__global__ void __launch_bounds__(256) kv_append_kernel(const KvAppend p, int page_items, int pages_each) {
    if (p.hp) __builtin_amdgcn_s_setprio(3);
    const int lane = threadIdx.x & 63;
    const int item = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + (int)(threadIdx.x >> 6));
    const int D = p.cache.head_dim, P = p.cache.page_tokens, H = p.cache.kv_heads;
    const int per = D / 8;                              // lanes that hold a head
    if (I8 && item < page_items) {
        const int v = item & 1, h = (item >> 1) % H, c = (item >> 1) / H % pages_each, b = (item >> 1) / H / pages_each;
        const Sequence s = sequence(p.batch, b);
        const int begin = s.past < 0 ? 0 : s.past, end = s.past + s.n;      // positions that are stored
        const int column = begin / P + c;
        const int lo = begin > column * P ? begin : column * P, hi = end < (column + 1) * P ? end : (column + 1) * P;
        if (lo >= hi) return;
        const int page = p.batch.page_table[(long long)b * p.batch.table_pitch + column];
        if ((unsigned)page >= (unsigned)p.cache.pages) return;
        const long long place = (long long)page * H + h;
        int8_t* codes = (int8_t*)(v ? p.cache.v : p.cache.k) + place * P * D;
        float* scale = (v ? p.cache.v_scale : p.cache.k_scale) + place;
        const half_t* x = (v ? p.v : p.k) + h * D;
        const long long pitch = v ? p.pitch_v : p.pitch_k;
        const int d = lane % per * 8, sub = lane / per, rows = 64 / per;
        auto number = [&](int position) __attribute__((always_inline)) {
            return rotated<true>(x + (long long)(s.first + position - s.past) * pitch, d, p.rope && !v ? p.rope + (long long)position * p.rope_dim : nullptr, p.rope_dim, p.interleaved);
        };
        float top = 0.f;
        for (int t = lo + sub; t < hi; t += rows) {
            const Eight e = number(t);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = __builtin_fmaxf(top, __builtin_fabsf(e.v[i]));
        }
#pragma unroll
        for (int i = 32; i; i >>= 1) top = __builtin_fmaxf(top, __shfl_xor(top, i));
        const bool fresh = lo == column * P;
        const float before = fresh ? 0.f : *scale, candidate = top * (1.f / 127.f), now = candidate > before ? candidate : before;
        if (!fresh && now > before) {
            const float by = before / now;
            for (int t = column * P + sub; t < lo; t += rows) {
                uintx2* at = (uintx2*)(codes + (t - column * P) * D + d);
                const uintx2 w = *at;
                float old[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) old[i] = (float)(int8_t)(w[i >> 2] >> (8 * (i & 3)));
                *at = codes_of(old, by);
            }
        }
        const float inverse = now > 0.f ? 1.f / now : 0.f;
        for (int t = lo + sub; t < hi; t += rows) *(uintx2*)(codes + (t - column * P) * D + d) = codes_of(number(t).v, inverse);
        if (lane == 0) *scale = now;
        return;
    }
    const int t = item - page_items;
    if (t >= p.batch.tokens) return;
    const int b = sequence_of(p.batch, t);
    if (b < 0) return;
    const Sequence s = sequence(p.batch, b);
    const int i = t - s.first, position = s.past + i;
    if (i < 0 || i >= s.n) return;
    const float* rope = p.rope && position >= 0 ? p.rope + (long long)position * p.rope_dim : nullptr;
    for (int c = lane; c < p.heads * per; c += 64) {
        const int h = c / per, d = c % per * 8;
        store_half8(p.q_out + ((long long)t * p.heads + h) * D + d, rotated<false>(p.q + t * p.pitch_q + h * D, d, rope, p.rope_dim, p.interleaved));
    }
    if (I8 || position < 0) return;
    const int column = position / P;
    const int page = p.batch.page_table[(long long)b * p.batch.table_pitch + column];
    if ((unsigned)page >= (unsigned)p.cache.pages) return;
    for (int c = lane; c < 2 * H * per; c += 64) {
        const int v = c >= H * per, r = v ? c - H * per : c, h = r / per, d = r % per * 8;
        half_t* at = (half_t*)(v ? p.cache.v : p.cache.k) + (((long long)page * H + h) * P + position - column * P) * D + d;
        store_half8(at, rotated<false>((v ? p.v : p.k) + t * (v ? p.pitch_v : p.pitch_k) + h * D, d, v ? nullptr : rope, p.rope_dim, p.interleaved));
    }
}

int launch_kv_append(const KvAppend& p, hipStream_t stream) {
    const bool i8 = p.cache.type == STRAIT_KV_I8;
    const int pages_each = (p.batch.max_q + p.cache.page_tokens - 2) / p.cache.page_tokens + 1;     // that a sequence's new tokens can touch
    const long long page_items = i8 ? (long long)p.batch.seqs * pages_each * p.cache.kv_heads * 2 : 0;
    const long long items = page_items + (i8 && !p.heads ? 0 : p.batch.tokens);
    if (items > 0x7fffff00LL) { set_error("kv_append: grid too large"); return STRAIT_E_SHAPE; }
    const dim3 grid((unsigned)((items + 3) / 4));
    if (i8) hipLaunchKernelGGL((kv_append_kernel<true>), grid, dim3(256), 0, stream, p, (int)page_items, pages_each);
    else hipLaunchKernelGGL((kv_append_kernel<false>), grid, dim3(256), 0, stream, p, 0, pages_each);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("kv_append launch: %s", hipGetErrorString(e)); return -2; }
    return 0;
}

}  // namespace strait
