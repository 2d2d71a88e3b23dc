// A step's keys and values into a paged cache, rotated by their positions on the way, and the queries rotated with them, for gfx950.
//
//   dimensions (a, b) of a head at position p become (a cos - b sin, b cos + a sin), cos and sin from row p of a table; pairs (j, j + R/2) or (2j, 2j + 1)
//
// One launch.  Queries, and keys and values on their way into an fp16 cache, are worked on token by token: a wavefront or a workgroup has a token, a thread 8 numbers of a head at a
// time, the other halves of its pairs from the cache lines that the threads beside it read anyway.  An int8 cache has a scale for each page and head, so there a
// wavefront (up to 128 pieces of 8 numbers: steps of single tokens) or a workgroup has what a step brings of one page and head, of K or of V: the numbers stay in registers
// from the largest magnitude to their codes, and the page's older codes follow where the scale grows.  Nothing is shared between items, and no order changes a result.
// Every number moves once, 2 bytes in and 1 or 2 out: the memory bounds it, and a step of single tokens is a launch's latency.  128 single tokens of 32 query heads and 8 heads of 128
// in int8 4.4 us; nine chunks of 1 to 900 tokens of the same heads 25.6 us (3.8 TB/s of what moves);
// six prompts of 700 to 2048 tokens, 16 + 16 + 16 heads of 64, fp16, half of each rotated, 27.4 us (3.9 TB/s).
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

// Of the pages that the step's tokens come to lie on, sequence after sequence, the index-th one: its sequence, and its place among the sequence's (false: there are fewer).
__device__ __forceinline__ bool find_page(const strait_kv_batch& batch, int P, int index, int& b, int& c) {
    const int lane = threadIdx.x & 63;
    for (int s0 = 0; s0 < batch.seqs; s0 += 64) {
        int n = 0;
        if (s0 + lane < batch.seqs) {
            const Sequence s = sequence(batch, s0 + lane);
            const int begin = s.past < 0 ? 0 : s.past, end = s.past + s.n;
            n = end > begin ? (end - 1) / P - begin / P + 1 : 0;
        }
        int upto = n;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(upto, d);
            upto += lane >= d ? v : 0;
        }
        const int all = __builtin_amdgcn_readlane(upto, 63);
        if (index < all) {
            const int at = __builtin_ctzll(__ballot(upto > index));
            b = s0 + at;
            c = index - __builtin_amdgcn_readlane(upto - n, at);
            return true;
        }
        index -= all;
    }
    return false;
}

struct AppendGrid {
    int blocks;              // workgroups of the int8 cache's items
    int items;               // (page of the step, head, K or V)
    int pages_each;          // pages that a sequence can come to lie on, each with an item; 0: the items are found by counting
    int token_threads;       // of a token: 64 or 256
    Divisor by_heads, by_pages_each;
};

// Workgroups: first the int8 cache's items, of TPI threads each, which hold ITER pieces of 8 numbers; then tokens.
template <bool I8, int TPI, int ITER>
__global__ void __launch_bounds__(256) kv_append_kernel(const KvAppend p, const AppendGrid grid) {
    __shared__ float part[4];
    if (p.hp) __builtin_amdgcn_s_setprio(3);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int D = p.cache.head_dim, P = p.cache.page_tokens, H = p.cache.kv_heads;
    const int shift = D == 128 ? 4 : 3, per = 1 << shift;               // threads that hold a head
    if (I8 && (int)blockIdx.x < grid.blocks) {
        const int item = TPI == 256 ? (int)blockIdx.x : (int)blockIdx.x * 4 + wave;
        if (item >= grid.items) return;
        const int v = item & 1, i1 = divide(item >> 1, grid.by_heads), h = (item >> 1) - i1 * H;
        int b, c;
        if (grid.pages_each) {
            b = divide(i1, grid.by_pages_each);
            c = i1 - b * grid.pages_each;
        } else if (!find_page(p.batch, P, i1, b, c)) return;
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
        const float old_scale = *scale;
        const half_t* x = (v ? p.v : p.k) + h * D;
        const long long pitch = v ? p.pitch_v : p.pitch_k;
        const int t = TPI == 256 ? (int)threadIdx.x : lane, d = (t & (per - 1)) * 8, sub = t >> shift, rows = TPI >> shift;
        Eight e[ITER];
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int position = lo + sub + i * rows;
            if (position < hi)
                e[i] = rotated<true>(x + (long long)(s.first + position - s.past) * pitch, d, p.rope && !v ? p.rope + (long long)position * p.rope_dim : nullptr, p.rope_dim, p.interleaved);
        }
#pragma unroll
        for (int i = 0; i < ITER; ++i)
            if (lo + sub + i * rows < hi) {
#pragma unroll
                for (int k = 0; k < 8; ++k) top = __builtin_fmaxf(top, __builtin_fabsf(e[i].v[k]));
            }
#pragma unroll
        for (int i = 32; i; i >>= 1) top = __builtin_fmaxf(top, __shfl_xor(top, i));
        if (TPI == 256) {
            if (lane == 0) part[wave] = top;
            __syncthreads();
            top = __builtin_fmaxf(__builtin_fmaxf(part[0], part[1]), __builtin_fmaxf(part[2], part[3]));
        }
        const bool fresh = lo == column * P;
        const float before = fresh ? 0.f : old_scale, candidate = top * (1.f / 127.f), now = candidate > before ? candidate : before;
        if (!fresh && now > before) {
            const float by = before / now;
            uintx2* at = (uintx2*)(codes + d);
            for (int r0 = sub; r0 < lo - column * P; r0 += 4 * rows) {       // (four rows under way)
                uintx2 w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (r0 + k * rows < lo - column * P) w[k] = at[(r0 + k * rows) << shift];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (r0 + k * rows >= lo - column * P) continue;
                    float old[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) old[i] = (float)(int8_t)(w[k][i >> 2] >> (8 * (i & 3)));
                    at[(r0 + k * rows) << shift] = codes_of(old, by);
                }
            }
        }
        const float inverse = now > 0.f ? 1.f / now : 0.f;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int position = lo + sub + i * rows;
            if (position < hi) *(uintx2*)(codes + (position - column * P) * D + d) = codes_of(e[i].v, inverse);
        }
        if (t == 0) *scale = now;
        return;
    }
    const int first = (int)blockIdx.x - grid.blocks, t = grid.token_threads == 256 ? first : first * 4 + wave;
    if (t >= p.batch.tokens) return;
    const int b = sequence_of(p.batch, t);
    if (b < 0) return;
    const Sequence s = sequence(p.batch, b);
    const int i = t - s.first, position = s.past + i;
    if (i < 0 || i >= s.n) return;
    const float* rope = p.rope && position >= 0 ? p.rope + (long long)position * p.rope_dim : nullptr;
    // pieces of 8 numbers: the queries', then, of an fp16 cache, the keys' and the values'
    const int nq = p.heads << shift, nkv = H << shift;
    int column = 0, page = -1;
    if (!I8 && position >= 0) {
        column = position / P;
        page = p.batch.page_table[(long long)b * p.batch.table_pitch + column];
    }
    const int all = (unsigned)page < (unsigned)p.cache.pages ? nq + 2 * nkv : nq;
    const long long row0 = (long long)page * H * P + position - column * P;
    for (int c = threadIdx.x & (grid.token_threads - 1); c < all; c += grid.token_threads) {
        const int what = c < nq ? 0 : c < nq + nkv ? 1 : 2, r = what == 0 ? c : what == 1 ? c - nq : c - nq - nkv, h = r >> shift, d = (r & (per - 1)) * 8;
        const half_t* x = what == 0 ? p.q + t * p.pitch_q : what == 1 ? p.k + t * p.pitch_k : p.v + t * p.pitch_v;
        half_t* at = what == 0 ? p.q_out + ((long long)t * p.heads + h) * D : (half_t*)(what == 1 ? p.cache.k : p.cache.v) + (row0 + (long long)h * P) * D;
        const Eight e = rotated<false>(x + h * D, d, what == 2 ? nullptr : rope, p.rope_dim, p.interleaved);
        __builtin_amdgcn_wave_barrier();               // (q_out may be q: a wavefront has whole heads, and both halves of its pairs before it stores)
        store_half8(at + d, e);
    }
}

int launch_kv_append(const KvAppend& p, hipStream_t stream) {
    const bool i8 = p.cache.type == STRAIT_KV_I8;
    const int P = p.cache.page_tokens;
    AppendGrid g{};
    g.by_heads = divisor(p.cache.kv_heads);
    const int most = p.batch.max_q < P ? p.batch.max_q : P, pieces = most * p.cache.head_dim / 8;     // of an item
    const bool waves = pieces <= 128;
    if (i8) {
        // pages that a sequence's tokens can touch; all sequences' together touch no more than a page per P tokens and two for each
        const long long each = (p.batch.max_q + P - 2) / P + 1, direct = each * p.batch.seqs, counted = p.batch.tokens / P + 2LL * p.batch.seqs;
        if (direct <= counted) { g.pages_each = (int)each; g.by_pages_each = divisor(each); }
        const long long items = (direct <= counted ? direct : counted) * p.cache.kv_heads * 2;
        if (items > MOST_WORKGROUPS) { set_error("kv_append: grid too large"); return STRAIT_E_SHAPE; }
        g.items = (int)items;
        g.blocks = waves ? (g.items + 3) / 4 : g.items;
    }
    // A wavefront for each token, or four where the tokens are too few to fill the units (to 8 times a token's pieces, beside an int8 cache's items 10 times), and where each has so many pieces
    // that its finding does not count.  64 and 256 threads, us, 64-token pages, fp16 cache: 128 single tokens of 80 pieces 4.4 and 3.5, of 768 8.6 and 4.8; chunks of 2048 tokens of 80 4.8 and
    // 5.6, of 288 8.5 and 8.2, of 512 11.5 and 10.0; of 4096 of 80 6.1 and 8.9, of 512 15.2 and 15.6, of 1280 44.5 and 43.5; of 8000 of 384 26.3 and 32.2, of 512 33.2 and 36.7, of 768 51.2
    // and 50.9, of 1280 78.5 and 73.6; of 16384 of 512 59.3 and 69.1; int8: 4096 of 320 14.4 and 15.8, uneven chunks of 4279 of 512 28.4 and 26.1, 8000 of 512 51.7 and 52.6.  Of 250 such
    // pairs the one taken is 6 % slower at most, but for 4096 single tokens of 512 pieces and more, where each wavefront looks for its sequence among so many (768: 46 and 64).
    const long long token_pieces = (p.heads + (i8 ? 0 : 2LL * p.cache.kv_heads)) * p.cache.head_dim / 8;
    g.token_threads = token_pieces * (i8 ? 10 : 8) <= p.batch.tokens && token_pieces <= 768 ? 64 : 256;
    const long long tokens = i8 && !p.heads ? 0 : g.token_threads == 64 ? (p.batch.tokens + 3) / 4 : p.batch.tokens;
    if (g.blocks + tokens > MOST_WORKGROUPS) { set_error("kv_append: grid too large"); return STRAIT_E_SHAPE; }
    const dim3 grid((unsigned)(g.blocks + tokens)), block(256);
    if (!i8) hipLaunchKernelGGL((kv_append_kernel<false, 256, 1>), grid, block, 0, stream, p, g);
    else if (pieces <= 64) hipLaunchKernelGGL((kv_append_kernel<true, 64, 1>), grid, block, 0, stream, p, g);
    else if (waves) hipLaunchKernelGGL((kv_append_kernel<true, 64, 2>), grid, block, 0, stream, p, g);
    else if (pieces <= 512) hipLaunchKernelGGL((kv_append_kernel<true, 256, 2>), grid, block, 0, stream, p, g);
    else if (pieces <= 1024) hipLaunchKernelGGL((kv_append_kernel<true, 256, 4>), grid, block, 0, stream, p, g);
    else if (pieces <= 2048) hipLaunchKernelGGL((kv_append_kernel<true, 256, 8>), grid, block, 0, stream, p, g);
    else hipLaunchKernelGGL((kv_append_kernel<true, 256, 16>), grid, block, 0, stream, p, g);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("kv_append launch: %s", hipGetErrorString(e)); return -2; }
    return 0;
}

}  // namespace strait
