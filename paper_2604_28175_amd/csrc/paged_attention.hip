// Attention of a step's tokens over a paged cache, with a causal mask, an optional sliding window and a few first tokens that stay visible, for gfx950.
//
//   out[t, h] = sum_j softmax_j( scale q[t, h] . k_j ) v_j  over the keys j <= p  with  window == 0  or  p - j < window  or  j < sinks
//
// The rows of a tile are (token, head of the group) pairs of one kv head: all of them read the same keys.  The keys that any of them sees come in blocks of
// 32 that lie on one page each.  One pass with a running maximum, which follows the true one only where that is more than 8 (in log2) ahead, so that the output is rescaled a few times
// in all.  Scores, statistics and outputs are fp32; the probabilities are rounded to fp16, half a step each, to be an operand of the second product (2^-32 of the largest one where they are small).
//
//   paged_stream_kernel, tiles of 16 or 32 rows (steps of single tokens, or few): bound by the cache's bytes.  Blocks are shared out over workgroups (parts of `per_part` blocks, whose
//   results a second launch joins) and over a workgroup's four wavefronts, which take every fourth block and meet only at the end:
//   - a wavefront's page numbers and scales are fetched at once, a lane for each block, and named by v_readlane; the next block's bytes are on their way to
//     registers while a block is worked on, and none goes through LDS;
//   - scores^T = K Q^T with v_mfma_f32_16x16x32_f16: a lane names 16 bytes of a key, as they lie in memory, and Q is enumerated in the same order; it then holds
//     8 of the block's keys for ONE row;
//   - an int8 code becomes fp16 by way of the number 2^-24 (code + 128), a subnormal whose bits are the code's: one fused multiply-add makes
//     code 2^-9 of it, exactly.  The scale of the block's page multiplies the scores and the block's share of the output, in fp32;
//   - the probabilities are the "B" operand of out^T = V^T P^T as they are, keys enumerated in the order that the scores came in; V^T's lanes
//     read 8 keys at D / 16 dimensions each and exchange bytes within a lane.
//   32 sequences of 1000 to 16383 tokens, 8 heads of 128 for 32, int8: 118 us, 4.8 TB/s with the join; 24 of 60000 and more, 4 heads for 32, fp16, the last 4096 and 4 of them seen: 47 us, 4.3 TB/s.
//   One sequence of 4100: 9.7 us in a graph, the latency of two launches.
//
//   paged_tile_kernel, 128 rows (prompts and their chunks): bound by the wavefronts' own chain of reads, products, powers and products (at two wavefronts to a SIMD, which the output's registers
//   allow at 128 dimensions, no unit is full: vector instructions 62 % of the time, LDS 31, the matrix pipes 41; at 64 dimensions, three wavefronts and half the products per power, 62, 22 and 29).
//   - 64 keys at a time go through LDS, which holds them twice as fp16: two blocks are worked on, the next two become fp16 on their way from registers to LDS, once
//     for all four wavefronts, and the two after them are on their way from memory;
//   - a wavefront issues in order, so its products and its vector instructions are woven by hand: the way to LDS between the products of the scores, a step's powers between
//     the products that the step before it goes into (a twentieth of the calls below; blocks that none
//     of a wavefront's rows see are worked on all the same, which costs nothing: the others are waited for);
//   - scores^T with v_mfma_f32_32x32x16_f16, a row to a lane and its partner 32 lanes on; V^T's operands come from LDS transposed (ds_read_b64_tr_b16);
//   - an int8 value's power of two is its page's, exact in fp16, and the rest of the page's scale goes into the powers (see look_up).
//   Four chunks of 1200 to 2048 tokens behind up to 2048, 8 heads of 128 for 32, int8: 243 us, 755 TFLOP/s of what the masks leave; five of 333 to 4001 with a window of 1024, 12 heads
//   of 64, fp16: 64 us, 476 TFLOP/s.
#include <float.h>

#include <algorithm>

#include "decoder.hpp"

namespace strait {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));

constexpr int KEYS = 32;                 // of a block
constexpr int NOWHERE = 0x30000000;      // a key behind all others (max_kv is 2^29 at most), and
constexpr int NO_WINDOW = 0x3fffffff;    // a window that holds every key: differences of positions, these and sinks stay in 32 bits
constexpr int PAGED_WAVES = 4;

// Bytes e and e + 1 of a word of codes (biased by 128) as fp16: 0x6400 + byte is 1024 + byte, from which one fused multiply-add takes 1152 and makes any power of two's multiple
__device__ __forceinline__ half2_t scaled_codes(unsigned w, int e, half_t by) {
    const half2_t u = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, w, e ? 0x04030402u : 0x04010400u));
    return __builtin_elementwise_fma(u, half2_t{by, by}, half2_t{(half_t)(-1152.f) * by, (half_t)(-1152.f) * by});
}
// Two of the 8-bit codes in `a` and `b` (biased by 128: codes ^ 0x80) as fp16 code 2^-9; sel: v_perm_b32's selector of the two bytes
__device__ __forceinline__ half2_t two_codes(unsigned a, unsigned b, unsigned sel) {
    const half2_t u = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(b, a, sel));
    const half2_t by = {(half_t)32768.f, (half_t)32768.f}, off = {(half_t)-0.25f, (half_t)-0.25f};
    return __builtin_elementwise_fma(u, by, off);
}

// Probabilities are powers of 2 of score - m, where m is any number that is the same for all of a row's sums.  It is the largest score less
constexpr float ROOM = 7.f;              // (so that the powers use what fp16 holds, up to 2^15: those of far keys become 0 from 2^-32 of the largest one on, not from 2^-25),
constexpr float UNSEEN = -FLT_MAX;       // (before the first one: no score lies further below it than 0, and minus infinity less this is no NaN)
constexpr float LEAD = 15.f;             // whenever one is further ahead of it than this.
// A score is a product, of which m is rounded: a power has to be one of the rounded product too, or for scores of 2^28 and more half a step between them is an overflow.
// Where m is below this, half a step is nothing, and product and difference may be one fused multiply-add.
constexpr float LARGE = 0x1p20f;
// What an int8 page's key scale and the score's scale make: finite and above 0, so that minus infinity stays what it is (a NaN stays one)
__device__ __forceinline__ float factor(float f) { return __builtin_elementwise_minimum(__builtin_elementwise_maximum(f, 0x1p-126f), FLT_MAX); }

// (not to be contracted with what comes after it)
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}

// A sum of probabilities as they were rounded, so that a key which takes nearly all gives its value, whatever its probability was rounded to
__device__ __forceinline__ float plus_both(float sum, half2_t p) { return __builtin_amdgcn_fdot2(p, half2_t{(half_t)1.f, (half_t)1.f}, sum, false); }

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
// The most blocks that a tile of `rows` rows can see.
static int most_blocks(const PagedAttention& p, int rows) {
    const int all = (p.batch.max_kv + KEYS - 1) / KEYS;
    if (!p.window) return all;
    const int group = p.heads / p.cache.kv_heads, apart = (rows + group - 2) / group;      // positions of two rows
    return (int)std::min<long long>(all, ((long long)apart + p.window - 1) / KEYS + 2 + (p.sinks + KEYS - 1) / KEYS);
}

struct PagedArgs {
    PagedAttention p;
    int group;                           // query heads of a kv head
    int from, to;                        // of sequences with more than `from` and at most `to` rows (new tokens times group) of a kv head
    int tiles, rows;                     // tiles of a sequence's rows and head, rows of a tile
    int items;                           // (sequence, tile) pairs that are found by counting; 0: each sequence has `tiles`
    int per_part, parts;                 // blocks of a part, parts at most
    int join_tokens;                     // of each sequence that the join looks at; 0: all tokens, of which it finds the sequences
    int slots;                           // parts of a row that the workspace has room for
    float* o; float* ml;                 // of parts: [joined tokens][heads][slots][D] and [..][2]: the output over the sum, the maximum and the sum
    Divisor by_group, by_heads, by_seqs, by_tiles, by_items, by_q_heads, by_join;
};

// A tile's rows: of sequence s, lo .. hi the positions of the first and last one.
struct Tile { int r0, lo, hi; bool any; };
__device__ __forceinline__ Tile tile_of(const PagedArgs& a, const Sequence& s, int tile) {
    const int r0 = tile * a.rows, last = divide(r0 + a.rows - 1, a.by_group), rows = s.n * a.group;
    return {r0, s.past + divide(r0, a.by_group), s.past + (last < s.n ? last : s.n - 1), r0 < rows && rows > a.from && rows <= a.to};
}

// Where the parts of a sequence's i-th token lie: joined tokens are numbered by sequence, or as they come.
__device__ __forceinline__ long long joined_token(const PagedArgs& a, int b, const Sequence& s, int i) {
    return a.join_tokens ? (long long)b * a.join_tokens + i : s.first + i;
}

// Workgroup ((part tiles + tile) seqs + b') heads + h: every sequence's first part comes before any second one, a sequence's last tile, which sees the most keys, before the others,
// and a head stays on a chiplet where there are 8.  The hardware deals workgroups out to the parts of a chiplet in turn and in order, one that is full holding up the others; so
// that no part of it gets the longest sequence of every round, the sequences are moved on by one from round to round (chunks of four prompts: 0.56 -> 0.85 of the places busy).
// Where sequences bring uneven numbers of tokens most of those workgroups would have none: then (part items + item) heads + h, the item-th of the tiles that there are, found by counting.
__device__ __forceinline__ bool place_item(const PagedArgs& a, int item, int& h, int& b, int& part, int& tile) {
    const int i1 = divide(item, a.by_heads);
    h = item - i1 * a.p.cache.kv_heads;
    if (!a.items) {
        const int i2 = divide(i1, a.by_seqs);
        b = i1 - i2 * a.p.batch.seqs + i2 - divide(i2, a.by_seqs) * a.p.batch.seqs;
        if (b >= a.p.batch.seqs) b -= a.p.batch.seqs;
        part = divide(i2, a.by_tiles);
        tile = a.tiles - 1 - (i2 - part * a.tiles);
        return true;
    }
    part = divide(i1, a.by_items);
    int index = i1 - part * a.items;
    const int lane = threadIdx.x & 63;
    for (int s0 = 0; s0 < a.p.batch.seqs; s0 += 64) {
        int n = 0;
        if (s0 + lane < a.p.batch.seqs) {
            const int rows = sequence(a.p.batch, s0 + lane).n * a.group;
            n = rows > a.from && rows <= a.to ? (rows + a.rows - 1) / a.rows : 0;
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
            tile = __builtin_amdgcn_readlane(upto, at) - 1 - index;
            return true;
        }
        index -= all;
    }
    return false;
}

// A block's bytes as they come from memory: keys 16 kb + l16 at 16-byte pieces of their dimensions, and the values of 8 keys at J dimensions.
template <int D, bool I8>
struct RawBlock {
    static constexpr int KP = D * (I8 ? 1 : 2) / 64, VW = D / 16 * (I8 ? 1 : 2) / 4;       // pieces of a key per lane; words of a value
    uintx4 k[2][KP];
    unsigned v[8][VW];
    __device__ __forceinline__ void load_k(const strait_kv_cache& c, int place, int row, int l16, int g4) {
        const char* kp = (const char*)c.k + ((long long)place * c.page_tokens + row) * (D * (I8 ? 1 : 2));
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int u = 0; u < KP; ++u) k[kb][u] = *(const uintx4*)(kp + (unsigned)((kb * 16 + l16) * KP * 64 + 16 * g4 + 64 * u));
    }
    __device__ __forceinline__ void load_v(const strait_kv_cache& c, int place, int row, int l16, int g4) {
        const char* vp = (const char*)c.v + ((long long)place * c.page_tokens + row) * (D * (I8 ? 1 : 2));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const char* src = vp + (unsigned)((16 * (e >> 2) + 4 * g4 + (e & 3)) * KP * 64 + l16 * VW * 4);
            if constexpr (VW == 4) *(uintx4*)v[e] = *(const uintx4*)src;
            else if constexpr (VW == 2) *(uint2*)v[e] = *(const uint2*)src;
            else v[e][0] = *(const unsigned*)src;
        }
    }
};

template <int D, bool I8, int RT>
__global__ void __launch_bounds__(64 * PAGED_WAVES, 2) paged_stream_kernel(const PagedArgs a) {
    constexpr int J = D / 16, LDO = D + 4;
    constexpr bool AHEAD = D == 64 || I8 || RT == 1;   // registers for a whole block beside the one that is worked on (two rows' tiles of fp16: the next keys where these are done with)
    __shared__ float so[2][RT * 16][LDO];
    __shared__ float sml[2][RT * 16][2];
    const PagedAttention& p = a.p;
    if (p.hp) __builtin_amdgcn_s_setprio(3);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l16 = lane & 15, g4 = lane >> 4;
    const int H = p.cache.kv_heads, P = p.cache.page_tokens;
    int h, b, part, tile;
    if (!place_item(a, (int)blockIdx.x, h, b, part, tile)) return;
    const Sequence s = sequence(p.batch, b);
    const Tile t = tile_of(a, s, tile);
    if (!t.any) return;
    const Blocks blocks = visible_blocks(t.lo, t.hi, p.window, p.sinks);
    const int begin = part * a.per_part, end = begin + a.per_part < blocks.count ? begin + a.per_part : blocks.count;
    if (part && begin >= end) return;

    // Q: dimension of element e of step u: int8 16 g4 + 64 (u / 2) + 8 (u % 2) + e, fp16 8 g4 + 32 u + e
    half8 qf[RT][D / 32];
    int pos[RT], head[RT], token[RT];                  // of this lane's rows
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        const int r = t.r0 + 16 * x + l16, i = divide(r, a.by_group);
        head[x] = h * a.group + r - i * a.group;
        token[x] = i < s.n ? s.first + i : -1;
        pos[x] = s.past + i;
        const half_t* qrow = p.q + (long long)(token[x] < 0 ? s.first : token[x]) * p.pitch_q + head[x] * D;
#pragma unroll
        for (int u = 0; u < D / 32; ++u) qf[x][u] = *(const half8*)(qrow + (I8 ? 16 * g4 + 64 * (u >> 1) + 8 * (u & 1) : 8 * g4 + 32 * u));
    }
    floatx4 o[RT][J];
    float m[RT], l[RT];
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        m[x] = UNSEEN;
        l[x] = 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j) o[x][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    const float c = factor(p.scale * 1.44269504088896340736f);

    // whether a row sees the key `off` behind some key of which it is `past` tokens past and which is `sinks` keys in front of the last sink
    const int window = p.window ? p.window : NO_WINDOW;
    auto sees = [&](int off, int past, int sinks) __attribute__((always_inline)) { return off <= past && (off > past - window || off < sinks); };
    // keys_done, values_done: when the registers of a block's keys and values are free
    auto work = [&](const RawBlock<D, I8>& raw, int k0, float kc, float vs, bool mask, auto keys_done, auto values_done) __attribute__((always_inline)) {
        half8 kf[2][D / 32];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int u = 0; u < RawBlock<D, I8>::KP; ++u) {
                if constexpr (I8) {
                    const uintx4 w = raw.k[kb][u] ^ 0x80808080u;
#pragma unroll
                    for (int e = 0; e < 16; e += 2) {
                        const half2_t y = two_codes(w[e >> 2], 0, e & 2 ? 0x0c030c02u : 0x0c010c00u);
                        kf[kb][2 * u + (e >> 3)][e & 7] = y[0];
                        kf[kb][2 * u + (e >> 3)][(e & 7) + 1] = y[1];
                    }
                } else kf[kb][u] = __builtin_bit_cast(half8, raw.k[kb][u]);
            }
        half8 pf[RT];
#pragma unroll
        for (int x = 0; x < RT; ++x) {
            float sc[8];                               // keys k0 + 16 kb + 4 g4 + v, at e = 4 kb + v
            float top = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                floatx4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int u = 0; u < D / 32; ++u) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[kb][u], qf[x][u], d, 0, 0, 0);
#pragma unroll
                for (int v = 0; v < 4; ++v) sc[4 * kb + v] = rounded_product(d[v], kc);
            }
            if (mask) {
                asm volatile("");                      // (a branch: most blocks have nothing to mask)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!sees(16 * (e >> 2) + (e & 3), pos[x] - k0 - 4 * g4, p.sinks - k0 - 4 * g4)) sc[e] = -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, sc[e]);
            if (__any(top - m[x] > LEAD)) {
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float now = fmaxf(m[x], top - ROOM), alpha = __builtin_amdgcn_exp2f(m[x] - now);
                m[x] = now;
                l[x] *= alpha;
#pragma unroll
                for (int j = 0; j < J; ++j) o[x][j] *= alpha;
            }
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const half2_t y = {(half_t)__builtin_amdgcn_exp2f(sc[e] - m[x]), (half_t)__builtin_amdgcn_exp2f(sc[e + 1] - m[x])};
                l[x] = plus_both(l[x], y);
                pf[x][e] = y[0];
                pf[x][e + 1] = y[1];
            }
        }
        keys_done();
        unsigned w[8][RawBlock<D, I8>::VW];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            // (a value that no row sees may be anything: 0 times an infinity is none of its business)
            const int key = k0 + 16 * (e >> 2) + 4 * g4 + (e & 3);
            const bool seen = !mask || I8 || (key <= t.hi && (!p.window || t.lo - key < p.window || key < p.sinks));
#pragma unroll
            for (int u = 0; u < RawBlock<D, I8>::VW; ++u) w[e][u] = I8 ? raw.v[e][u] ^ 0x80808080u : seen ? raw.v[e][u] : 0u;
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
            half8 vf;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                half2_t y;
                if constexpr (I8) y = two_codes(w[e][j >> 2], w[e + 1][j >> 2], 0x0c040c00u + 0x00010001u * (j & 3));
                else y = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(w[e + 1][j >> 1], w[e][j >> 1], j & 1 ? 0x07060302u : 0x05040100u));
                vf[e] = y[0];
                vf[e + 1] = y[1];
            }
#pragma unroll
            for (int x = 0; x < RT; ++x) {
                if constexpr (I8) {
                    const floatx4 d = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[x], floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                    for (int v = 0; v < 4; ++v) o[x][j][v] = __builtin_fmaf(d[v], vs, o[x][j][v]);
                } else o[x][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[x], o[x][j], 0, 0, 0);
            }
        }
        values_done();
    };

    // 64 of this wavefront's blocks at a time
    for (int first = begin + wave; first < end; first += 64 * PAGED_WAVES) {
        const int mine = first + PAGED_WAVES * lane;
        int k0s = 0, places = -1;
        float kcs = 0.f, vss = 0.f;
        if (mine < end) {
            k0s = blocks.at(mine) * KEYS;
            const int page = p.batch.page_table[(long long)b * p.batch.table_pitch + k0s / P];
            if ((unsigned)page < (unsigned)p.cache.pages) {
                places = page * H + h;
                if (I8) { kcs = factor(p.cache.k_scale[places] * 512.f * c); vss = p.cache.v_scale[places] * 512.f; }
            }
        }
        unsigned long long left = __ballot(places >= 0);
        if (!left) continue;
        RawBlock<D, I8> next;
        int ni = __builtin_ctzll(left);
        auto next_k = [&]() __attribute__((always_inline)) { next.load_k(p.cache, __builtin_amdgcn_readlane(places, ni), __builtin_amdgcn_readlane(k0s, ni) & (P - 1), l16, g4); };
        auto next_v = [&]() __attribute__((always_inline)) { next.load_v(p.cache, __builtin_amdgcn_readlane(places, ni), __builtin_amdgcn_readlane(k0s, ni) & (P - 1), l16, g4); };
        next_k();
        next_v();
        while (left) {
            const int i = ni, k0 = __builtin_amdgcn_readlane(k0s, i);
            const float kc = I8 ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, kcs), i)) : c;
            const float vs = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, vss), i));
            const bool mask = !(k0 + KEYS - 1 <= t.lo && (!p.window || t.hi - k0 < p.window || k0 + KEYS - 1 < p.sinks));
            left &= left - 1;
            if (left) ni = __builtin_ctzll(left);
            if constexpr (AHEAD) {
                const RawBlock<D, I8> raw = next;
                if (left) {
                    next_k();
                    next_v();
                }
                work(raw, k0, kc, vs, mask, [] {}, [] {});
            } else {                                   // (behind the last block: that one again)
                work(next, k0, kc, vs, mask, next_k, next_v);
            }
        }
    }
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        l[x] += __shfl_xor(l[x], 16);
        l[x] += __shfl_xor(l[x], 32);
    }
    // four wavefronts' results become one: 2 and 3 hand theirs to 0 and 1, then 1 to 0; a lane holds row l16's dimensions J (4 g4 + v) + j
    auto put = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < RT; ++x) {
            float* row = so[slot][16 * x + l16];
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
                for (int j = 0; j < J; j += 4) *(floatx4*)(row + J * (4 * g4 + v) + j) = floatx4{o[x][j][v], o[x][j + 1][v], o[x][j + 2][v], o[x][j + 3][v]};
            if (g4 == 0) { sml[slot][16 * x + l16][0] = m[x]; sml[slot][16 * x + l16][1] = l[x]; }
        }
    };
    auto take = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < RT; ++x) {
            const float m2 = sml[slot][16 * x + l16][0], l2 = sml[slot][16 * x + l16][1], now = fmaxf(m[x], m2);
            const float a1 = __builtin_amdgcn_exp2f(m[x] - now), a2 = __builtin_amdgcn_exp2f(m2 - now);
            m[x] = now;
            l[x] = l[x] * a1 + l2 * a2;
            const float* row = so[slot][16 * x + l16];
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
                for (int j = 0; j < J; j += 4) {
                    const floatx4 y = *(const floatx4*)(row + J * (4 * g4 + v) + j);
#pragma unroll
                    for (int k = 0; k < 4; ++k) o[x][j + k][v] = o[x][j + k][v] * a1 + y[k] * a2;
                }
        }
    };
    if (wave >= 2) put(wave - 2);
    __syncthreads();
    if (wave < 2) take(wave);
    __syncthreads();
    if (wave == 1) put(0);
    __syncthreads();
    if (wave) return;
    take(0);
    const bool whole = blocks.count <= a.per_part;
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        if (token[x] < 0) continue;
        const float inv = l[x] == 0.f ? 0.f : 1.f / l[x];      // nothing seen: zeros
        if (whole) {
            half_t* out = p.out + ((long long)token[x] * p.heads + head[x]) * D;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                half_t y[J];
#pragma unroll
                for (int j = 0; j < J; ++j) y[j] = (half_t)(o[x][j][v] * inv);
                if constexpr (J == 8) *(uintx4*)(out + J * (4 * g4 + v)) = *(const uintx4*)y;
                else *(uint2*)(out + J * (4 * g4 + v)) = *(const uint2*)y;
            }
        } else {
            const long long slot = (joined_token(a, b, s, token[x] - s.first) * p.heads + head[x]) * a.slots + part;
            float* out = a.o + slot * D;
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
                for (int j = 0; j < J; j += 4) *(floatx4*)(out + J * (4 * g4 + v) + j) = floatx4{o[x][j][v], o[x][j + 1][v], o[x][j + 2][v], o[x][j + 3][v]} * inv;
            if (g4 == 0) *(float2*)(a.ml + slot * 2) = make_float2(m[x], l[x]);
        }
    }
}

// ---- many rows ----------------------------------------------------------------------------------------------------------

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __fp16 fp16x4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));

// The value of this lane and of lane ^ 32: {lanes 0-31's, lanes 32-63's}.
__device__ __forceinline__ float2 halves_of(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    const unsigned lo = r[0], hi = r[1];
    return {__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi)};
}

constexpr int TILE_KEYS = 64;            // two blocks
constexpr float VALUE = 128.f;           // what is left out of the values of an int8 cache until the end

template <int D, bool I8>
__global__ void __launch_bounds__(64 * PAGED_WAVES, 2) paged_tile_kernel(const PagedArgs a) {
    constexpr int NT = 64 * PAGED_WAVES, ROW = D * 2, STAGE = 2 * TILE_KEYS * ROW;      // bytes of a row of K or V in LDS, of a stage
    constexpr int ES = I8 ? 1 : 2, PER_ROW = D * ES / 16, HALF = TILE_KEYS * PER_ROW, NI = 2 * HALF / NT;   // 16-byte pieces in memory: of a row, of K; of a thread
    static_assert(HALF % NT == 0, "pieces");
    extern __shared__ __attribute__((aligned(16))) char tile_lds[];    // two stages
    const PagedAttention& p = a.p;
    if (p.hp) __builtin_amdgcn_s_setprio(3);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, lh = lane >> 5;
    const int H = p.cache.kv_heads, P = p.cache.page_tokens;
    int h, b, part, tile;
    if (!place_item(a, (int)blockIdx.x, h, b, part, tile)) return;
    const Sequence s = sequence(p.batch, b);
    const Tile t = tile_of(a, s, tile);
    if (!t.any) return;
    const Blocks blocks = visible_blocks(t.lo, t.hi, p.window, p.sinks);
    const int begin = part * a.per_part, end = begin + a.per_part < blocks.count ? begin + a.per_part : blocks.count;
    if (part && begin >= end) return;

    // this lane's row, and the positions that the wavefront's rows span
    const int r0 = t.r0 + wave * 32, r = r0 + l32, i = divide(r, a.by_group), head = h * a.group + r - i * a.group;
    const int token = i < s.n ? s.first + i : -1, pos = s.past + i;
    const bool any = r0 < s.n * a.group;
    const int lo = s.past + divide(r0, a.by_group), hi_i = divide(r0 + 31, a.by_group), hi = s.past + (hi_i < s.n ? hi_i : s.n - 1);
    half8 qf[D / 16];
    {
        const half_t* qrow = p.q + (long long)(token < 0 ? s.first : token) * p.pitch_q + head * D;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *(const half8*)(qrow + ks * 16 + lh * 8);
    }
    floatx16 o[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[db][v] = 0.f;
    float m = UNSEEN, l = 0.f;
    bool large = false;                                // of some row's m
    const float c = factor(p.scale * 1.44269504088896340736f);

    // ---- memory -> registers -> LDS.  Chunk q of 16 bytes of row r lies at q ^ (r % 16) for K (D = 64: r / 2 % 8, two rows to the width of the banks), whose operand is 16 rows at one
    // chunk.  V's operand is 4 rows at 4 chunks at a time: the rows' bits go to the chunk's bits above those.  Eight lanes store at a time, and codes go to every second chunk: so that they meet
    // no bank twice, they are those of two rows (lanes' bits 2 and 3 change places) whose chunks differ in the lowest bit.
    auto kswz = [](int row) { return D == 128 ? row & 15 : row >> 1 & 7; };
    auto vswz = [](int row) { return D == 128 ? (row & 3) << 2 | (row & 1) : (row & 2) << 1 | (row >> 1 & 1); };
    const int ptid = I8 ? (tid & ~12) | (tid & 4) << 1 | (tid & 8) >> 1 : tid;
    uintx4 raw[NI];
    // A lane of each wavefront holds what is to be known of a block: where it begins (behind all rows: not seen) and lies in the cache, and its scales; masks say
    // which of the 64 blocks all of the wavefront's rows see whole, of which each key is seen by some row of the tile, and of which the rest of the values'
    // scale is below 1.
    int k0s = 0;
    unsigned from_lo = 0, from_hi = 0;
    float kcs = c, vpow = 1.f, vlog = 0.f, vinv = 1.f;
    unsigned long long full = 0, open = 0, tiny = 0;
    auto look_up = [&](int first) __attribute__((always_inline)) {
        k0s = NOWHERE;
        from_lo = from_hi = 0;
        if (first + lane < end) {
            const int k0 = blocks.at(first + lane) * KEYS, page = p.batch.page_table[(long long)b * p.batch.table_pitch + k0 / P];
            if ((unsigned)page < (unsigned)p.cache.pages) {
                const int place = page * H + h;
                const unsigned long long from = ((unsigned long long)place * P + (k0 & (P - 1))) * (D * ES);
                k0s = k0;
                from_lo = (unsigned)from;
                from_hi = (unsigned)(from >> 32);
                if (I8) {
                    kcs = factor(p.cache.k_scale[place] * c);
                    // a value is 2^7 code 2^f: code 2^f is exact in fp16, f between -24 and 5 (1152 2^f is a number of fp16 too), and 2^7 comes at the end; the rest of the page's scale, between
                    // 1 and 2 for scales of 2^-17 to 8192, goes into the powers.  Scales below 2^-60, of which no output would show a bit, count as 0: the rest would take the powers out of fp32.
                    const float vs = p.cache.v_scale[place] < 0x1p-60f ? 0.f : p.cache.v_scale[place];
                    vpow = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, vs) & 0x7f800000u) * (1.f / VALUE);
                    vpow = vs == 0.f ? 0.f : fminf(fmaxf(vpow, 0x1p-24f), 0x1p5f);
                    const float ratio = vs == 0.f ? 1.f : vs / (vpow * VALUE);
                    vlog = __builtin_amdgcn_logf(ratio);
                    vinv = 1.f / ratio;
                }
            }
        }
        full = __ballot(k0s + KEYS - 1 <= lo && (!p.window || hi - k0s < p.window || k0s + KEYS - 1 < p.sinks));
        if (I8) tiny = __ballot(vinv > 1.f);
        else open = __ballot(k0s + KEYS - 1 <= t.hi && (!p.window || t.lo - k0s < p.window || k0s + KEYS - 1 < p.sinks));
    };
    auto of_block = [](int v, int n) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(v, n); };
    auto of_blockf = [](float v, int n) __attribute__((always_inline)) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), n)); };
    auto fetch = [&](int n) __attribute__((always_inline)) {       // blocks n and n + 1 of the 64 that were looked up
#pragma unroll
        for (int x = 0; x < NI; ++x) {
            const int v = x * NT >= HALF, rem = x * NT + ptid - v * HALF, row = rem / PER_ROW;
            const int blk = n + (PER_ROW * KEYS >= NT ? x * NT % HALF / (PER_ROW * KEYS) : __builtin_amdgcn_readfirstlane(row >> 5));
            const unsigned long long from = (unsigned long long)(unsigned)of_block((int)from_hi, blk) << 32 | (unsigned)of_block((int)from_lo, blk);
            raw[x] = *(const uintx4*)((const char*)(v ? p.cache.v : p.cache.k) + from + (unsigned)(rem & (KEYS * PER_ROW - 1)) * 16u);
        }
    };
    // Of what was fetched of blocks n and n + 1, the q-th of 2 D / 16 equal shares: a word of codes, or half a piece (that is, every second time a piece).
    constexpr int SHARES = D / 8;
    static_assert(I8 ? SHARES == 4 * NI : SHARES == 2 * NI, "shares");
    half8 widened;
    auto stage = [&](int q, int n, int st) __attribute__((always_inline)) {
        if (!I8 && q % 2 == 0) return;
        const int x = I8 ? q / 4 : q / 2, v = x * NT >= HALF, rem = x * NT + ptid - v * HALF, row = rem / PER_ROW, piece = rem % PER_ROW;
        char* dst = tile_lds + st * STAGE + v * (TILE_KEYS * ROW) + row * ROW;
        const int swz = v ? vswz(row) : kswz(row);
        if constexpr (I8) {
            unsigned w = raw[x][q % 4];
            asm volatile("" : "+v"(w));                 // (its bytes are spread here, not ahead of all products)
            w ^= 0x80808080u;
            const half_t by = v ? (half_t)of_blockf(vpow, __builtin_amdgcn_readfirstlane(n + (row >> 5))) : (half_t)1.f;
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const half2_t z = scaled_codes(w, e, by);
                widened[q % 2 * 4 + e] = z[0];
                widened[q % 2 * 4 + e + 1] = z[1];
            }
            if (q % 2) *(half8*)(dst + ((2 * piece + q % 4 / 2) ^ swz) * 16) = widened;
        } else {
            if ((open >> n & 3) != 3) {                // what no row of the tile sees may be anything: it becomes zeros (of int8 it is finite, and its probability 0)
                const int key = of_block(k0s, __builtin_amdgcn_readfirstlane(n + (row >> 5))) + (row & 31);
                if (!(key <= t.hi && (!p.window || t.lo - key < p.window || key < p.sinks))) raw[x] = uintx4{0, 0, 0, 0};
            }
            *(uintx4*)(dst + (piece ^ swz) * 16) = raw[x];
        }
    };
    auto stage_all = [&](int n, int st) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < SHARES; ++q) stage(q, n, st);
    };

    // V: lane i of a group of 16 names keys 4 lh + (i >> 2), dimensions 16 ((lane >> 4) & 1) + 4 (i & 3) .. + 3 of a 16-key step and 32 dimensions, and receives
    // the step's keys 4 lh .. 4 lh + 3 of dimension 16 ((lane >> 4) & 1) + i
    const unsigned lds0 = (unsigned)(uintptr_t)tile_lds;
    const int i16 = lane & 15, vr = lh * 4 + (i16 >> 2);
    unsigned vaddr[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
        vaddr[db] = lds0 + TILE_KEYS * ROW + vr * ROW + (((db * 4 + ((lane >> 4) & 1) * 2 + ((i16 & 3) >> 1)) ^ vswz(vr)) << 4) + (i16 & 1) * 8;
    auto vread = [](unsigned at) { return __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) fp16x4*)(uintptr_t)at); };

    // whether a row sees the key `off` behind some key of which it is `past` tokens past and which is `sinks` keys in front of the last sink
    const int window = p.window ? p.window : NO_WINDOW;
    auto sees = [&](int off, int past, int sinks) __attribute__((always_inline)) { return off <= past && (off > past - window || off < sinks); };
    // Blocks n and n + 1 from stage st.  A wavefront issues in order, and a product holds the matrix pipe for 8 vector instructions: so that these run beside it, each product of the scores
    // is followed by a share of the next two blocks' way to LDS, and each of the output by powers that the next ones need.
    auto work = [&](int n, int st, bool mask, auto scores_done) __attribute__((always_inline)) {
        const char* ks0 = tile_lds + st * STAGE;
        floatx16 sc[2];                                // lane holds its row against keys 32 kb + 8 g + 4 lh + j of the tile (v = 4 g + j)
        float kc[2], most[2];
        half8 kf[D / 16];
        auto read_key = [&](int kb, int ks) __attribute__((always_inline)) { kf[ks] = *(const half8*)(ks0 + (kb * 32 + l32) * ROW + (((ks * 2 + lh) ^ kswz(l32)) << 4)); };
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) read_key(0, ks);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int v = 0; v < 16; ++v) sc[kb][v] = 0.f;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                sc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[ks], qf[ks], sc[kb], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
                if (kb == 0) read_key(1, ks);
                stage(kb * (D / 16) + ks, (n + 2) & 63, st ^ 1);      // (behind the last block: what is there already, where nobody looks)
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        scores_done();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            kc[kb] = I8 ? of_blockf(kcs, n + kb) : c;
            if (mask) {
                asm volatile("");                      // (a branch: most blocks have nothing to mask)
                const int k0 = of_block(k0s, n + kb);
#pragma unroll
                for (int v = 0; v < 16; ++v) sc[kb][v] = sees(8 * (v >> 2) + (v & 3), pos - k0 - 4 * lh, p.sinks - k0 - 4 * lh) ? sc[kb][v] : -INFINITY;
            }
            most[kb] = sc[kb][0];
#pragma unroll
            for (int v = 1; v < 16; ++v) most[kb] = fmaxf(most[kb], sc[kb][v]);
        }
        // (what is added to a block's scores; here the scores' maximum is one of the powers' exponents, the rest of a page's scale among them)
        float rest[2], off[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            rest[kb] = I8 ? of_blockf(vlog, n + kb) : 0.f;
            off[kb] = rest[kb] - m;
        }
        if (__any(fmaxf(__builtin_fmaf(most[0], kc[0], off[0]), __builtin_fmaf(most[1], kc[1], off[1])) > LEAD)) {
            const float2 both = halves_of(fmaxf(rounded_product(most[0], kc[0]) + rest[0], rounded_product(most[1], kc[1]) + rest[1]));
            const float now = fmaxf(m, fmaxf(both.x, both.y) - ROOM), alpha = __builtin_amdgcn_exp2f(m - now);
            m = now;
            off[0] = rest[0] - m;
            off[1] = rest[1] - m;
            large = __any(fabsf(m) > LARGE && m != UNSEEN);
            l *= alpha;
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[db][v] *= alpha;
        }
        __builtin_amdgcn_sched_barrier(0);
        // four steps of 16 keys each
        half8 pf[2], vf[D / 32];
        float sum[2] = {0.f, 0.f}, exact[2] = {-1.f, -1.f};
        unsigned vbase[D / 32];
        if (large) {                                   // (no power beyond what fp16 holds: off may have lost the page's part of it)
            asm volatile("");
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
                for (int v = 0; v < 16; ++v) sc[kb][v] = __builtin_elementwise_minimum(rounded_product(sc[kb][v], kc[kb]) + off[kb], LEAD);
                kc[kb] = 1.f;
                off[kb] = 0.f;
            }
        }
        if (I8 && (tiny >> n & 3)) {                   // (with the rest of such a scale in them, probabilities may leave nothing in fp16: summed before they are rounded)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                exact[kb] = 0.f;
#pragma unroll
                for (int v = 0; v < 16; ++v) exact[kb] += __builtin_amdgcn_exp2f(__builtin_fmaf(sc[kb][v], kc[kb], off[kb]));
            }
        }
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
            vbase[db] = vaddr[db] + (unsigned)(st * STAGE);
            asm("" : "+v"(vbase[db]));                 // (one addition, and what follows in the instructions' offsets)
        }
        auto read_values = [&](int step, int db) __attribute__((always_inline)) {
            const fp16x4 lo4 = vread(vbase[db] + step * 16 * ROW), hi4 = vread(vbase[db] + (step * 16 + 8) * ROW);
#pragma unroll
            for (int j = 0; j < 4; ++j) { vf[db][j] = (half_t)lo4[j]; vf[db][4 + j] = (half_t)hi4[j]; }
        };
        // two of a step's 8 probabilities of this lane: computed and summed here, neither ahead of the products nor behind them all
        auto powers = [&](int step, int j) __attribute__((always_inline)) {
            const int kb = step >> 1, at = 8 * (step & 1) + j;
            float x = sc[kb][at], y = sc[kb][at + 1];
            asm volatile("" : "+v"(x), "+v"(y));
            x = __builtin_amdgcn_exp2f(__builtin_fmaf(x, kc[kb], off[kb]));
            y = __builtin_amdgcn_exp2f(__builtin_fmaf(y, kc[kb], off[kb]));
            const half2_t both = {(half_t)x, (half_t)y};
            sum[kb] = plus_both(sum[kb], both);
            asm volatile("" : "+v"(sum[kb]));
            pf[step & 1][j] = both[0];
            pf[step & 1][j + 1] = both[1];
        };
#pragma unroll
        for (int db = 0; db < D / 32; ++db) read_values(0, db);
#pragma unroll
        for (int j = 0; j < 8; j += 2) powers(0, j);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int step = 0; step < 4; ++step)
#pragma unroll
            for (int db = 0; db < D / 32; ++db) {
                o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[db], pf[step & 1], o[db], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
                if (step < 3) {
                    constexpr int EACH = 8 / (D / 32);
                    read_values(step + 1, db);
#pragma unroll
                    for (int j = 0; j < EACH; j += 2) powers(step + 1, db * EACH + j);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) l = I8 ? __builtin_fmaf(exact[kb] < 0.f ? sum[kb] : exact[kb], of_blockf(vinv, n + kb), l) : l + sum[kb];
    };

    // 64 blocks that are looked up at once: two of them in LDS and worked on, two in registers on their way there, two more requested once these are written
    for (int first = begin; first < end; first += 64) {
        const int count = end - first < 64 ? end - first : 64;
        look_up(first);
        fetch(0);
        stage_all(0, 0);
        if (count > 2) fetch(2);
        __syncthreads();
        for (int n = 0, st = 0; n < count; n += 2, st ^= 1) {
            auto next = [&]() __attribute__((always_inline)) {
                if (n + 4 < count) fetch(n + 4);
                else {
#pragma unroll
                    for (int x = 0; x < NI; ++x) raw[x] = uintx4{0, 0, 0, 0};      // (rather than keep what is there, in other registers than what a fetch brings)
                }
            };
            work(n, st, (full >> n & 3) != 3, next);
            __syncthreads();
        }
    }
    const float2 ll = halves_of(l);
    l = ll.x + ll.y;
    if (!any) return;
    const float inv = l == 0.f ? 0.f : (I8 ? VALUE : 1.f) / l;         // nothing seen: zeros
    const bool whole = blocks.count <= a.per_part;
    if (whole) {
        half_t* out = p.out + ((long long)(token < 0 ? 0 : token) * p.heads + head) * D;
        // lane holds dimensions db * 32 + 8 g + 4 lh + j of its row; after the exchange with lane ^ 32, 8 of one g
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int g = 0; g < 4; g += 2) {
                half_t e[4], f[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) { e[j] = (half_t)(o[db][4 * g + j] * inv); f[j] = (half_t)(o[db][4 * g + 4 + j] * inv); }
                const uintx2 eu = *(const uintx2*)e, fu = *(const uintx2*)f;
                const auto x = __builtin_amdgcn_permlane32_swap(eu[0], fu[0], false, false);
                const auto y = __builtin_amdgcn_permlane32_swap(eu[1], fu[1], false, false);
                if (token >= 0) *(uintx4*)(out + db * 32 + 8 * (g + lh)) = uintx4{x[0], y[0], x[1], y[1]};
            }
    } else if (token >= 0) {
        const long long slot = (joined_token(a, b, s, i) * p.heads + head) * a.slots + part;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g) *(floatx4*)(a.o + slot * D + db * 32 + 8 * g + 4 * lh) = floatx4{o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]} * inv;
        if (lh == 0) *(float2*)(a.ml + slot * 2) = make_float2(m, l);
    }
}

// Joins the parts of rows that were shared out: a workgroup per (token, head), whose threads take 4 dimensions each and every few parts.  Latency bounds it: what the first parts' places
// hold is requested beside the sequence's lengths, which say how many parts there are.
template <int D>
__global__ void __launch_bounds__(256) paged_join_kernel(const PagedArgs few, const PagedArgs many) {
    constexpr int GROUP = D / 4, GROUPS = 256 / GROUP, AT_ONCE = 4;
    __shared__ floatx4 sums[GROUPS][GROUP];
    const PagedAttention& p = few.p;
    if (p.hp) __builtin_amdgcn_s_setprio(3);
    const int lane = threadIdx.x & 63, group = (int)threadIdx.x / GROUP, d = (int)threadIdx.x % GROUP, slots = few.slots;
    const long long row = blockIdx.x;                  // (joined_token's number times the heads, and the head)
    const float2* ml = (const float2*)few.ml + row * slots;
    const floatx4* o = (const floatx4*)(few.o + row * slots * D) + d;
    float2 mine = ml[lane < slots ? lane : 0];
    floatx4 part[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) part[k] = o[(long long)(group + k * GROUPS < slots ? group + k * GROUPS : 0) * GROUP];
    const int bi = divide((int)blockIdx.x, few.by_q_heads), hq = (int)blockIdx.x - bi * p.heads;
    int b, i;
    if (few.join_tokens) {                             // of each sequence the first few tokens
        b = divide(bi, few.by_join);
        i = bi - b * few.join_tokens;
    } else {                                           // each token
        int ended = 0;
        for (int s0 = 0; s0 < p.batch.seqs; s0 += 64) ended += __popcll(__ballot(s0 + lane < p.batch.seqs && p.batch.q_start[s0 + lane + 1] <= bi));
        b = ended;
        if (b >= p.batch.seqs) return;
        i = bi - p.batch.q_start[b];
        if (i < 0) return;
    }
    const Sequence s = sequence(p.batch, b);
    asm volatile("" : "+v"(mine.x), "+v"(mine.y), "+v"(part[0]), "+v"(part[1]), "+v"(part[2]), "+v"(part[3]));      // (requested above, whatever follows)
    if (i >= s.n) return;
    const PagedArgs& a = s.n * few.group <= few.to ? few : many;
    const int g = hq - divide(hq, a.by_group) * a.group;
    const Tile t = tile_of(a, s, (i * a.group + g) / a.rows);
    const Blocks blocks = visible_blocks(t.lo, t.hi, p.window, p.sinks);
    const int parts = (blocks.count + a.per_part - 1) / a.per_part;
    if (parts <= 1) return;
    if (lane >= parts) mine = make_float2(-INFINITY, 0.f);
    // (every wavefront finds the maximum and the sum for itself)
    float top = mine.x, sum;
    for (int x = lane + 64; x < parts; x += 64) top = fmaxf(top, ml[x].x);
#pragma unroll
    for (int k = 32; k; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
    auto weight = [&](float2 v) { return v.y == 0.f ? 0.f : v.y * __builtin_amdgcn_exp2f(v.x - top); };    // (NaN stays NaN)
    const float my_weight = weight(mine);
    sum = my_weight;
    for (int x = lane + 64; x < parts; x += 64) sum += weight(ml[x]);
#pragma unroll
    for (int k = 32; k; k >>= 1) sum += __shfl_xor(sum, k);
    floatx4 y = {0.f, 0.f, 0.f, 0.f};
    static_assert(AT_ONCE * GROUPS <= 64, "a lane for each of the first parts");
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
        const float w = __shfl(my_weight, group + k * GROUPS);
        if (group + k * GROUPS < parts) y += part[k] * w;
    }
    for (int x = group + AT_ONCE * GROUPS; x < parts; x += AT_ONCE * GROUPS) {
        float w[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int at = x + k * GROUPS;
            part[k] = o[(long long)(at < parts ? at : x) * GROUP];
            w[k] = at < parts ? weight(ml[at]) : 0.f;
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)
            if (x + k * GROUPS < parts) y += part[k] * w[k];
    }
    sums[group][d] = y;
    __syncthreads();
    if (group) return;
#pragma unroll
    for (int k = 1; k < GROUPS; ++k) y += sums[k][d];
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    half_t h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = (half_t)(y[j] * inv);
    *(uint2*)(p.out + ((long long)(s.first + i) * p.heads + hq) * D + d * 4) = *(const uint2*)h;
}

// How a call is launched.  Sequences with up to 16 or 32 rows of a kv head: the stream kernel, tiles of 16 or 32 rows, and two of these for 49 to 64 (64 rows: 64 sequences of 950 keys and 8 heads
// 46 us and on the tile kernel 58, 4 heads 28 and 41, 16 of 3100 and 8 heads 59 and 64, 128 of up to 1000 73 and 68; but of 40 rows 32 sequences of 1200 keys 56 and 47).  More: the tile kernel, 128 rows, of which a compute unit holds
// two, or three of 64 dimensions.  (256 rows by eight wavefronts fill LDS half as often, but all of them stand at one barrier: chunks of four prompts as fast, with a window a third slower.)  A step of
// both kinds gets both launches.  Parts of as many blocks as give each compute unit several workgroups (tile kernel: where it would not have one).
struct PagedPlan { PagedArgs few, many; size_t workspace; long long joins; };

static void plan_class(PagedArgs& a, bool stream) {
    const PagedAttention& p = a.p;
    const long long rows = std::min<long long>((long long)p.batch.max_q * a.group, a.to);
    a.tiles = (int)((rows + a.rows - 1) / a.rows);
    const long long direct = (long long)p.batch.seqs * a.tiles, counted = (long long)p.batch.tokens * a.group / a.rows + p.batch.seqs;
    a.items = direct > 2 * counted ? (int)counted : 0;
    const int most = most_blocks(p, a.rows);
    // Stream kernel: about 1024 parts (512 of 32 rows, whose results are more to join), but no more than 32 blocks each while there are 4096 or fewer of those: lengths differ, and
    // what is left to the longest parts at the end is read by few compute units (24 streams of 129 blocks and 4 heads, parts of 8, 16 and 28 blocks: 53.7, 47.5 and 47.0 us; 32 sequences of
    // 32 to 512 and 8 heads, parts of 16, 32, 64 and 128: 128, 122, 127 and 129; all of 256: 133, 115, 108 and 109).  Tile kernel: one part, or 512 where there are few tiles.
    const long long work = std::min(direct, counted) * p.cache.kv_heads * most;
    auto share = [&](long long n) { return ((work + n - 1) / n + PAGED_WAVES - 1) / PAGED_WAVES * PAGED_WAVES; };
    const long long per = stream ? std::max<long long>(8, std::min(share(a.rows == 16 ? 1024 : 512), std::max<long long>(32, share(4096)))) : std::max<long long>(16, share(512));
    a.per_part = (int)std::min<long long>(most, per);
    if (!stream && std::min(direct, counted) * p.cache.kv_heads >= 256) a.per_part = most;
    a.parts = (most + a.per_part - 1) / a.per_part;
    a.by_tiles = divisor(a.tiles);
    a.by_items = divisor(a.items);
}
static long long paged_grid(const PagedArgs& a) { return a.tiles ? (a.items ? a.items : (long long)a.p.batch.seqs * a.tiles) * a.p.cache.kv_heads * a.parts : 0; }

static PagedPlan paged_plan(const PagedAttention& p) {
    PagedPlan r{};
    PagedArgs& few = r.few;
    few.p = p;
    few.group = p.heads / p.cache.kv_heads;
    few.by_group = divisor(few.group); few.by_heads = divisor(p.cache.kv_heads); few.by_seqs = divisor(p.batch.seqs); few.by_q_heads = divisor(p.heads);
    r.many = few;
    const long long rows = (long long)p.batch.max_q * few.group;
    // (single tokens beside prompts' chunks are worth launches of their own where their caches may be long: taken to be there if the sequences but for the longest bring few tokens)
    const bool singles = p.batch.seqs > 1 && p.batch.tokens - p.batch.max_q <= 128LL * (p.batch.seqs - 1) && p.batch.max_kv > 512;
    few.to = rows <= 32 ? 32 : rows > 48 && rows <= 64 ? 64 : few.group > 32 || !singles ? 0 : few.group > 16 ? 32 : 16;
    few.rows = std::min<long long>(rows, few.to) <= 16 ? 16 : 32;
    r.many.from = few.to; r.many.to = 0x7fffffff; r.many.rows = 128;
    if (few.to) plan_class(few, true);
    if (rows > few.to) plan_class(r.many, false);
    few.slots = r.many.slots = std::max(few.parts, r.many.parts);
    if (few.slots > 1) {
        // the tokens to be joined: the first few of each sequence, or all where tiles were shared out too, or where they are fewer than half as many
        few.join_tokens = r.many.parts > 1 ? 0 : (int)std::min<long long>(p.batch.max_q, std::max(1, few.to / few.group));
        if ((long long)p.batch.seqs * few.join_tokens > 2LL * p.batch.tokens) few.join_tokens = 0;
        few.by_join = divisor(few.join_tokens);
        r.joins = (few.join_tokens ? (long long)p.batch.seqs * few.join_tokens : p.batch.tokens) * p.heads;
        const size_t slots = (size_t)r.joins * few.slots, head = (slots * 2 * sizeof(float) + 15) / 16 * 16;
        r.workspace = head + slots * p.cache.head_dim * sizeof(float);
        few.ml = r.many.ml = p.ws;
        few.o = r.many.o = (float*)((char*)p.ws + head);
    }
    return r;
}

size_t paged_attention_workspace(const PagedAttention& p) { return paged_plan(p).workspace; }

template <int D, bool I8>
static void launch_paged(const PagedPlan& r, unsigned few, unsigned many, unsigned joins, hipStream_t stream) {
    constexpr unsigned lds = 2 * 2 * TILE_KEYS * D * 2;
    static_assert(lds <= 64 * 1024, "what a kernel may have unasked");
    if (many) hipLaunchKernelGGL((paged_tile_kernel<D, I8>), dim3(many), dim3(64 * PAGED_WAVES), lds, stream, r.many);
    if (few) {
        auto kernel = r.few.rows == 16 ? paged_stream_kernel<D, I8, 1> : paged_stream_kernel<D, I8, 2>;
        hipLaunchKernelGGL(kernel, dim3(few), dim3(64 * PAGED_WAVES), 0, stream, r.few);
    }
    if (joins) hipLaunchKernelGGL(paged_join_kernel<D>, dim3(joins), dim3(256), 0, stream, r.few, r.many);
}

int launch_paged_attention(const PagedAttention& p, hipStream_t stream) {
    const PagedPlan r = paged_plan(p);
    const long long few = paged_grid(r.few), many = paged_grid(r.many), joins = r.joins;
    if (few > MOST_WORKGROUPS || many > MOST_WORKGROUPS || joins > MOST_WORKGROUPS) { set_error("attention_paged: grid too large"); return STRAIT_E_SHAPE; }
    const bool i8 = p.cache.type == STRAIT_KV_I8;
    if (p.cache.head_dim == 64) i8 ? launch_paged<64, true>(r, (unsigned)few, (unsigned)many, (unsigned)joins, stream) : launch_paged<64, false>(r, (unsigned)few, (unsigned)many, (unsigned)joins, stream);
    else i8 ? launch_paged<128, true>(r, (unsigned)few, (unsigned)many, (unsigned)joins, stream) : launch_paged<128, false>(r, (unsigned)few, (unsigned)many, (unsigned)joins, stream);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("attention_paged launch: %s", hipGetErrorString(e)); return -2; }
    return 0;
}

}  // namespace strait
