// Products in 8-bit integers with a scale for each token and each output channel, for gfx950.
//
//   y[m, n] = act( xs[m] ws[n] sum_k x[m, k] w[n, k] + bias[n] (+ res[m, n]) )
//
// The sum is an int32 of the integer MFMAs and exact in any order; the epilogue is fp32, rounded once.  Two kernels:
//
//   gemm_i8_stream_kernel, few rows: bound by the weights' bytes.  A workgroup of 8 wavefronts has 16 NT channels and shares the reduction
//   out in pieces of 256; weights go from memory to registers in the layout of v_mfma_i32_16x16x64_i8's operand, a piece ahead, and each byte is read
//   once on the whole chip.  The partial sums meet in LDS as integers.  1 x 4096 x 4096 6.2 us (2.7 TB/s), 16 x 16384 x 4096 13.0 us (5.2 TB/s).
//
//   gemm_i8_tile_kernel: bound by the matrix pipes.  Slices of 128 of the reduction travel to a ring in LDS without passing through registers, the operands of
//   the next MFMAs are read while the current ones run, and one barrier per slice hands a stage on.  8192 x 16384 x 4096 500 to 530 us, 2.1 POP/s, where the library's largest products
//   reach 2.15 and MFMAs on registers alone 2.3: the card's power.  An epilogue for each activation: one that asks at every output took 15 to 20 % of the whole kernel's time.
#include <type_traits>

#include "activation.hpp"
#include "conv_dma.hpp"
#include "decoder.hpp"

namespace strait {

typedef int intx16 __attribute__((ext_vector_type(16)));

typedef float floatx4 __attribute__((ext_vector_type(4)));
struct __attribute__((packed, aligned(2))) AnyHalf8 { half8 h; };      // at any address of an element
struct __attribute__((packed, aligned(4))) AnyFloat4 { floatx4 f; };

// One output of a sum: the same operations in the same order in every kernel, so that a row has the same bits whatever launch it is part of.
// (maximum and minimum: a NaN, which is how a row that was not finite arrives here, stays one in every activation.)
__device__ __forceinline__ float finish(int sum, float xs, float ws, float bias, float res, int act) {
    const float v = __builtin_fmaf((float)sum, xs * ws, bias) + res;
    if (act == ACT_RELU) return __builtin_elementwise_maximum(v, 0.f);
    if (act == ACT_RELU6) return __builtin_elementwise_minimum(__builtin_elementwise_maximum(v, 0.f), 6.f);
    return apply_act(v, act);
}

// ---- few rows -------------------------------------------------------------------------------------------------------

constexpr int STREAM_WAVES = 8;

template <int MT, int NT, int STREAM_STEPS>
__global__ void __launch_bounds__(64 * STREAM_WAVES) gemm_i8_stream_kernel(const GemmI8 p) {
    __shared__ int sums[16 * MT][16 * NT + 1];          // (+ 1: 16 rows at one channel lie in 16 banks)
    if (p.hp) __builtin_amdgcn_s_setprio(3);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l16 = lane & 15, g4 = lane >> 4;
    const int n0 = (int)blockIdx.x * 16 * NT;
    constexpr int PIECE = 64 * STREAM_STEPS;
    const int pieces = (p.K + PIECE - 1) / PIECE;
    const int8_t* wr[NT];
    const int8_t* xr[MT];
#pragma unroll
    for (int t = 0; t < NT; ++t) wr[t] = p.w + (long long)(n0 + 16 * t + l16 < p.N ? n0 + 16 * t + l16 : p.N - 1) * p.K;    // (rows past the end: the last one, not stored)
#pragma unroll
    for (int t = 0; t < MT; ++t) xr[t] = p.x + (long long)(16 * t + l16 < p.M ? 16 * t + l16 : p.M - 1) * p.K;
    auto at = [&](const int8_t* row, int piece, int s) __attribute__((always_inline)) {
        const int k = piece * PIECE + 64 * s + 16 * g4;
        return k < p.K ? *(const intx4*)(row + k) : intx4{0, 0, 0, 0};
    };
    intx4 acc[NT][MT] = {};
    intx4 w[NT][STREAM_STEPS], x[MT][STREAM_STEPS];
    auto load = [&](int piece) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int s = 0; s < STREAM_STEPS; ++s) w[t][s] = at(wr[t], piece, s);
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int s = 0; s < STREAM_STEPS; ++s) x[t][s] = at(xr[t], piece, s);
    };
    if (wave < pieces) load(wave);
    for (int i = threadIdx.x; i < 16 * MT * (16 * NT + 1); i += 64 * STREAM_WAVES) (&sums[0][0])[i] = 0;
    for (int piece = wave; piece < pieces; piece += STREAM_WAVES) {
        intx4 wc[NT][STREAM_STEPS], xc[MT][STREAM_STEPS];
#pragma unroll
        for (int s = 0; s < STREAM_STEPS; ++s) {
#pragma unroll
            for (int t = 0; t < NT; ++t) wc[t][s] = w[t][s];
#pragma unroll
            for (int t = 0; t < MT; ++t) xc[t][s] = x[t][s];
        }
        if (piece + STREAM_WAVES < pieces) load(piece + STREAM_WAVES);
#pragma unroll
        for (int s = 0; s < STREAM_STEPS; ++s)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int u = 0; u < MT; ++u) acc[t][u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wc[t][s], xc[u][s], acc[t][u], 0, 0, 0);
    }
    __syncthreads();
    // lane holds row l16 against channels 4 g4 .. + 3
    if (wave < pieces) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int u = 0; u < MT; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) atomicAdd(&sums[16 * u + l16][16 * t + 4 * g4 + v], acc[t][u][v]);     // (integers: the order is of no account)
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 256 * MT * NT; i += 64 * STREAM_WAVES) {
        const int m = i / (16 * NT), c = i - m * (16 * NT), n = n0 + c;
        if (m >= p.M || n >= p.N) continue;
        const long long o = (long long)m * p.N + n;
        const float y = finish(sums[m][c], p.xs[m], p.ws[n], p.bias ? p.bias[n] : 0.f, p.res ? (float)p.res[o] : 0.f, p.act);
        if (p.out_f32) ((float*)p.y)[o] = y;
        else ((half_t*)p.y)[o] = (half_t)y;
    }
}

// ---- tiles ------------------------------------------------------------------------------------------------------------

struct TileArgs { GemmI8 g; TileOrder order; };

constexpr int SLICE = 128;               // of the reduction, a whole cache line of each row
template <int BM, int BN, int STAGES, int G>
constexpr unsigned tile_lds() {
    const unsigned ring = G * STAGES * (BM + BN) * SLICE, out = BM * (BN + 8) * 2, parts = G > 1 ? BM * (BN + 4) * 4 : 0;
    return ring > out ? (ring > parts ? ring : parts) : (out > parts ? out : parts);
}
template <int BM, int BN, int STAGES, int G>
constexpr unsigned tile_lds_all() { return tile_lds<BM, BN, STAGES, G>() + BN * 8; }      // + the channels' scales and biases
template <int BM, int BN, int WAVES, int STAGES, int G>
constexpr int tile_waves_per_simd() {
    const int w = 160 * 1024 / (int)tile_lds_all<BM, BN, STAGES, G>() * WAVES * G / 4;
    return w < 1 ? 1 : w > 4 ? 4 : w;
}

// G > 1: so many sets of wavefronts, each with a ring of its own, take every G-th slice; their sums meet in LDS.
template <int BM, int BN, int WGM, int WGN, int STAGES, int G>
__global__ void __launch_bounds__(64 * WGM * WGN * G, (tile_waves_per_simd<BM, BN, WGM * WGN, STAGES, G>())) gemm_i8_tile_kernel(const TileArgs a) {
    const GemmI8& p = a.g;
    constexpr int NW = WGM * WGN, NT = 64 * NW * G;
    constexpr int TM = BM / WGM, TN = BN / WGN, TMB = TM / 32, TNB = TN / 32, KS = SLICE / 32;
    constexpr int XI = BM / (8 * NW), WI = BN / (8 * NW), NX = XI + WI, NM = TMB * TNB;      // transfers of 8 rows per wavefront and slice; MFMAs per step
    constexpr unsigned STAGE = (BM + BN) * SLICE;
    constexpr int LDC = BN + 8;
    static_assert(TM % 32 == 0 && TN % 32 == 0 && BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && NW % 2 == 0 && STAGES >= 2 && tile_lds_all<BM, BN, STAGES, G>() <= 160 * 1024, "tile");

    extern __shared__ __attribute__((aligned(1024))) char tile_smem[];
    if (p.hp) __builtin_amdgcn_s_setprio(3);
    const int tid = threadIdx.x, lane = tid & 63, nth = __builtin_amdgcn_readfirstlane(tid >> 6), set = G > 1 ? nth / NW : 0, wave = G > 1 ? nth % NW : nth, l32 = lane & 31, lh = lane >> 5;
    const char* const ring = tile_smem + set * (int)(STAGES * STAGE);
    const unsigned lds0 = (unsigned)(uintptr_t)ring;
    const int wm0 = (wave % WGM) * TM, wn0 = (wave / WGM) * TN;
    int tm, tn;
    place_tile(a.order, xcd_range(a.order.tiles, blockIdx.x), tm, tn);
    const int m0 = tm * BM, n0 = tn * BN;

    // the channels' scales and biases lie behind the ring (zeros past the end)
    float* const channels = (float*)(tile_smem + tile_lds<BM, BN, STAGES, G>());
    for (int i = tid; i < BN; i += NT) {
        channels[i] = n0 + i < p.N ? p.ws[n0 + i] : 0.f;
        channels[BN + i] = p.bias && n0 + i < p.N ? p.bias[n0 + i] : 0.f;
    }
    // a residual's part of the epilogue: LANES lanes lie along a row, 8 outputs each; on tiles of 32 rows to a wavefront all of it is requested ahead of the first slice
    constexpr int LANES = BN / 8, ROWS = WGM * 32 / (NT / LANES);      // rows of a lane among 32 of each wavefront
    const int c0 = tid % LANES * 8, n = n0 + c0, many = p.N - n;
    half8 res[ROWS];
    auto row_of = [&](int b, int i) __attribute__((always_inline)) {
        const int r = i * (NT / LANES) + tid / LANES;
        return m0 + r / 32 * TM + b * 32 + r % 32;
    };
    auto load_res = [&](int b) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int m = row_of(b, i);
#pragma unroll
            for (int j = 0; j < 8; ++j) res[i][j] = (half_t)0.f;
            if (!p.res || m >= p.M || many <= 0) continue;
            const half_t* from = p.res + (long long)m * p.N + n;
            if (many >= 8) res[i] = ((const AnyHalf8*)from)->h;
            else {                                     // (the last channels: seven loads under way at once, not one for each that there is in turn)
#pragma unroll
                for (int j = 0; j < 7; ++j) res[i][j] = from[j < many ? j : 0];
            }
        }
    };
    if (TMB == 1) load_res(0);
    // the tile's rows as buffers of their own: offsets stay below 256 * 131056 whatever the operands' size; rows and numbers past the end arrive as zeros
    const intx4 xrsrc = make_rsrc(p.x + (long long)m0 * p.K, (unsigned)(p.M - m0 < BM ? p.M - m0 : BM) * (unsigned)p.K);
    const intx4 wrsrc = make_rsrc(p.w + (long long)n0 * p.K, (unsigned)(p.N - n0 < BN ? p.N - n0 : BN) * (unsigned)p.K);
    // lane i brings 16 bytes of row i / 8; LDS holds chunk c of a row r at c ^ (r / 2 % 8), so that 16 rows read at one chunk meet no bank twice
    const int rsub = lane >> 3, cl = (lane & 7) ^ (((wave * 8 + rsub) >> 1) & 7);
    unsigned xoff[XI], woff[WI];
#pragma unroll
    for (int j = 0; j < XI; ++j) xoff[j] = m0 + (j * NW + wave) * 8 + rsub < p.M ? (unsigned)((j * NW + wave) * 8 + rsub) * (unsigned)p.K + cl * 16 : OOB_OFFSET;
#pragma unroll
    for (int j = 0; j < WI; ++j) woff[j] = n0 + (j * NW + wave) * 8 + rsub < p.N ? (unsigned)((j * NW + wave) * 8 + rsub) * (unsigned)p.K + cl * 16 : OOB_OFFSET;
    const int nk = (p.K + G * SLICE - 1) / (G * SLICE);
    auto issue_one = [&](int stage, int nth_slice, int j) __attribute__((always_inline)) {
        const int slice = nth_slice * G + set;
        const bool there = slice * SLICE + cl * 16 < p.K;          // (the last slice may be ragged)
        const unsigned at = lds0 + (unsigned)stage * STAGE;
        if (j < XI) dma16(xrsrc, there ? xoff[j] : OOB_OFFSET, (unsigned)(slice * SLICE), at + (unsigned)((j * NW + wave) * 1024));
        else dma16(wrsrc, there ? woff[j - XI] : OOB_OFFSET, (unsigned)(slice * SLICE), at + BM * SLICE + (unsigned)(((j - XI) * NW + wave) * 1024));
    };
    intx16 acc[TNB][TMB] = {};
    intx4 wf[2][TNB], xf[2][TMB];
    auto load_frags = [&](int buf, int stage, int ks) __attribute__((always_inline)) {
        const char* xs = ring + stage * (int)STAGE;
        const char* ws = xs + BM * SLICE;
        const int pos = ((ks * 2 + lh) ^ ((l32 >> 1) & 7)) * 16;
#pragma unroll
        for (int i = 0; i < TNB; ++i) wf[buf][i] = *(const intx4*)(ws + (wn0 + i * 32 + l32) * SLICE + pos);
#pragma unroll
        for (int i = 0; i < TMB; ++i) xf[buf][i] = *(const intx4*)(xs + (wm0 + i * 32 + l32) * SLICE + pos);
    };
    // STAGES slices under way; slices past the end are requested as zeros, so that every wait counts the same
#pragma unroll
    for (int s = 0; s < STAGES; ++s)
#pragma unroll
        for (int j = 0; j < NX; ++j) issue_one(s, s, j);
    wait_loads_then_barrier<(STAGES - 1) * NX>();
    load_frags(0, 0, 0);
    int rd = 0;
    for (int kt = 0; kt < nk; ++kt) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int left = rd;
            if (ks + 1 < KS) load_frags((ks + 1) & 1, rd, ks + 1);
            else {
                wait_loads_then_barrier<(STAGES - 2) * NX>();      // slice kt + 1 is there, and everyone has read slice kt
                rd = rd + 1 == STAGES ? 0 : rd + 1;
                load_frags(0, rd, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int q = 0; q < NM; ++q) {
                acc[q / TMB][q % TMB] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[ks & 1][q / TMB], xf[ks & 1][q % TMB], acc[q / TMB][q % TMB], 0, 0, 0);
                if (ks == KS - 1) {
                    constexpr int PER = (NX + NM - 1) / NM;
#pragma unroll
                    for (int j = q * PER; j < (q + 1) * PER && j < NX; ++j) issue_one(left, kt + STAGES, j);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");   // the zeros past the end have arrived: LDS is free

    if (G > 1) {                                       // the sets' sums become the first one's
        int* const parts = (int*)tile_smem;
        auto each = [&](auto body) __attribute__((always_inline)) {
#pragma unroll
            for (int b = 0; b < TMB; ++b)
#pragma unroll
                for (int t = 0; t < TNB; ++t)
#pragma unroll
                    for (int g = 0; g < 4; ++g) body(acc[t][b], 4 * g, (intx4*)(parts + (wm0 + b * 32 + l32) * (BN + 4) + wn0 + t * 32 + 8 * g + 4 * lh));
        };
#pragma unroll
        for (int other = 1; other < G; ++other) {
            if (set == other) each([](intx16& sum, int v, intx4* at) __attribute__((always_inline)) { *at = intx4{sum[v], sum[v + 1], sum[v + 2], sum[v + 3]}; });
            __syncthreads();
            if (set == 0)
                each([](intx16& sum, int v, intx4* at) __attribute__((always_inline)) {
                    const intx4 y = *at;
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum[v + j] += y[j];
                });
            __syncthreads();
        }
    }

    // ---- epilogue, one for each activation: a lane holds the sums of y[m][n .. n + 3], n at 8 g + 4 lh.  Rows of the result begin at any multiple of its element (N may be odd): 16 bytes at a time
    // all the same, which the memory takes at any address.
    auto epilogue = [&](auto activation) __attribute__((always_inline)) {
    constexpr int ACT = decltype(activation)::value;
    if (!p.out_f32 && !p.res) {
        // rounded results leave through LDS
        half_t* const out = (half_t*)tile_smem;
        if (set == 0)
#pragma unroll
        for (int b = 0; b < TMB; ++b) {
            const int mt = wm0 + b * 32 + l32;
            const float xs = m0 + mt < p.M ? p.xs[m0 + mt] : 0.f;
#pragma unroll
            for (int t = 0; t < TNB; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int nt = wn0 + t * 32 + 8 * g + 4 * lh;
                    const floatx4 ws = *(const floatx4*)(channels + nt), bias = *(const floatx4*)(channels + BN + nt);
                    half4 h;
#pragma unroll
                    for (int j = 0; j < 4; ++j) h[j] = (half_t)finish(acc[t][b][4 * g + j], xs, ws[j], bias[j], 0.f, ACT);
                    *(half4*)(out + mt * LDC + nt) = h;
                }
        }
        __syncthreads();
        for (int i = tid; i < BM * (BN / 8); i += NT) {
            const int r = i / (BN / 8), c = (i - r * (BN / 8)) * 8, m = m0 + r, n = n0 + c;
            if (m >= p.M || n >= p.N) continue;
            half_t* y = (half_t*)p.y + (long long)m * p.N + n;
            const half8 h = *(const half8*)(out + r * LDC + c);
            if (n + 8 <= p.N) *(AnyHalf8*)y = AnyHalf8{h};
            else
#pragma unroll 1
                for (int j = 0; j < p.N - n; ++j) y[j] = out[r * LDC + c + j];
        }
        return;
    }
    // with a residual, or in fp32: the sums go through LDS, 32 rows of each wavefront at a time, and are finished by lanes that lie along a row, 8 outputs each
    int* const sums = (int*)tile_smem;
    constexpr int LDS_N = BN + 4;
    static_assert(WGM * 32 * LDS_N * 4 <= (int)tile_lds<BM, BN, STAGES, G>() && WGM * 32 % (NT / LANES) == 0, "staging");
#pragma unroll
    for (int b = 0; b < TMB; ++b) {
        __builtin_amdgcn_sched_barrier(0);             // (nothing of the next 32 rows ahead of these: there are no registers for it)
        float xs[ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) xs[i] = row_of(b, i) < p.M ? p.xs[row_of(b, i)] : 0.f;
        if (TMB > 1) load_res(b);                      // (on its way while the sums are)
        if (b) __syncthreads();
        if (set == 0)
#pragma unroll
        for (int t = 0; t < TNB; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(intx4*)(sums + ((wave % WGM) * 32 + l32) * LDS_N + wn0 + t * 32 + 8 * g + 4 * lh) = intx4{acc[t][b][4 * g], acc[t][b][4 * g + 1], acc[t][b][4 * g + 2], acc[t][b][4 * g + 3]};
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int* from = sums + (i * (NT / LANES) + tid / LANES) * LDS_N + c0;
            const intx4 lo = *(const intx4*)from, hi = *(const intx4*)(from + 4);
            const int m = row_of(b, i);
            if (m >= p.M || many <= 0) continue;
            const long long at = (long long)m * p.N + n;
            floatx4 y[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const floatx4 ws = *(const floatx4*)(channels + c0 + 4 * k), bias = *(const floatx4*)(channels + BN + c0 + 4 * k);
#pragma unroll
                for (int j = 0; j < 4; ++j) y[k][j] = finish((k ? hi : lo)[j], xs[i], ws[j], bias[j], (float)res[i][4 * k + j], ACT);
            }
            if (many < 8) {
#pragma unroll
                for (int j = 0; j < 7; ++j) {
                    if (j >= many) continue;
                    if (p.out_f32) ((float*)p.y)[at + j] = y[j >> 2][j & 3];
                    else ((half_t*)p.y)[at + j] = (half_t)y[j >> 2][j & 3];
                }
            } else if (p.out_f32) {
                *(AnyFloat4*)((float*)p.y + at) = AnyFloat4{y[0]};
                *(AnyFloat4*)((float*)p.y + at + 4) = AnyFloat4{y[1]};
            } else {
                half8 h;
#pragma unroll
                for (int j = 0; j < 8; ++j) h[j] = (half_t)y[j >> 2][j & 3];
                *(AnyHalf8*)((half_t*)p.y + at) = AnyHalf8{h};
            }
        }
    }
    };
    if (p.act == ACT_GELU) epilogue(std::integral_constant<int, ACT_GELU>{});
    else if (p.act == ACT_RELU) epilogue(std::integral_constant<int, ACT_RELU>{});
    else if (p.act == ACT_RELU6) epilogue(std::integral_constant<int, ACT_RELU6>{});
    else epilogue(std::integral_constant<int, ACT_NONE>{});
}

template <int BM, int BN, int WGM, int WGN, int STAGES, int G = 1>
static int launch_tile(const GemmI8& p, hipStream_t stream) {
    const long long tiles_m = (p.M + BM - 1LL) / BM, tiles_n = (p.N + BN - 1LL) / BN;
    if (tiles_m * tiles_n * (WGM * WGN * G / 4) > MOST_WORKGROUPS) { set_error("gemm_i8: grid too large"); return STRAIT_E_SHAPE; }
    ConvParams order{};
    set_tile_order(order, tiles_m, (int)tiles_n, BM, BN, SLICE, 1);
    const TileArgs a{p, order.order};
    constexpr unsigned lds = tile_lds_all<BM, BN, STAGES, G>();
    auto kernel = gemm_i8_tile_kernel<BM, BN, WGM, WGN, STAGES, G>;
    if (lds > 64 * 1024) {                             // asked for once per tile and device (twice is harmless; devices beyond the 64th each time)
        static std::atomic<unsigned long long> asked{0};
        int device = 0;
        hipError_t e = hipGetDevice(&device);
        const unsigned long long bit = device < 64 ? 1ULL << device : 0;
        if (e == hipSuccess && !(asked.load(std::memory_order_acquire) & bit)) {
            e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            if (e == hipSuccess) asked.fetch_or(bit, std::memory_order_release);
        }
        if (e != hipSuccess) { set_error("gemm_i8: cannot reserve %u bytes of LDS: %s", lds, hipGetErrorString(e)); return STRAIT_E_HIP; }
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)(tiles_m * tiles_n)), dim3(64 * WGM * WGN * G), lds, stream, a);
    return 0;
}
template <int MT, int NT, int STEPS>
static int launch_stream(const GemmI8& p, hipStream_t stream) {
    const long long groups = (p.N + 16LL * NT - 1) / (16 * NT);
    if (groups * (STREAM_WAVES / 4) > MOST_WORKGROUPS) { set_error("gemm_i8: grid too large"); return STRAIT_E_SHAPE; }
    hipLaunchKernelGGL((gemm_i8_stream_kernel<MT, NT, STEPS>), dim3((unsigned)groups), dim3(64 * STREAM_WAVES), 0, stream, p);
    return 0;
}

// Up to 16 rows, and up to 48 where 16 channels to a workgroup are one round of workgroups: the stream, 16 NT channels to a workgroup, NT so that there are 256 workgroups where the channels
// allow it (16384 x 4096 at 16 rows, NT = 4: 13.0 us; a tile 13.5; 4096 x 4096 7.0 and 10.7), pieces of 128 or 256 as the registers allow.  Every workgroup of it reads all of x, so the
// tile's 64 channels win from there on: 17 x 12288 x 4096 16.3 and 11.3 us, 32 x 16384 x 4096 15.4 and 13.6, 48 x 4096 x 4096 11.8 and 10.9, 64 x 4096 x 16384 38.6 and 29.8; for the stream still
// 32 x 4096 x 4096 8.9 and 10.8, 33 x 4096 x 2048 6.0 and 7.0, 33 x 2304 x 1024 4.4 and 5.3.
// More: the tile with the least time for the most tiles that a compute unit gets.  A slice of 128 takes a unit 0.24 us on a 64 x 64 tile, 0.66 on 128 x 128, 1.11 on 256 x 128
// and 2.05 on 256 x 256 with all units at work (256 x 4096 x 4096 12.0, 17.9, 27.0 and 45.1 us; 512 x 5120 x 2048 16.5, 12.8, 17.9 and 28.0; 2048 x 4096 x 4096 62.7, 45.7, 38.3 and 49.6;
// 4096 x 4096 x 4096 119, 88.2, 75.6 and 68.2; 8192 x 16384 x 4096 1191, 777, 615 and 529).
// Where one round of small tiles is all there is, a unit's one tile waits for its own transfers and barriers: two sets of wavefronts share out its slices if there are enough of these (64 x 64:
// 128 x 4096 x 4096 11.2 and 10.1 us, 64 x 4096 x 16384 29.2 and 24.2, 300 x 1024 x 8192 17.5 and 15.0, but 48 x 2304 x 768 4.9 and 5.0, and with two rounds 512 x 4096 x 4096 18.8 and
// 19.8; 128 x 64 with two sets, 64 x 64 and 128 x 128 without: 512 x 4096 x 4096 16.9, 18.8 and 20.3, 300 x 5120 x 4096 14.8, 16.0 and 18.1, 400 x 4096 x 8192 25.6, 27.8 and 31.1).
int launch_gemm_i8(const GemmI8& p, hipStream_t stream) {
    int rc = 0;
    if (p.M <= 16) {
        rc = p.N >= 16384 ? launch_stream<1, 4, 2>(p, stream) : p.N >= 8192 ? launch_stream<1, 2, 4>(p, stream) : launch_stream<1, 1, 4>(p, stream);
    } else if (p.M <= 32 && p.N <= 4096) {
        rc = launch_stream<2, 1, 4>(p, stream);
    } else if (p.M <= 48 && p.N <= 4096 && p.K <= 2048) {
        rc = launch_stream<3, 1, 4>(p, stream);
    } else {
        const struct { int bm, bn; float us; bool two; } tile[6] = {{64, 64, 0.24f, false}, {128, 128, 0.66f, false}, {256, 128, 1.11f, false}, {256, 256, 2.05f, false}, {64, 64, 0.21f, true}, {128, 64, 0.36f, true}};
        int best = 0;
        float least = 0.f;
        for (int i = 0; i < 6; ++i) {
            const long long tiles = (p.M + tile[i].bm - 1LL) / tile[i].bm * ((p.N + tile[i].bn - 1LL) / tile[i].bn);
            if (tile[i].two && (tiles > 256 || p.K <= 2048)) continue;
            const float us = (float)((tiles + 255) / 256) * tile[i].us;
            if (!i || us < least) { best = i; least = us; }
        }
        rc = best == 0 ? launch_tile<64, 64, 2, 2, 4>(p, stream) : best == 1 ? launch_tile<128, 128, 4, 2, 4>(p, stream) : best == 2 ? launch_tile<256, 128, 4, 2, 3>(p, stream)
             : best == 3 ? launch_tile<256, 256, 2, 4, 2>(p, stream) : best == 4 ? launch_tile<64, 64, 2, 2, 4, 2>(p, stream) : launch_tile<128, 64, 4, 2, 3, 2>(p, stream);
    }
    if (rc) return rc;
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error("gemm_i8 launch: %s", hipGetErrorString(e)); return -2; }
    return 0;
}

}  // namespace strait
