// Launchers of a decoder's operators (quantize.hip, gemm_i8.hip, kv_append.hip, paged_attention.hip), called by decoder.cpp with checked arguments.
#pragma once
#include "../../include/strait.h"
#include "kernels.hpp"

namespace strait {

int launch_quantize_rows(const half_t* x, int M, int K, long long pitch, int8_t* q, float* scale, int hp, hipStream_t stream);

constexpr long long MOST_WORKGROUPS = 0xffffff;        // of 256 threads: a launch has less than 2^32 of these

struct GemmI8 {
    const int8_t* x; const float* xs;
    const int8_t* w; const float* ws;
    const float* bias;       // [N] or nullptr
    const half_t* res;       // [M][N] or nullptr
    void* y;                 // fp16, or fp32 where out_f32, [M][N]
    int M, N, K, act, out_f32, hp;
};
int launch_gemm_i8(const GemmI8& p, hipStream_t stream);

// A sequence's new tokens and lengths as the kernels take them: everything that was read from device memory is held inside what the launch was made for.
struct Sequence {
    int first;               // row of its first new token
    int n;                   // new tokens that are worked on, at most max_q
    int past;                // position of the first one; negative where kv_len is smaller than the number of new tokens
    int total;               // tokens in the cache
};
#ifdef __HIPCC__
__device__ __forceinline__ Sequence sequence(const strait_kv_batch& b, int s) {
    auto inside = [](int v, int hi) { return v < 0 ? 0 : v > hi ? hi : v; };
    const int q0 = inside(b.q_start[s], b.tokens), q1 = inside(b.q_start[s + 1], b.tokens);
    const int all = q1 > q0 ? q1 - q0 : 0, total = inside(b.kv_len[s], b.max_kv);
    return {q0, all < b.max_q ? all : b.max_q, total - all, total};
}
#endif

struct KvAppend {
    strait_kv_cache cache; strait_kv_batch batch;
    const half_t* q; const half_t* k; const half_t* v;
    long long pitch_q, pitch_k, pitch_v;
    int heads;               // of q; 0: none
    const float* rope; int rope_dim, interleaved;
    half_t* q_out;
    int hp;
};
int launch_kv_append(const KvAppend& p, hipStream_t stream);

struct PagedAttention {
    strait_kv_cache cache; strait_kv_batch batch;
    const half_t* q; long long pitch_q;
    int heads;
    float scale;
    int window, sinks;
    half_t* out;
    float* ws;
    int hp;
};
size_t paged_attention_workspace(const PagedAttention& p);         // bytes
int launch_paged_attention(const PagedAttention& p, hipStream_t stream);

}  // namespace strait
