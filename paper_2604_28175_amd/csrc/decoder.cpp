// The C entry points of a decoder's operators: what the host arguments say is checked here, before anything is launched.
#include <math.h>

#include "decoder.hpp"

using namespace strait;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int invalid(const char* what, const char* why) { set_error("%s: %s", what, why); return STRAIT_E_INVALID; }
int shape(const char* what, const char* why) { set_error("%s: %s", what, why); return STRAIT_E_SHAPE; }

int check_cache(const char* what, const strait_kv_cache* c) {
    if (!c) return invalid(what, "null cache");
    if (c->type != STRAIT_KV_F16 && c->type != STRAIT_KV_I8) return invalid(what, "unknown cache type");
    if (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return invalid(what, "k and v of the cache must be 16-byte aligned device memory");
    if (c->type == STRAIT_KV_I8 && (!c->k_scale || !c->v_scale)) return invalid(what, "an int8 cache needs its scales");
    if (c->pages < 1 || c->kv_heads < 1) return invalid(what, "the cache needs pages and heads");
    if (c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128 && c->page_tokens != 256) return shape(what, "pages hold 32, 64, 128 or 256 tokens");
    if (c->head_dim != 64 && c->head_dim != 128) return shape(what, "head dimensions are 64 or 128");
    if ((long long)c->pages * c->kv_heads > 0x7fffffffLL) return shape(what, "too many pages");
    return STRAIT_OK;
}
// E_BATCH stands for a step of no tokens, which is no error: the caller returns OK
int check_batch(const char* what, const strait_kv_cache* c, const strait_kv_batch* b) {
    if (!b) return invalid(what, "null batch");
    if (b->tokens < 0 || b->seqs < 0) return invalid(what, "negative sizes");
    if (b->tokens == 0 || b->seqs == 0) return STRAIT_E_BATCH;
    if (!b->q_start || !b->kv_len || !b->page_table) return invalid(what, "null q_start, kv_len or page_table");
    if (b->max_q < 1 || b->max_q > b->tokens || b->max_kv < 1) return invalid(what, "needs 1 <= max_q <= tokens and max_kv >= 1");
    if (b->table_pitch < (b->max_kv + (long long)c->page_tokens - 1) / c->page_tokens) return invalid(what, "table_pitch is too small for max_kv");
    if (b->max_kv > 1 << 29) return shape(what, "max_kv is 2^29 at most");
    return STRAIT_OK;
}
int check_rows(const char* what, const void* p, int64_t pitch, long long width, const char* why) {
    return !p || !aligned16(p) || pitch < width || pitch % 8 ? invalid(what, why) : STRAIT_OK;
}
// rows of `heads` heads: what the kernels hold in 32 bits
int check_heads(const char* what, const strait_kv_cache* c, const strait_kv_batch* b, long long heads) {
    if (heads < 1) return invalid(what, "needs heads");
    if (heads % c->kv_heads) return invalid(what, "heads must be a multiple of the cache's kv_heads");
    if (heads > 65536 || (heads + 2LL * c->kv_heads) * b->tokens > 0x7fffffffLL / 16 || (long long)b->max_q * heads > 0x3fffffffLL) return shape(what, "too many heads or tokens");
    return STRAIT_OK;
}

int paged_arguments(const char* what, const strait_kv_cache* cache, const strait_kv_batch* batch, int32_t heads, int32_t window, int32_t sinks, PagedAttention& p) {
    if (int rc = check_cache(what, cache)) return rc;
    if (int rc = check_batch(what, cache, batch)) return rc;
    if (int rc = check_heads(what, cache, batch, heads)) return rc;
    if (window < 0 || sinks < 0) return invalid(what, "window and sinks are not negative");
    // (each has a workgroup at least; with fewer of them no product of sizes in the plan leaves its type)
    if ((long long)batch->seqs * cache->kv_heads > MOST_WORKGROUPS) return shape(what, "grid too large");
    p.cache = *cache;
    p.batch = *batch;
    p.heads = heads;
    // (a window that holds every key is none; sums of positions and these stay in 32 bits)
    p.window = window >= batch->max_kv ? 0 : window;
    p.sinks = p.window ? (sinks < batch->max_kv ? sinks : batch->max_kv) : 0;
    return STRAIT_OK;
}

}  // namespace

extern "C" {

strait_status strait_k_quantize_rows(void* stream, const void* x, int32_t M, int32_t K, int64_t pitch, int8_t* q, float* scale, int32_t hp) {
    const char* what = "quantize_rows";
    if (M < 0 || K < 1) return invalid(what, "needs M >= 0 and K >= 1");
    if (K % 16) return shape(what, "K must be a multiple of 16");
    if (M == 0) return STRAIT_OK;
    if (int rc = check_rows(what, x, pitch, K, "x must be 16-byte aligned, its pitch a multiple of 8 and at least K")) return rc;
    if (!q || !scale || !aligned16(q) || reinterpret_cast<uintptr_t>(scale) % 4) return invalid(what, "null or misaligned q or scale");
    return launch_quantize_rows((const half_t*)x, M, K, pitch, q, scale, hp, (hipStream_t)stream);
}

strait_status strait_k_gemm_i8(void* stream, const int8_t* x, const float* x_scale, const int8_t* w, const float* w_scale, const float* bias,
                               int32_t M, int32_t N, int32_t K, int32_t act, const void* res, void* y, int32_t out_f32, int32_t hp) {
    const char* what = "gemm_i8";
    if (M < 0 || N < 1 || K < 1) return invalid(what, "needs M >= 0, N >= 1 and K >= 1");
    if (K % 16 || K > 131056) return shape(what, "K must be a multiple of 16 up to 131056");
    if (act < STRAIT_ACT_NONE || act > STRAIT_ACT_GELU) return invalid(what, "unknown activation");
    if (M == 0) return STRAIT_OK;
    if (res && out_f32 && res == y) return invalid(what, "y may be res only where both are fp16");
    if (!x || !x_scale || !w || !w_scale || !y || !aligned16(x) || !aligned16(w)) return invalid(what, "null or misaligned operands");
    if (reinterpret_cast<uintptr_t>(y) % (out_f32 ? 4 : 2) || reinterpret_cast<uintptr_t>(res) % 2 || reinterpret_cast<uintptr_t>(x_scale) % 4 ||
        reinterpret_cast<uintptr_t>(w_scale) % 4 || reinterpret_cast<uintptr_t>(bias) % 4) return invalid(what, "misaligned operands");
    GemmI8 p{x, x_scale, w, w_scale, bias, (const half_t*)res, y, M, N, K, act, out_f32, hp};
    return launch_gemm_i8(p, (hipStream_t)stream);
}

strait_status strait_rope_table(float* table, int32_t positions, int32_t dim, double base) {
    const char* what = "rope_table";
    if (positions < 0 || dim < 2 || dim % 2 || !(base > 0) || !isfinite(base)) return invalid(what, "needs positions >= 0, an even dim and a positive base");
    if (positions && !table) return invalid(what, "null table");
    const int half = dim / 2;
    for (int j = 0; j < half; ++j) {
        const double turn = pow(base, -2.0 * j / dim);
        for (int p = 0; p < positions; ++p) {
            table[(size_t)p * dim + j] = (float)cos(p * turn);
            table[(size_t)p * dim + half + j] = (float)sin(p * turn);
        }
    }
    return STRAIT_OK;
}

strait_status strait_k_kv_append(void* stream, const strait_kv_cache* cache, const strait_kv_batch* batch, const void* q, const void* k, const void* v,
                                 int64_t pitch_q, int64_t pitch_k, int64_t pitch_v, int32_t heads, const float* rope, int32_t rope_rows, int32_t rope_dim,
                                 int32_t interleaved, void* q_out, int32_t hp) {
    const char* what = "kv_append";
    if (int rc = check_cache(what, cache)) return rc;
    if (int rc = check_batch(what, cache, batch)) return rc == STRAIT_E_BATCH ? STRAIT_OK : rc;
    if (!q != !q_out) return invalid(what, "q and q_out come together");
    if (int rc = check_heads(what, cache, batch, q ? heads : cache->kv_heads)) return rc;
    const long long d = cache->head_dim, kv = cache->kv_heads * d;
    if (int rc = check_rows(what, k, pitch_k, kv, "k must be 16-byte aligned, its pitch a multiple of 8 and at least kv_heads * head_dim")) return rc;
    if (int rc = check_rows(what, v, pitch_v, kv, "v must be 16-byte aligned, its pitch a multiple of 8 and at least kv_heads * head_dim")) return rc;
    if (q) {
        if (int rc = check_rows(what, q, pitch_q, heads * d, "q must be 16-byte aligned, its pitch a multiple of 8 and at least heads * head_dim")) return rc;
        if (!aligned16(q_out)) return invalid(what, "q_out must be 16-byte aligned");
        if (q == q_out && pitch_q != heads * d) return invalid(what, "q_out may be q only where the rows of q lie end to end");
    }
    if (rope) {
        if (rope_dim < 16 || rope_dim % 16 || rope_dim > d) return shape(what, "rope_dim must be a multiple of 16 up to head_dim");
        if (rope_rows < batch->max_kv) return invalid(what, "the rotation table is shorter than max_kv");
        if (!aligned16(rope)) return invalid(what, "the rotation table must be 16-byte aligned");
    } else if (rope_dim) return invalid(what, "rope_dim without a rotation table");
    KvAppend p{*cache, *batch, (const half_t*)q, (const half_t*)k, (const half_t*)v, pitch_q, pitch_k, pitch_v, q ? heads : 0, rope, rope_dim, interleaved, (half_t*)q_out, hp};
    return launch_kv_append(p, (hipStream_t)stream);
}

strait_status strait_k_attention_paged_workspace(const strait_kv_cache* cache, const strait_kv_batch* batch, int32_t heads, int32_t window, int32_t sinks, size_t* bytes) {
    const char* what = "attention_paged_workspace";
    if (!bytes) return invalid(what, "null output");
    *bytes = 0;
    PagedAttention p{};
    if (int rc = paged_arguments(what, cache, batch, heads, window, sinks, p)) return rc == STRAIT_E_BATCH ? STRAIT_OK : rc;
    *bytes = paged_attention_workspace(p);
    return STRAIT_OK;
}

strait_status strait_k_attention_paged(void* stream, const strait_kv_cache* cache, const strait_kv_batch* batch, const void* q, int64_t pitch_q, int32_t heads,
                                       float scale, int32_t window, int32_t sinks, void* out, void* workspace, size_t workspace_bytes, int32_t hp) {
    const char* what = "attention_paged";
    PagedAttention p{};
    if (int rc = paged_arguments(what, cache, batch, heads, window, sinks, p)) return rc == STRAIT_E_BATCH ? STRAIT_OK : rc;
    if (int rc = check_rows(what, q, pitch_q, (long long)heads * cache->head_dim, "q must be 16-byte aligned, its pitch a multiple of 8 and at least heads * head_dim")) return rc;
    if (!out || !aligned16(out)) return invalid(what, "out must be 16-byte aligned device memory");
    if (!(scale > 0.f) || !isfinite(scale)) return invalid(what, "scale must be finite and positive");
    const size_t need = paged_attention_workspace(p);
    if (need && (!workspace || workspace_bytes < need)) { set_error("%s: needs a workspace of %zu bytes, got %zu", what, need, workspace ? workspace_bytes : (size_t)0); return STRAIT_E_NOMEM; }
    if (need && !aligned16(workspace)) return invalid(what, "the workspace must be 16-byte aligned");
    p.q = (const half_t*)q;
    p.pitch_q = pitch_q;
    p.scale = scale;
    p.out = (half_t*)out;
    p.ws = (float*)workspace;
    p.hp = hp;
    return launch_paged_attention(p, (hipStream_t)stream);
}

}  // extern "C"
