// C ABI of the bounded cache (sparsp_bounded.h) but for the window over a cache of rows, which is
// attention like the other (api_cache.cpp): argument checks and dispatch, plain host C++.
#include "../../include/sparsp_bounded.h"
#include "api_checks.h"

namespace {

// No token is further from another than this: longer windows and more sinks are the same.
constexpr int kFarthest = 1 << 30;

// The cache as the kernels take it: codes in place of K and V, rows of `dtype`.
int check_cache4(const sparsp_cache4* c, int dtype, sparsp_cache* out) {
    if (!c) return fail(SPARSP_E_INVALID, "cache is NULL");
    if (dtype != SPARSP_F32 && dtype != SPARSP_BF16)
        return fail(SPARSP_E_DTYPE, "unknown dtype %d", dtype);
    if (c->d <= 0) return fail(SPARSP_E_INVALID, "d = %d must be positive", c->d);
    if (c->d % 32 || c->d > 128)
        return fail(SPARSP_E_UNSUPPORTED, "d = %d must be a multiple of 32 up to 128", c->d);
    *out = {c->K,     c->V,  nullptr, c->table, c->new_off, c->kv_len, c->pages,
            c->H,     c->page, c->d,  dtype,    c->width,   c->B,      0};
    return check_cache(out);
}

int check_pointers4(const sparsp_cache4* c) {
    if (!c->K || !c->V || !c->K_scales || !c->V_scales || !c->table || !c->new_off || !c->kv_len)
        return fail(SPARSP_E_INVALID, "NULL cache pointer");
    if (!aligned16(c->K) || !aligned16(c->V) || !aligned16(c->K_scales) || !aligned16(c->V_scales))
        return fail(SPARSP_E_INVALID, "codes and scales must be 16-byte aligned");
    return SPARSP_OK;
}

int check_apart4(const sparsp_cache4* c) {
    const void* at[4] = {c->K, c->V, c->K_scales, c->V_scales};
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < i; ++j)
            if (at[i] == at[j])
                return fail(SPARSP_E_INVALID, "codes and scales of K and V are the same memory");
    return SPARSP_OK;
}

// K and V of a call, as moves 0 and 1.
int check_new_rows(const sparsp_cache& c, int tokens, const sparsp_rows* K, const sparsp_rows* V,
                   bool written, sparsp::RotateArgs* a) {
    if (int rc = check_tokens(tokens)) return rc;
    const int size = c.dtype == SPARSP_BF16 ? 2 : 4;
    if (int rc = check_rows(K, "K", tokens, c.d, size, written)) return rc;
    if (int rc = check_rows(V, "V", tokens, c.d, size, written)) return rc;
    if (K->heads != c.H || V->heads != c.H)
        return fail(SPARSP_E_INVALID, "K and V have %d and %d heads, the cache has %d", K->heads,
                    V->heads, c.H);
    a->move[0] = row_move(*K, *K, false);
    a->move[1] = row_move(*V, *V, false);
    a->moves = 2;
    a->tokens = tokens;
    a->d = c.d;
    a->bf16 = c.dtype == SPARSP_BF16;
    a->cache = c;
    return SPARSP_OK;
}

int check_attn4(const sparsp_cache4* cache, int tokens, int dtype, const sparsp_rows* Q, int window,
                int sinks, float scale, int max_new, int max_kv, sparsp::PagedArgs* a) {
    sparsp_cache c;
    if (int rc = check_cache4(cache, dtype, &c)) return rc;
    if (int rc = check_query(&c, tokens, Q, scale, max_new, max_kv, a)) return rc;
    if (window < 0) return fail(SPARSP_E_INVALID, "window = %d must not be negative", window);
    if (sinks < 0) return fail(SPARSP_E_INVALID, "sinks = %d must not be negative", sinks);
    if (sinks > 0 && window == 0) return fail(SPARSP_E_INVALID, "sinks need a window");
    a->window = window < kFarthest ? window : kFarthest;
    a->sinks = sinks < kFarthest ? sinks : kFarthest;
    a->k_scales = cache->K_scales;
    a->v_scales = cache->V_scales;
    return SPARSP_OK;
}

}  // namespace

extern "C" {

int sparsp_paged_append4(const sparsp_cache4* cache, int32_t tokens, int32_t dtype,
                         const sparsp_rows* K, const sparsp_rows* V, const sparsp_rotary* r,
                         const void* positions, int32_t position_bits, const float* inv_freq,
                         const sparsp_rows* Q, const sparsp_rows* Q_out, void* stream) {
    sparsp_cache c;
    sparsp::FourArgs f;
    if (int rc = check_cache4(cache, dtype, &c)) return rc;
    if (int rc = check_pointers4(cache)) return rc;
    if (int rc = check_apart4(cache)) return rc;
    if (int rc = check_new_rows(c, tokens, K, V, false, &f.rows)) return rc;
    if (r)
        if (int rc = check_rotary(r, c.d, positions, position_bits, inv_freq, &f.rows)) return rc;
    if ((Q != nullptr) != (Q_out != nullptr) || (Q && !r))
        return fail(SPARSP_E_INVALID, "Q needs Q_out and a rotation");
    if (Q) {
        const int size = dtype == SPARSP_BF16 ? 2 : 4;
        if (int rc = check_rows(Q, "Q", tokens, c.d, size)) return rc;
        if (int rc = check_rows(Q_out, "Q_out", tokens, c.d, size, true)) return rc;
        if (int rc = check_same_rows(Q, Q_out, "Q")) return rc;
        if (tokens > 0 && (Q_out->data == K->data || Q_out->data == V->data))
            return fail(SPARSP_E_INVALID, "Q_out is K or V");
        f.rows.move[f.rows.moves++] = row_move(*Q, *Q_out, true);
    }
    if (tokens == 0) return ok();
    f.k_scales = cache->K_scales;
    f.v_scales = cache->V_scales;
    return hip_status(sparsp::launch_four_append(f, (hipStream_t)stream), "sparsp_paged_append4");
}

int sparsp_paged_read4(const sparsp_cache4* cache, int32_t tokens, int32_t dtype,
                       const sparsp_rows* K, const sparsp_rows* V, void* stream) {
    sparsp_cache c;
    sparsp::FourArgs f;
    if (int rc = check_cache4(cache, dtype, &c)) return rc;
    if (int rc = check_pointers4(cache)) return rc;
    if (int rc = check_new_rows(c, tokens, K, V, true, &f.rows)) return rc;
    if (tokens > 0 && K->data == V->data) return fail(SPARSP_E_INVALID, "K and V are the same memory");
    if (tokens == 0) return ok();
    f.k_scales = cache->K_scales;
    f.v_scales = cache->V_scales;
    return hip_status(sparsp::launch_four_read(f, (hipStream_t)stream), "sparsp_paged_read4");
}

int64_t sparsp_paged_attn4_workspace_bytes(const sparsp_cache4* cache, int32_t tokens, int32_t dtype,
                                           int32_t q_heads, int32_t window, int32_t sinks,
                                           int32_t max_new, int32_t max_kv) {
    sparsp::PagedArgs a = {};
    alignas(16) char spot[16];  // (only the query rows' number of heads matters here)
    const sparsp_rows rows = {spot, 1024, 1024, q_heads, 0};
    if (int rc = check_attn4(cache, tokens, dtype, &rows, window, sinks, 1.0f, max_new, max_kv, &a))
        return rc;
    alignas(16) static const uint8_t scales[16] = {};
    a.k_scales = a.v_scales = scales;  // (that there are some)
    ok();
    return tokens == 0 ? 0 : sparsp::paged_attn_workspace(a);
}

int sparsp_paged_attn4(const sparsp_cache4* cache, int32_t tokens, int32_t dtype,
                       const sparsp_rows* Q, const sparsp_rows* O, int32_t out_dtype, float* lse,
                       int32_t causal, int32_t window, int32_t sinks, float softmax_scale,
                       int32_t max_new, int32_t max_kv, void* workspace, int64_t workspace_bytes,
                       void* stream) {
    sparsp::PagedArgs a;
    if (int rc = check_attn4(cache, tokens, dtype, Q, window, sinks, softmax_scale, max_new, max_kv, &a))
        return rc;
    if (int rc = check_pointers4(cache)) return rc;
    if (window > 0 && !causal) return fail(SPARSP_E_INVALID, "a window needs causal attention");
    if (int rc = check_output(tokens, Q, O, out_dtype, workspace, workspace_bytes, &a)) return rc;
    if (tokens == 0) return ok();
    a.causal = causal != 0;
    a.lse = lse;
    return hip_status(sparsp::launch_paged_attn(a, (hipStream_t)stream), "sparsp_paged_attn4");
}

}  // extern "C"
