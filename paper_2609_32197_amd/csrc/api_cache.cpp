// C ABI of the paged cache (sparsp_cache.h) and of attention with a window over it
// (sparsp_bounded.h): argument checks, the rotary frequencies and dispatch. Like api.cpp it is plain
// host C++; everything is checked before a launch.
#include "../../include/sparsp_bounded.h"
#include "api_checks.h"

namespace {

// No token is further from another than this: longer windows and more sinks are the same.
constexpr int kFarthest = 1 << 30;

int check_window(int window, int sinks) {
    if (window < 1) return fail(SPARSP_E_INVALID, "window = %d must be positive", window);
    if (sinks < 0) return fail(SPARSP_E_INVALID, "sinks = %d must not be negative", sinks);
    return SPARSP_OK;
}

int64_t attn_workspace(const sparsp_cache* cache, int tokens, int q_heads, int window, int sinks,
                       int max_new, int max_kv) {
    sparsp::PagedArgs a = {};
    // A stand-in for the query rows: only their number of heads matters here.
    if (!cache) return fail(SPARSP_E_INVALID, "cache is NULL");
    alignas(16) char spot[16];
    const sparsp_rows rows = {spot, 1024, 1024, q_heads, 0};
    if (int rc = check_query(cache, tokens, &rows, 1.0f, max_new, max_kv, &a)) return rc;
    a.window = window < kFarthest ? window : kFarthest;
    a.sinks = sinks < kFarthest ? sinks : kFarthest;
    ok();
    return tokens == 0 ? 0 : sparsp::paged_attn_workspace(a);
}

int attn(const sparsp_cache* cache, int tokens, const sparsp_rows* Q, const sparsp_rows* O,
         int out_dtype, float* lse, bool causal, int window, int sinks, float softmax_scale,
         int max_new, int max_kv, void* workspace, int64_t workspace_bytes, void* stream,
         const char* name) {
    sparsp::PagedArgs a;
    if (int rc = check_query(cache, tokens, Q, softmax_scale, max_new, max_kv, &a)) return rc;
    if (int rc = check_pointers(cache, true, false, true)) return rc;
    if (int rc = check_output(tokens, Q, O, out_dtype, workspace, workspace_bytes, &a)) return rc;
    if (tokens == 0) return ok();
    a.causal = causal;
    a.window = window < kFarthest ? window : kFarthest;
    a.sinks = sinks < kFarthest ? sinks : kFarthest;
    a.lse = lse;
    return hip_status(sparsp::launch_paged_attn(a, (hipStream_t)stream), name);
}

}  // namespace

extern "C" {

int sparsp_rope_frequencies(int32_t rot_dim, double theta, int32_t scaling, double scale,
                            double trained, double low, double high, float* inv_freq,
                            float* factor) {
    if (!inv_freq || !factor) return fail(SPARSP_E_INVALID, "NULL pointer");
    if (rot_dim < 2 || rot_dim % 2 || rot_dim > 256)
        return fail(SPARSP_E_INVALID, "rot_dim = %d must be even and in [2, 256]", rot_dim);
    if (!(theta > 0.0) || !std::isfinite(theta))
        return fail(SPARSP_E_INVALID, "theta must be positive and finite");
    if (scaling < SPARSP_ROPE_PLAIN || scaling > SPARSP_ROPE_PARTS)
        return fail(SPARSP_E_INVALID, "unknown scaling %d", scaling);
    if (scaling != SPARSP_ROPE_PLAIN && !(scale >= 1.0 && std::isfinite(scale)))
        return fail(SPARSP_E_INVALID, "scale must be at least 1 and finite");
    if (scaling == SPARSP_ROPE_BASE && rot_dim == 2)
        return fail(SPARSP_E_INVALID, "raising the base needs rot_dim > 2");
    if (scaling == SPARSP_ROPE_PARTS &&
        !(trained > 0.0 && std::isfinite(trained) && low < high && std::isfinite(high - low)))
        return fail(SPARSP_E_INVALID, "PARTS needs trained > 0 and low < high");
    if (scaling == SPARSP_ROPE_BASE) theta *= std::pow(scale, double(rot_dim) / (rot_dim - 2));
    for (int p = 0; p < rot_dim / 2; ++p) {
        double f = std::pow(theta, -2.0 * p / rot_dim);
        if (scaling == SPARSP_ROPE_LINEAR) f /= scale;
        if (scaling == SPARSP_ROPE_PARTS) {
            const double turns = trained * f / 6.283185307179586476925;
            double g = (turns - low) / (high - low);
            g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
            f *= g + (1.0 - g) / scale;
        }
        inv_freq[p] = float(f);
        if (!std::isfinite(inv_freq[p]))
            return fail(SPARSP_E_INVALID, "theta = %g: frequency %d is no float32", theta, p);
    }
    *factor = scaling == SPARSP_ROPE_PARTS ? float(0.1 * std::log(scale) + 1.0) : 1.0f;
    return ok();
}

int sparsp_rope(const sparsp_rotary* r, int32_t tokens, int32_t d, int32_t dtype,
                const sparsp_rows* x, const sparsp_rows* y, int32_t count, const void* positions,
                int32_t position_bits, const float* inv_freq, void* stream) {
    sparsp::RotateArgs a;
    if (int rc = check_type(d, dtype, 256)) return rc;
    if (int rc = check_tokens(tokens)) return rc;
    if (count < 1 || count > 2 || !x || !y)
        return fail(SPARSP_E_INVALID, "count = %d must be 1 or 2, with x and y", count);
    if (int rc = check_rotary(r, d, positions, position_bits, inv_freq, &a)) return rc;
    const int size = dtype == SPARSP_BF16 ? 2 : 4;
    for (int k = 0; k < count; ++k) {
        if (int rc = check_rows(x + k, "X", tokens, d, size)) return rc;
        if (int rc = check_rows(y + k, "Y", tokens, d, size, true)) return rc;
        if (int rc = check_same_rows(x + k, y + k, "X")) return rc;
        a.move[k] = row_move(x[k], y[k], true);
    }
    // (empty tensors have no address of their own)
    if (tokens > 0 && count == 2 &&
        (y[0].data == y[1].data || y[0].data == x[1].data || y[1].data == x[0].data))
        return fail(SPARSP_E_INVALID, "an output is the other output or the other's input");
    if (tokens == 0) return ok();
    a.moves = count;
    a.tokens = tokens;
    a.d = d;
    a.bf16 = dtype == SPARSP_BF16;
    return hip_status(sparsp::launch_rotate_rows(a, (hipStream_t)stream), "sparsp_rope");
}

int sparsp_paged_append(const sparsp_cache* cache, int32_t tokens, const sparsp_rows* K,
                        const sparsp_rows* V, const sparsp_rotary* r, const void* positions,
                        int32_t position_bits, const float* inv_freq, const sparsp_rows* Q,
                        const sparsp_rows* Q_out, void* stream) {
    sparsp::RotateArgs a;
    if (int rc = check_cache(cache)) return rc;
    if (int rc = check_tokens(tokens)) return rc;
    if (int rc = check_pointers(cache, true, false, true)) return rc;
    if (int rc = check_apart(cache)) return rc;
    const int size = cache->dtype == SPARSP_BF16 ? 2 : 4;
    if (int rc = check_rows(K, "K", tokens, cache->d, size)) return rc;
    if (int rc = check_rows(V, "V", tokens, cache->d, size)) return rc;
    if (K->heads != cache->H || V->heads != cache->H)
        return fail(SPARSP_E_INVALID, "K and V have %d and %d heads, the cache has %d", K->heads,
                    V->heads, cache->H);
    if (r)
        if (int rc = check_rotary(r, cache->d, positions, position_bits, inv_freq, &a)) return rc;
    if ((Q != nullptr) != (Q_out != nullptr) || (Q && !r))
        return fail(SPARSP_E_INVALID, "Q needs Q_out and a rotation");
    a.move[0] = page_move(*K, cache->K, r != nullptr);
    a.move[1] = page_move(*V, cache->V, false);
    a.moves = 2;
    if (Q) {
        if (int rc = check_rows(Q, "Q", tokens, cache->d, size)) return rc;
        if (int rc = check_rows(Q_out, "Q_out", tokens, cache->d, size, true)) return rc;
        if (int rc = check_same_rows(Q, Q_out, "Q")) return rc;
        a.move[a.moves++] = row_move(*Q, *Q_out, true);
    }
    if (tokens == 0) return ok();
    a.tokens = tokens;
    a.d = cache->d;
    a.bf16 = cache->dtype == SPARSP_BF16;
    a.cache = *cache;
    return hip_status(sparsp::launch_rotate_rows(a, (hipStream_t)stream), "sparsp_paged_append");
}

int64_t sparsp_paged_attn_workspace_bytes(const sparsp_cache* cache, int32_t tokens,
                                          int32_t q_heads, int32_t max_new, int32_t max_kv) {
    return attn_workspace(cache, tokens, q_heads, 0, 0, max_new, max_kv);
}

int64_t sparsp_paged_attn_window_workspace_bytes(const sparsp_cache* cache, int32_t tokens,
                                                 int32_t q_heads, int32_t window, int32_t sinks,
                                                 int32_t max_new, int32_t max_kv) {
    if (int rc = check_window(window, sinks)) return rc;
    return attn_workspace(cache, tokens, q_heads, window, sinks, max_new, max_kv);
}

int sparsp_paged_attn(const sparsp_cache* cache, int32_t tokens, const sparsp_rows* Q,
                      const sparsp_rows* O, int32_t out_dtype, float* lse, int32_t causal,
                      float softmax_scale, int32_t max_new, int32_t max_kv, void* workspace,
                      int64_t workspace_bytes, void* stream) {
    return attn(cache, tokens, Q, O, out_dtype, lse, causal != 0, 0, 0, softmax_scale, max_new,
                max_kv, workspace, workspace_bytes, stream, "sparsp_paged_attn");
}

int sparsp_paged_attn_window(const sparsp_cache* cache, int32_t tokens, const sparsp_rows* Q,
                             const sparsp_rows* O, int32_t out_dtype, float* lse, int32_t window,
                             int32_t sinks, float softmax_scale, int32_t max_new, int32_t max_kv,
                             void* workspace, int64_t workspace_bytes, void* stream) {
    if (int rc = check_window(window, sinks)) return rc;
    return attn(cache, tokens, Q, O, out_dtype, lse, true, window, sinks, softmax_scale, max_new,
                max_kv, workspace, workspace_bytes, stream, "sparsp_paged_attn_window");
}

int sparsp_paged_weights(const sparsp_cache* cache, int32_t tokens, const sparsp_rows* Q,
                         const float* lse, int32_t causal, float softmax_scale,
                         int32_t accumulate, int32_t max_new, int32_t max_kv, void* stream) {
    sparsp::PagedArgs a;
    if (int rc = check_query(cache, tokens, Q, softmax_scale, max_new, max_kv, &a)) return rc;
    if (int rc = check_pointers(cache, false, true, true)) return rc;
    if (!lse) return fail(SPARSP_E_INVALID, "lse is NULL");
    if (tokens == 0 && accumulate) return ok();
    a.causal = causal != 0;
    a.lse_in = lse;
    a.accumulate = accumulate != 0;
    return hip_status(sparsp::launch_paged_weights(a, (hipStream_t)stream), "sparsp_paged_weights");
}

int64_t sparsp_cache_evict_workspace_bytes(const sparsp_cache* cache) {
    if (int rc = check_cache(cache)) return rc;
    ok();
    return sparsp::evict_workspace(*cache);
}

int sparsp_cache_evict(const sparsp_cache* cache, int32_t keep, int32_t first, int32_t recent,
                       const int32_t* dst_table, int32_t dst_width, int32_t* kv_len_out,
                       int32_t* kept, void* workspace, int64_t workspace_bytes, void* stream) {
    if (int rc = check_cache(cache)) return rc;
    if (int rc = check_pointers(cache, true, true, false)) return rc;
    if (int rc = check_apart(cache)) return rc;
    if (!kv_len_out || !kept) return fail(SPARSP_E_INVALID, "kv_len_out or kept is NULL");
    if (kv_len_out == cache->kv_len)
        return fail(SPARSP_E_INVALID, "kv_len_out may not be the cache's kv_len");
    if (kept == cache->kv_len || kept == kv_len_out)
        return fail(SPARSP_E_INVALID, "kept may not be a list of lengths");
    if (keep < 1 || keep > (1 << 30)) return fail(SPARSP_E_INVALID, "keep = %d must be positive", keep);
    if (first < 0 || recent < 0 || int64_t(first) + recent > keep)
        return fail(SPARSP_E_INVALID, "first = %d and recent = %d must fit into keep = %d", first,
                    recent, keep);
    if (dst_table) {
        if (dst_table == cache->table)
            return fail(SPARSP_E_INVALID, "dst_table may not be the cache's table (pass NULL)");
        if (dst_width < 1 || int64_t(dst_width) * cache->page < keep ||
            int64_t(dst_width) * cache->page > (int64_t(1) << 30))
            return fail(SPARSP_E_CAPACITY, "dst_width = %d pages of %d hold fewer than keep = %d",
                        dst_width, cache->page, keep);
    }
    if (workspace_bytes < 0) return fail(SPARSP_E_INVALID, "workspace_bytes < 0");
    if (!aligned16(workspace)) return fail(SPARSP_E_INVALID, "workspace must be 16-byte aligned");
    return hip_status(sparsp::launch_cache_evict(*cache, keep, first, recent, dst_table, dst_width,
                                                 kv_len_out, kept, workspace,
                                                 workspace ? workspace_bytes : 0,
                                                 (hipStream_t)stream),
                      "sparsp_cache_evict");
}

}  // extern "C"
