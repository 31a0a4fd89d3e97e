// C ABI of the paged cache (sparsp_cache.h): argument checks, the rotary frequencies and
// dispatch. Like api.cpp it is plain host C++; everything is checked before a launch.
#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "cache_launch.h"

namespace {

constexpr int64_t kMaxPairs = int64_t(1) << 20;  // sequences x heads: workgroups of a launch

int fail(int code, const char* fmt, ...) {
    char msg[400];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof(msg), fmt, ap);
    va_end(ap);
    return sparsp::set_error(code, msg);
}

int ok() { return sparsp::set_error(SPARSP_OK, ""); }

int hip_status(hipError_t e, const char* what) {
    if (e != hipSuccess) return fail(SPARSP_E_HIP, "%s: %s", what, hipGetErrorString(e));
    return ok();
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_type(int d, int dtype, int most) {
    if (dtype != SPARSP_F32 && dtype != SPARSP_BF16)
        return fail(SPARSP_E_DTYPE, "unknown dtype %d", dtype);
    if (d <= 0) return fail(SPARSP_E_INVALID, "d = %d must be positive", d);
    const int vec = dtype == SPARSP_BF16 ? 8 : 4;
    if (d > most || d % vec)
        return fail(SPARSP_E_UNSUPPORTED, "d = %d must be a multiple of %d up to %d for this dtype",
                    d, vec, most);
    return SPARSP_OK;
}

// Whether two of a tensor's rows share a channel; both strides are d at least. Heads beside one
// another behind all tokens, or tokens behind all heads, are seen at once; else the token that begins
// next to each head's first decides.
bool rows_overlap(const sparsp_rows* r, int tokens, int d) {
    const int64_t hs = r->head_stride, ts = r->token_stride;
    if (r->heads < 2 || tokens < 2) return false;
    if ((hs - d) / ts >= tokens - 1 || (ts - d) / hs >= r->heads - 1) return false;
    for (int64_t at = hs; at < r->heads * hs; at += hs) {
        const int64_t t = at / ts;
        if (t < tokens && at - t * ts < d) return true;
        if (t + 1 < tokens && (t + 1) * ts - at < d) return true;
    }
    return false;
}

// A [heads, tokens, d] tensor of elements of `size` bytes.
int check_rows(const sparsp_rows* r, const char* name, int tokens, int d, int size,
               bool written = false) {
    if (!r || !r->data) return fail(SPARSP_E_INVALID, "%s is NULL", name);
    if (r->heads < 1 || r->heads > 1024)
        return fail(SPARSP_E_UNSUPPORTED, "%s has %d heads, 1 to 1024 are supported", name, r->heads);
    if (!aligned16(r->data) || r->head_stride * size % 16 || r->token_stride * size % 16)
        return fail(SPARSP_E_INVALID, "%s: address and strides must be multiples of 16 bytes", name);
    const int64_t most = int64_t(1) << 40;
    if (r->head_stride < 0 || r->token_stride < 0 || r->head_stride > most || r->token_stride > most)
        return fail(SPARSP_E_INVALID, "%s: stride out of range", name);
    if ((tokens > 1 && r->token_stride < d) || (r->heads > 1 && r->head_stride < d))
        return fail(SPARSP_E_INVALID, "%s: strides below d = %d", name, d);
    if (written && rows_overlap(r, tokens, d))
        return fail(SPARSP_E_INVALID, "%s: its rows overlap", name);
    return SPARSP_OK;
}

int check_cache(const sparsp_cache* c) {
    if (!c) return fail(SPARSP_E_INVALID, "cache is NULL");
    if (int rc = check_type(c->d, c->dtype, 128)) return rc;
    if (c->pages < 1 || c->width < 1 || c->B < 1)
        return fail(SPARSP_E_INVALID, "pages, width and B must be positive (%d, %d, %d)", c->pages,
                    c->width, c->B);
    if (c->H < 1 || c->H > 1024)
        return fail(SPARSP_E_UNSUPPORTED, "H = %d, 1 to 1024 are supported", c->H);
    if (c->page < 16 || c->page > 256 || (c->page & (c->page - 1)))
        return fail(SPARSP_E_UNSUPPORTED, "page = %d must be a power of two from 16 to 256", c->page);
    if (int64_t(c->width) * c->page > (int64_t(1) << 30))
        return fail(SPARSP_E_UNSUPPORTED, "width * page = %lld exceeds 2^30",
                    (long long)(int64_t(c->width) * c->page));
    if (c->B > 65536 || int64_t(c->B) * c->H > kMaxPairs)
        return fail(SPARSP_E_UNSUPPORTED, "B = %d exceeds 65536, or B * H = %lld exceeds 2^20", c->B,
                    (long long)(int64_t(c->B) * c->H));
    return SPARSP_OK;
}

// The device arrays that a call reads.
int check_pointers(const sparsp_cache* c, bool values, bool weights, bool batch) {
    if (!c->K || (values && !c->V) || !c->table || !c->kv_len || (batch && !c->new_off))
        return fail(SPARSP_E_INVALID, "NULL cache pointer");
    if (!aligned16(c->K) || !aligned16(c->V))
        return fail(SPARSP_E_INVALID, "K and V of the cache must be 16-byte aligned");
    if (weights && !c->weights) return fail(SPARSP_E_INVALID, "the cache has no weights");
    return SPARSP_OK;
}

// For calls that write both.
int check_apart(const sparsp_cache* c) {
    if (c->K == c->V) return fail(SPARSP_E_INVALID, "K and V of the cache are the same memory");
    return SPARSP_OK;
}

int check_tokens(int tokens) {
    if (tokens < 0 || tokens > (1 << 26))
        return fail(SPARSP_E_INVALID, "tokens = %d outside [0, 2^26]", tokens);
    return SPARSP_OK;
}

// The rotation of rows of d channels, into a.
int check_rotary(const sparsp_rotary* r, int d, const void* positions, int bits,
                 const float* inv_freq, sparsp::RotateArgs* a) {
    if (!r) return fail(SPARSP_E_INVALID, "the rotation is NULL");
    if (r->rot_dim < 2 || r->rot_dim > d || r->rot_dim % 2)
        return fail(SPARSP_E_INVALID, "rot_dim = %d must be even and in [2, d = %d]", r->rot_dim, d);
    if (r->layout != SPARSP_ROPE_HALF && r->layout != SPARSP_ROPE_INTERLEAVED)
        return fail(SPARSP_E_INVALID, "unknown layout %d", r->layout);
    if (r->axes < 1 || r->axes > 3)
        return fail(SPARSP_E_INVALID, "axes = %d outside [1, 3]", r->axes);
    int sum = 0;
    for (int x = 0; x < 3; ++x) {
        const int pairs = x < r->axes ? r->axis_pairs[x] : 0;
        if (pairs < 0 || pairs > r->rot_dim / 2)
            return fail(SPARSP_E_INVALID, "axis_pairs[%d] = %d out of range", x, pairs);
        sum += pairs;
        a->axis_end[x] = x < r->axes - 1 ? sum : 1 << 30;  // the last axis takes the rest
    }
    if (sum != r->rot_dim / 2)
        return fail(SPARSP_E_INVALID, "axis_pairs sum to %d, rot_dim / 2 is %d", sum, r->rot_dim / 2);
    if (!std::isfinite(r->factor)) return fail(SPARSP_E_INVALID, "factor must be finite");
    if (!positions || !inv_freq) return fail(SPARSP_E_INVALID, "positions or inv_freq is NULL");
    if (bits != 32 && bits != 64)
        return fail(SPARSP_E_DTYPE, "position_bits = %d must be 32 or 64", bits);
    a->rot = r->rot_dim;
    a->layout = r->layout;
    a->factor = r->factor;
    a->inverse = r->inverse != 0;
    a->positions = positions;
    a->wide = bits == 64;
    a->inv_freq = inv_freq;
    return SPARSP_OK;
}

sparsp::RowMove row_move(const sparsp_rows& x, const sparsp_rows& y, bool rotate) {
    sparsp::RowMove m;
    m.src = x.data;
    m.src_head = x.head_stride;
    m.src_token = x.token_stride;
    m.dst = y.data;
    m.dst_head = y.head_stride;
    m.dst_token = y.token_stride;
    m.heads = x.heads;
    m.rotate = rotate;
    return m;
}

sparsp::RowMove page_move(const sparsp_rows& x, void* cache, bool rotate) {
    sparsp::RowMove m = row_move(x, x, rotate);
    m.dst = cache;
    m.paged = true;
    return m;
}

int check_same_rows(const sparsp_rows* x, const sparsp_rows* y, const char* name) {
    if (x->heads != y->heads)
        return fail(SPARSP_E_INVALID, "%s: input and output have %d and %d heads", name, x->heads,
                    y->heads);
    if (x->data == y->data &&
        (x->head_stride != y->head_stride || x->token_stride != y->token_stride))
        return fail(SPARSP_E_INVALID, "%s: a rotation in place needs equal strides", name);
    return SPARSP_OK;
}

// What attention and weights share.
int check_query(const sparsp_cache* c, int tokens, const sparsp_rows* Q, float scale, int max_new,
                int max_kv, sparsp::PagedArgs* a) {
    if (int rc = check_cache(c)) return rc;
    if (int rc = check_tokens(tokens)) return rc;
    if (int rc = check_rows(Q, "Q", tokens, c->d, c->dtype == SPARSP_BF16 ? 2 : 4)) return rc;
    if (Q->heads % c->H)
        return fail(SPARSP_E_INVALID, "%d query heads are no multiple of H = %d", Q->heads, c->H);
    if (int64_t(c->B) * Q->heads > kMaxPairs)
        return fail(SPARSP_E_UNSUPPORTED, "B * query heads exceeds 2^20");
    if (int64_t(tokens) * (Q->heads / c->H) > (int64_t(1) << 30))
        return fail(SPARSP_E_UNSUPPORTED, "tokens * query heads of a key head exceeds 2^30");
    if (!(scale > 0.0f) || scale > 1e30f)
        return fail(SPARSP_E_INVALID, "softmax_scale must be positive and finite");
    if (max_new < 0 || max_kv < 0) return fail(SPARSP_E_INVALID, "max_new or max_kv < 0");
    *a = {};
    a->cache = *c;
    a->tokens = tokens;
    a->q_heads = Q->heads;
    a->Q = Q->data;
    a->q_head = Q->head_stride;
    a->q_token = Q->token_stride;
    a->scale = scale;
    a->max_new = max_new;
    a->max_kv = max_kv;
    return SPARSP_OK;
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
    sparsp::PagedArgs a = {};
    // A stand-in for the query rows: only their number of heads matters here.
    if (!cache) return fail(SPARSP_E_INVALID, "cache is NULL");
    alignas(16) char spot[16];
    const sparsp_rows rows = {spot, 1024, 1024, q_heads, 0};
    if (int rc = check_query(cache, tokens, &rows, 1.0f, max_new, max_kv, &a)) return rc;
    ok();
    return tokens == 0 ? 0 : sparsp::paged_attn_workspace(a);
}

int sparsp_paged_attn(const sparsp_cache* cache, int32_t tokens, const sparsp_rows* Q,
                      const sparsp_rows* O, int32_t out_dtype, float* lse, int32_t causal,
                      float softmax_scale, int32_t max_new, int32_t max_kv, void* workspace,
                      int64_t workspace_bytes, void* stream) {
    sparsp::PagedArgs a;
    if (int rc = check_query(cache, tokens, Q, softmax_scale, max_new, max_kv, &a)) return rc;
    if (int rc = check_pointers(cache, true, false, true)) return rc;
    if (out_dtype != SPARSP_F32 && out_dtype != SPARSP_BF16)
        return fail(SPARSP_E_DTYPE, "unknown out_dtype %d", out_dtype);
    if (cache->dtype == SPARSP_F32 && out_dtype != SPARSP_F32)
        return fail(SPARSP_E_DTYPE, "f32 inputs produce f32 output only");
    if (int rc = check_rows(O, "O", tokens, cache->d, out_dtype == SPARSP_BF16 ? 2 : 4, true)) return rc;
    if (O->heads != Q->heads)
        return fail(SPARSP_E_INVALID, "O has %d heads, Q has %d", O->heads, Q->heads);
    if (O->data == Q->data) return fail(SPARSP_E_INVALID, "O may not be Q");
    if (workspace_bytes < 0) return fail(SPARSP_E_INVALID, "workspace_bytes < 0");
    if (!aligned16(workspace)) return fail(SPARSP_E_INVALID, "workspace must be 16-byte aligned");
    if (tokens == 0) return ok();
    a.causal = causal != 0;
    a.O = O->data;
    a.o_head = O->head_stride;
    a.o_token = O->token_stride;
    a.out_bf16 = out_dtype == SPARSP_BF16;
    a.lse = lse;
    a.ws = workspace;
    a.ws_bytes = workspace ? workspace_bytes : 0;
    return hip_status(sparsp::launch_paged_attn(a, (hipStream_t)stream), "sparsp_paged_attn");
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
