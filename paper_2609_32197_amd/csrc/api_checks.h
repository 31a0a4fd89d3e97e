// Argument checks that the paged cache's entry points share (api_cache.cpp, api_bounded.cpp). Plain
// host C++, one copy for each of the two.
#pragma once

#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "cache_launch.h"

namespace {

constexpr int64_t kMaxPairs = int64_t(1) << 20;  // sequences x heads: workgroups of a launch

inline int fail(int code, const char* fmt, ...) {
    char msg[400];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof(msg), fmt, ap);
    va_end(ap);
    return sparsp::set_error(code, msg);
}

inline int ok() { return sparsp::set_error(SPARSP_OK, ""); }

inline int hip_status(hipError_t e, const char* what) {
    if (e != hipSuccess) return fail(SPARSP_E_HIP, "%s: %s", what, hipGetErrorString(e));
    return ok();
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int check_type(int d, int dtype, int most) {
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
inline bool rows_overlap(const sparsp_rows* r, int tokens, int d) {
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
inline int check_rows(const sparsp_rows* r, const char* name, int tokens, int d, int size,
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

inline int check_cache(const sparsp_cache* c) {
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
inline int check_pointers(const sparsp_cache* c, bool values, bool weights, bool batch) {
    if (!c->K || (values && !c->V) || !c->table || !c->kv_len || (batch && !c->new_off))
        return fail(SPARSP_E_INVALID, "NULL cache pointer");
    if (!aligned16(c->K) || !aligned16(c->V))
        return fail(SPARSP_E_INVALID, "K and V of the cache must be 16-byte aligned");
    if (weights && !c->weights) return fail(SPARSP_E_INVALID, "the cache has no weights");
    return SPARSP_OK;
}

// For calls that write both.
inline int check_apart(const sparsp_cache* c) {
    if (c->K == c->V) return fail(SPARSP_E_INVALID, "K and V of the cache are the same memory");
    return SPARSP_OK;
}

inline int check_tokens(int tokens) {
    if (tokens < 0 || tokens > (1 << 26))
        return fail(SPARSP_E_INVALID, "tokens = %d outside [0, 2^26]", tokens);
    return SPARSP_OK;
}

// The rotation of rows of d channels, into a.
inline int check_rotary(const sparsp_rotary* r, int d, const void* positions, int bits,
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

inline sparsp::RowMove row_move(const sparsp_rows& x, const sparsp_rows& y, bool rotate) {
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

inline sparsp::RowMove page_move(const sparsp_rows& x, void* cache, bool rotate) {
    sparsp::RowMove m = row_move(x, x, rotate);
    m.dst = cache;
    m.paged = true;
    return m;
}

inline int check_same_rows(const sparsp_rows* x, const sparsp_rows* y, const char* name) {
    if (x->heads != y->heads)
        return fail(SPARSP_E_INVALID, "%s: input and output have %d and %d heads", name, x->heads,
                    y->heads);
    if (x->data == y->data &&
        (x->head_stride != y->head_stride || x->token_stride != y->token_stride))
        return fail(SPARSP_E_INVALID, "%s: a rotation in place needs equal strides", name);
    return SPARSP_OK;
}

// What attention and weights share.
inline int check_query(const sparsp_cache* c, int tokens, const sparsp_rows* Q, float scale, int max_new,
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

// An attention call's output and workspace, into a.
inline int check_output(int tokens, const sparsp_rows* Q, const sparsp_rows* O, int out_dtype,
                 void* workspace, int64_t workspace_bytes, sparsp::PagedArgs* a) {
    if (out_dtype != SPARSP_F32 && out_dtype != SPARSP_BF16)
        return fail(SPARSP_E_DTYPE, "unknown out_dtype %d", out_dtype);
    if (a->cache.dtype == SPARSP_F32 && out_dtype != SPARSP_F32)
        return fail(SPARSP_E_DTYPE, "f32 inputs produce f32 output only");
    if (int rc = check_rows(O, "O", tokens, a->cache.d, out_dtype == SPARSP_BF16 ? 2 : 4, true)) return rc;
    if (O->heads != Q->heads)
        return fail(SPARSP_E_INVALID, "O has %d heads, Q has %d", O->heads, Q->heads);
    if (O->data == Q->data) return fail(SPARSP_E_INVALID, "O may not be Q");
    if (workspace_bytes < 0) return fail(SPARSP_E_INVALID, "workspace_bytes < 0");
    if (!aligned16(workspace)) return fail(SPARSP_E_INVALID, "workspace must be 16-byte aligned");
    a->O = O->data;
    a->o_head = O->head_stride;
    a->o_token = O->token_stride;
    a->out_bf16 = out_dtype == SPARSP_BF16;
    a->ws = workspace;
    a->ws_bytes = workspace ? workspace_bytes : 0;
    return SPARSP_OK;
}

}  // namespace
