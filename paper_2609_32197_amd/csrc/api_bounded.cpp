// C ABI of the bounded cache (sparsp_bounded.h) but for the window over a cache of rows, which is
// attention like the other (api_cache.cpp): argument checks and dispatch, plain host C++.
#include <initializer_list>

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

int check_pages(const sparsp_pages* p, bool lengths) {
    if (!p) return fail(SPARSP_E_INVALID, "pages is NULL");
    if (!p->refs || !p->table || (lengths && !p->kv_len))
        return fail(SPARSP_E_INVALID, "NULL pointer of pages");
    if (p->pages < 1 || p->width < 1 || p->B < 1)
        return fail(SPARSP_E_INVALID, "pages, width and B must be positive (%d, %d, %d)", p->pages,
                    p->width, p->B);
    if (p->page < 16 || p->page > 256 || (p->page & (p->page - 1)))
        return fail(SPARSP_E_UNSUPPORTED, "page = %d must be a power of two from 16 to 256", p->page);
    if (p->pages > (1 << 30) || p->B > 65536 || int64_t(p->B) * p->width > (int64_t(1) << 30) ||
        int64_t(p->width) * p->page > (int64_t(1) << 30))
        return fail(SPARSP_E_UNSUPPORTED, "pages, B * width or width * page exceed 2^30, or B 65536");
    return SPARSP_OK;
}

int check_buffers(const sparsp_page_buffer* b, int count, sparsp::PageBuffers* f) {
    if (count < 0 || count > sparsp::kMaxBuffers || (count > 0 && !b))
        return fail(SPARSP_E_INVALID, "%d buffers, 0 to %d are supported", count, sparsp::kMaxBuffers);
    *f = {};
    int64_t units = 0;
    for (int i = 0; i < count; ++i) {
        if (!b[i].data || !aligned16(b[i].data))
            return fail(SPARSP_E_INVALID, "buffer %d must be 16-byte aligned memory", i);
        if (b[i].page_bytes < 16 || b[i].page_bytes % 16 || b[i].page_bytes > (int64_t(1) << 32))
            return fail(SPARSP_E_INVALID, "buffer %d: a page of %lld bytes is no multiple of 16", i,
                        (long long)b[i].page_bytes);
        for (int j = 0; j < i; ++j)
            if (b[j].data == b[i].data)
                return fail(SPARSP_E_INVALID, "buffers %d and %d are the same memory", j, i);
        f->data[i] = static_cast<char*>(b[i].data);
        f->bytes[i] = b[i].page_bytes;
        f->first[i] = int(units);
        units += (b[i].page_bytes + sparsp::kPageUnit - 1) / sparsp::kPageUnit;
    }
    f->count = count;
    f->units = int(units);
    return SPARSP_OK;
}

// The workspace: what a call counts and lists. Returns its size in bytes.
constexpr int kScanPages = 16384, kScanRows = 1024;  // at most so many a count
int64_t lay_out(const sparsp_pages* p, int rows, void* workspace, sparsp::PageArgs* a) {
    const int64_t counts = ((p->pages + kScanPages - 1) / kScanPages + (rows + kScanRows - 1) / kScanRows + 3) / 4 * 4;
    int32_t* at = static_cast<int32_t*>(workspace);
    const int64_t total = 4 * (4 + counts + int64_t(3) * p->pages + rows);
    if (!at) return total;
    a->moves = at;
    a->counts = at + 4;
    a->src = a->counts + counts;
    a->dst = a->src + p->pages;
    a->to = a->dst + p->pages;
    a->from = a->to + p->pages;
    return total;
}

int check_workspace(const sparsp_pages* p, int rows, void* workspace, int64_t bytes,
                    sparsp::PageArgs* a) {
    if (!workspace || !aligned16(workspace))
        return fail(SPARSP_E_INVALID, "workspace must be 16-byte aligned memory");
    const int64_t need = lay_out(p, rows, workspace, a);
    if (bytes < need)
        return fail(SPARSP_E_CAPACITY, "workspace of %lld bytes, %lld are needed", (long long)bytes,
                    (long long)need);
    return SPARSP_OK;
}

// Device memory of a page call, and whether the call writes it; apart: that it may not lie in a buffer.
struct Extent {
    const char* name;
    const void* at;
    int64_t bytes;
    bool written;
    bool apart = true;
};
bool overlap(const void* x, int64_t x_bytes, const void* y, int64_t y_bytes) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(x), b = reinterpret_cast<uintptr_t>(y);
    return a < b ? b - a < uintptr_t(x_bytes) : a - b < uintptr_t(y_bytes);
}
// What a call writes is its alone: kernels index by what they have written (a compaction by its lists
// in the workspace and by *live, say), so that memory that is two things at once would lead them
// anywhere. The contents that a call moves are written too.
int check_extents(std::initializer_list<Extent> all, const sparsp::PageBuffers* f = nullptr,
                  int64_t pages = 0) {
    for (const Extent* x = all.begin(); x != all.end(); ++x) {
        for (const Extent* y = all.begin(); y != x; ++y)
            if ((x->written || y->written) && overlap(x->at, x->bytes, y->at, y->bytes))
                return fail(SPARSP_E_INVALID, "%s and %s overlap", y->name, x->name);
        for (int i = 0; f && x->apart && i < f->count; ++i)
            if (overlap(x->at, x->bytes, f->data[i], f->bytes[i] * pages))
                return fail(SPARSP_E_INVALID, "%s and buffer %d overlap", x->name, i);
    }
    return SPARSP_OK;
}
int64_t table_bytes(int64_t rows, int width) { return 4 * rows * width; }

sparsp::PageArgs page_args(const sparsp_pages* p) {
    sparsp::PageArgs a = {};
    a.refs = p->refs;
    a.table = p->table;
    a.kv_len = p->kv_len;
    a.pages = p->pages;
    a.page = p->page;
    a.width = p->width;
    a.rows = a.old_rows = p->B;
    return a;
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

int64_t sparsp_pages_workspace_bytes(const sparsp_pages* pages, int32_t rows) {
    sparsp_pages p;
    if (!pages) return fail(SPARSP_E_INVALID, "pages is NULL");
    p = *pages;
    int32_t spot = 0;
    p.refs = p.table = &spot;  // (not read)
    if (int rc = check_pages(&p, false)) return rc;
    if (rows < 0 || rows > 65536)
        return fail(SPARSP_E_UNSUPPORTED, "rows = %d outside [0, 65536]", rows);
    ok();
    return lay_out(&p, rows > p.B ? rows : p.B, nullptr, nullptr);
}

int sparsp_pages_reserve(const sparsp_pages* pages, const int32_t* new_off, int32_t* left,
                         void* workspace, int64_t workspace_bytes, void* stream) {
    if (int rc = check_pages(pages, true)) return rc;
    if (!new_off || !left) return fail(SPARSP_E_INVALID, "new_off or left is NULL");
    sparsp::PageArgs a = page_args(pages);
    if (int rc = check_workspace(pages, pages->B, workspace, workspace_bytes, &a)) return rc;
    if (int rc = check_extents(
            {{"refs", pages->refs, 4 * int64_t(pages->pages), true},
             {"table", pages->table, table_bytes(pages->B, pages->width), true},
             {"kv_len", pages->kv_len, 4 * int64_t(pages->B), false},
             {"new_off", new_off, 4 * (int64_t(pages->B) + 1), false},
             {"left", left, 4, true},
             {"workspace", workspace, lay_out(pages, pages->B, nullptr, nullptr), true}}))
        return rc;
    a.moves = nullptr;
    a.from = nullptr;
    a.new_off = new_off;
    a.left = left;
    return hip_status(sparsp::launch_pages_reserve(a, (hipStream_t)stream), "sparsp_pages_reserve");
}

int sparsp_pages_release(const sparsp_pages* pages, int32_t window, int32_t sinks, void* stream) {
    if (int rc = check_pages(pages, true)) return rc;
    if (window < 0 || sinks < 0 || (sinks > 0 && window == 0))
        return fail(SPARSP_E_INVALID, "window = %d and sinks = %d must not be negative, sinks need a window",
                    window, sinks);
    if (int rc = check_extents({{"refs", pages->refs, 4 * int64_t(pages->pages), true},
                                {"table", pages->table, table_bytes(pages->B, pages->width), true},
                                {"kv_len", pages->kv_len, 4 * int64_t(pages->B), false}}))
        return rc;
    sparsp::PageArgs a = page_args(pages);
    a.window = window < kFarthest ? window : kFarthest;
    a.sinks = sinks;
    return hip_status(sparsp::launch_pages_release(a, (hipStream_t)stream), "sparsp_pages_release");
}

int sparsp_pages_fork(const sparsp_pages* pages, const int32_t* parents, int32_t rows,
                      const sparsp_page_buffer* buffers, int32_t count, int32_t* table_out,
                      int32_t* kv_len_out, int32_t* refs_out, int32_t* left, void* workspace,
                      int64_t workspace_bytes, void* stream) {
    sparsp::PageBuffers f;
    if (int rc = check_pages(pages, true)) return rc;
    if (rows < 1 || rows > 65536 || int64_t(rows) * pages->width > (int64_t(1) << 30))
        return fail(SPARSP_E_UNSUPPORTED, "rows = %d outside [1, 65536], or rows * width exceeds 2^30",
                    rows);
    if (int rc = check_buffers(buffers, count, &f)) return rc;
    if (!parents || !table_out || !kv_len_out || !refs_out || !left)
        return fail(SPARSP_E_INVALID, "NULL pointer of a fork");
    if (table_out == pages->table || refs_out == pages->refs || kv_len_out == pages->kv_len)
        return fail(SPARSP_E_INVALID, "a fork's outputs may not be its inputs");
    sparsp::PageArgs a = page_args(pages);
    if (int rc = check_workspace(pages, rows, workspace, workspace_bytes, &a)) return rc;
    if (int rc = check_extents(
            {{"refs", pages->refs, 4 * int64_t(pages->pages), false},
             {"table", pages->table, table_bytes(pages->B, pages->width), false},
             {"kv_len", pages->kv_len, 4 * int64_t(pages->B), false},
             {"parents", parents, 4 * int64_t(rows), false},
             {"table_out", table_out, table_bytes(rows, pages->width), true},
             {"kv_len_out", kv_len_out, 4 * int64_t(rows), true},
             {"refs_out", refs_out, 4 * int64_t(pages->pages), true},
             {"left", left, 4, true, false},  // (no kernel reads it back)
             {"workspace", workspace, lay_out(pages, rows, nullptr, nullptr), true}},
            &f, pages->pages))
        return rc;
    a.old_refs = pages->refs;
    a.old_table = pages->table;
    a.refs = refs_out;
    a.table = table_out;
    a.kv_out = kv_len_out;
    a.parents = parents;
    a.rows = rows;
    a.left = left;
    return hip_status(sparsp::launch_pages_fork(a, f, (hipStream_t)stream), "sparsp_pages_fork");
}

int sparsp_pages_compact(const sparsp_pages* pages, const sparsp_page_buffer* buffers, int32_t count,
                         int32_t* table_out, int32_t* refs_out, int32_t* live, void* workspace,
                         int64_t workspace_bytes, void* stream) {
    sparsp::PageBuffers f;
    if (int rc = check_pages(pages, false)) return rc;
    if (int rc = check_buffers(buffers, count, &f)) return rc;
    if (!table_out || !refs_out || !live) return fail(SPARSP_E_INVALID, "NULL pointer of a compaction");
    if (table_out == pages->table || refs_out == pages->refs)
        return fail(SPARSP_E_INVALID, "a compaction's outputs may not be its inputs");
    sparsp::PageArgs a = page_args(pages);
    if (int rc = check_workspace(pages, pages->B, workspace, workspace_bytes, &a)) return rc;
    if (int rc = check_extents(
            {{"refs", pages->refs, 4 * int64_t(pages->pages), false},
             {"table", pages->table, table_bytes(pages->B, pages->width), false},
             {"table_out", table_out, table_bytes(pages->B, pages->width), true},
             {"refs_out", refs_out, 4 * int64_t(pages->pages), true},
             {"live", live, 4, true},
             {"workspace", workspace, lay_out(pages, pages->B, nullptr, nullptr), true}},
            &f, pages->pages))
        return rc;
    a.old_refs = pages->refs;
    a.old_table = pages->table;
    a.refs = refs_out;
    a.table = table_out;
    a.left = live;
    return hip_status(sparsp::launch_pages_compact(a, f, (hipStream_t)stream), "sparsp_pages_compact");
}

int sparsp_pages_copy(const sparsp_page_buffer* buffers, int32_t count, int32_t pages,
                      const int32_t* src, const int32_t* dst, int32_t moves, void* stream) {
    sparsp::PageBuffers f;
    if (pages < 1 || pages > (1 << 30)) return fail(SPARSP_E_INVALID, "pages = %d out of range", pages);
    if (count < 1) return fail(SPARSP_E_INVALID, "nothing to copy");
    if (int rc = check_buffers(buffers, count, &f)) return rc;
    if (moves < 0 || moves > (1 << 30)) return fail(SPARSP_E_INVALID, "moves = %d out of range", moves);
    if (moves == 0) return ok();
    if (!src || !dst) return fail(SPARSP_E_INVALID, "src or dst is NULL");
    if (int rc = check_extents({{"src", src, 4 * int64_t(moves), false},
                                {"dst", dst, 4 * int64_t(moves), false}},
                               &f, pages))
        return rc;
    return hip_status(sparsp::launch_pages_copy(f, src, dst, moves, pages, (hipStream_t)stream),
                      "sparsp_pages_copy");
}

}  // extern "C"
