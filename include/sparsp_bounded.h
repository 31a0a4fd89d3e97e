/*
 * sparsp_bounded.h - C ABI of libsparsp for a paged cache (sparsp_cache.h) that is kept bounded: a
 * sliding window bounds what a token reads of it, 4 bits a value what it weighs, and pages are
 * shared, given back and moved together.
 *
 *   sparsp_paged_attn_window  attention over the latest tokens and a few first ones
 *   sparsp_paged_append4      new tokens' K and V into a cache of 4-bit values, K (and Q) rotated
 *   sparsp_paged_attn4        attention over such a cache, with or without a window
 *   sparsp_paged_read4        what such a cache holds of its latest tokens, back as rows
 *   sparsp_pages_reserve      pages for the tokens that come next
 *   sparsp_pages_release      back what no later token sees
 *   sparsp_pages_fork         sequences continue others, ended ones go
 *   sparsp_pages_compact      the pages in use moved together
 *   sparsp_pages_copy         contents of pages to others
 *
 * The conventions of sparsp.h and sparsp_cache.h hold.
 */
#ifndef SPARSP_BOUNDED_H
#define SPARSP_BOUNDED_H

#include "sparsp_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * sparsp_paged_attn, causal, with a sliding window: token i of n, the cached token p = kv_len - n + i,
 * sees the cached tokens t <= p with t > p - window (itself and the window - 1 before it) or
 * t < sinks. Table entries of pages that no row sees are not read, so they may name no page or
 * another sequence's; where a page is seen in part, all its tokens must be finite. window >= 1,
 * sinks >= 0. A launch costs what the window holds, not what the cache does. (Its lse is not one for
 * sparsp_paged_weights, whose rows see every cached token.)
 */
int sparsp_paged_attn_window(const sparsp_cache* cache, int32_t tokens, const sparsp_rows* Q,
                             const sparsp_rows* O, int32_t out_dtype, float* lse, int32_t window,
                             int32_t sinks, float softmax_scale, int32_t max_new, int32_t max_kv,
                             void* workspace, int64_t workspace_bytes, void* stream);

/* Workspace bytes that sparsp_paged_attn_window can use (>= 0), or a negative status. Host only. */
int64_t sparsp_paged_attn_window_workspace_bytes(const sparsp_cache* cache, int32_t tokens,
                                                 int32_t q_heads, int32_t window, int32_t sinks,
                                                 int32_t max_new, int32_t max_kv);

/*
 * A cache held in 4 bits. A code is sign (bit 3) and magnitude 0, 0.5, 1, 1.5, 2, 3, 4, 6 (bits 0-2);
 * 32 channels of a token share a scale byte s, and a code stands for its value times 2^(s - 127), or
 * for NaN where s is 255. Codes lie as [pages, H, page, d / 2], channel 2c in the low and 2c + 1 in
 * the high half of byte c; scales as [pages, H, d / 32, page], so a token's scales lie `page` bytes
 * apart. Page for page, codes and scales can be copied and shared like K and V of sparsp_cache. 4.25
 * bits a value. d is a multiple of 32 up to 128; the rest as for sparsp_cache.
 */
typedef struct {
    uint8_t *K, *K_scales, *V, *V_scales;
    const int32_t* table;   /* [B, width] page numbers */
    const int32_t* new_off; /* [B + 1] */
    const int32_t* kv_len;  /* [B] */
    int32_t pages, H, page, d, width, B;
    int32_t reserved[2]; /* 0 */
} sparsp_cache4;

/*
 * sparsp_paged_append into such a cache; rows K, V, Q and Q_out are of `dtype`. With a the largest
 * magnitude of a token's 32 channels their scale is 2^e, e = floor(log2 a) - 2 but at least -125
 * and at most 125; a code is the nearest one to the value over 2^e, of two as near the one with an
 * even code, and 6 for what is larger than 6. (So a value is off by a fifth of itself at most, or a
 * quarter where it is above 7 times the scale, or by a quarter of the scale where it is below half of
 * it.) 32 channels with an infinity or a NaN become NaN. The rotation of K is computed in 64 bits and
 * not rounded before that, so that codes do not depend on the rounding of a product; Q is rotated in
 * float32, as by sparsp_rope.
 */
int sparsp_paged_append4(const sparsp_cache4* cache, int32_t tokens, int32_t dtype,
                         const sparsp_rows* K, const sparsp_rows* V, const sparsp_rotary* r,
                         const void* positions, int32_t position_bits, const float* inv_freq,
                         const sparsp_rows* Q, const sparsp_rows* Q_out, void* stream);

/*
 * sparsp_paged_attn over what the codes stand for; Q is of `dtype`, O of out_dtype (F32 always; BF16
 * where dtype is BF16). window 0: every cached token is visible as there; window > 0 (with causal
 * only): as in sparsp_paged_attn_window. What the codes stand for is exact in bf16, and products run
 * on the bf16 matrix cores with float32 sums. bf16 rows: precision as in sparsp_paged_attn. float32
 * rows, and their probabilities, enter the products as three bf16 each, that is to 2^-24 of themselves.
 * Q must be finite, and no scale of 255 may lie among the tokens of a page that some row sees.
 */
int sparsp_paged_attn4(const sparsp_cache4* cache, int32_t tokens, int32_t dtype,
                       const sparsp_rows* Q, const sparsp_rows* O, int32_t out_dtype, float* lse,
                       int32_t causal, int32_t window, int32_t sinks, float softmax_scale,
                       int32_t max_new, int32_t max_kv, void* workspace, int64_t workspace_bytes,
                       void* stream);

/* Workspace bytes that sparsp_paged_attn4 can use (>= 0), or a negative status. Host only. */
int64_t sparsp_paged_attn4_workspace_bytes(const sparsp_cache4* cache, int32_t tokens, int32_t dtype,
                                           int32_t q_heads, int32_t window, int32_t sinks,
                                           int32_t max_new, int32_t max_kv);

/*
 * K and V [H, tokens, d] of `dtype` become what the cache holds of the new tokens (exact in either
 * type). With new_off as the running sums of kv_len that is the whole cache, token after token. A
 * token whose place has no page, or lies before the first cached one, reads as 0; columns of no
 * sequence stay as they are.
 */
int sparsp_paged_read4(const sparsp_cache4* cache, int32_t tokens, int32_t dtype,
                       const sparsp_rows* K, const sparsp_rows* V, void* stream);

/*
 * The pages of a cache and the sequences that use them. refs[p] counts the table entries that name
 * page p, and whatever else the caller counts as holding it (a prefix that is kept, say): 0 or less
 * is a free page. Tables that several calls share (one for each cache of a layer, or one for all) name
 * pages of the same numbers. Entries outside [0, pages) name no page. pages <= 2^30, B <= 65536,
 * B * width <= 2^30, width * page <= 2^30, page as in sparsp_cache.
 *
 * Calls work on the counts and tables as they find them on the stream: nothing comes back to the
 * host, so a step can be captured. Pages are taken lowest number first, in the order of the
 * entries that want them (by row, then by place), so results depend on the arguments only. Where a
 * call runs out of free pages the last of these entries name none, and *left, which otherwise is the
 * number of pages still free, is minus the number that is missing. Each call sets a *left of its own:
 * of several in a row (fork, release, reserve) each needs its own memory until all are read, and the
 * least of them says whether all pages were there. Whatever these arrays hold, no kernel leaves them, or
 * the buffers. What a call writes, its workspace and the buffers with it, may overlap no other memory of
 * its own, or it is SPARSP_E_INVALID. (Not looked at: whether two buffers overlap that begin at
 * different addresses, and whether a fork's left lies in one.)
 */
typedef struct {
    int32_t* refs;         /* [pages] */
    int32_t* table;        /* [B, width] */
    const int32_t* kv_len; /* [B] */
    int32_t pages, page, width, B;
} sparsp_pages;

/* [pages, page_bytes] of device memory: K, V, weights, codes or scales of a cache. 16-byte aligned,
 * page_bytes a multiple of 16 up to 2^32; at most 8 in a call, no memory twice. */
typedef struct {
    void* data;
    int64_t page_bytes;
} sparsp_page_buffer;

/* Workspace bytes of the calls below for these pages and rows (of a fork; otherwise B), or a negative
 * status. Host only; the pointers are not read. A workspace is 16-byte aligned device memory,
 * contents irrelevant, not shared by calls that overlap; one that is too small is SPARSP_E_CAPACITY. */
int64_t sparsp_pages_workspace_bytes(const sparsp_pages* pages, int32_t rows);

/*
 * Pages for the new tokens kv_len - n .. kv_len - 1 of every sequence (n = new_off[b+1] - new_off[b],
 * as for the append that follows): entries among theirs that name no page get a free one, its count
 * 1. The page that a sequence's last old token is on must be its own, as sparsp_pages_fork sees to.
 * Where that page is missing because an earlier call ran out of pages, the entry names none and gets
 * one like the others: the old tokens that were to be on it are not, and read as whatever the page
 * holds. *left does not tell; the earlier call's did (see above).
 */
int sparsp_pages_reserve(const sparsp_pages* pages, const int32_t* new_off, int32_t* left,
                         void* workspace, int64_t workspace_bytes, void* stream);

/*
 * Entries that no later token needs come to name no page, and their pages' counts go down by one:
 * those behind kv_len tokens (kv_len = 0 ends a sequence, a smaller kv_len takes tokens back), and
 * with window > 0 those all of whose tokens t lie in sinks <= t <= kv_len - window, which the next
 * token of a sequence of kv_len does not see (sparsp_paged_attn_window). window 0: none.
 */
int sparsp_pages_release(const sparsp_pages* pages, int32_t window, int32_t sinks, void* stream);

/*
 * Row i of the new tables continues the old row parents[i] (outside [0, B): an empty sequence), for
 * any number of rows; old rows that none continues end. Full pages are shared. A page that is filled
 * in part stays with the first row that continues its sequence if its count was 1, and is copied for
 * every other, in all the buffers, to a page of its own (never one that the call copies from). Counts:
 * refs_out is refs less the old table's entries and with the new one's. The old table, counts and
 * lengths stay as they are. So do the contents of pages that the new table names, that are copied from
 * or that something else holds, as long as nothing is written to the new table's; the pages of old rows
 * that end are free for the copies, which may overwrite them. A caller who may go back to the old table
 * counts them once more in refs, and gives that up in refs_out when it is decided. *left leaves
 * out pages that were copied from and that nothing holds any longer (a partly filled page that several
 * rows shared): no copy could go there, but refs_out has them free.
 *
 * Rows that share pages can be attended, appended to and forked on, and sparsp_pages_compact keeps them
 * shared. sparsp_paged_weights and sparsp_cache_evict take no shared pages: two rows would write the
 * same weights, and an eviction of one moves the other's tokens. A cache is cut before it is forked.
 *
 * table_out [rows, width], kv_len_out [rows], refs_out [pages], left [1].
 */
int sparsp_pages_fork(const sparsp_pages* pages, const int32_t* parents, int32_t rows,
                      const sparsp_page_buffer* buffers, int32_t count, int32_t* table_out,
                      int32_t* kv_len_out, int32_t* refs_out, int32_t* left, void* workspace,
                      int64_t workspace_bytes, void* stream);

/*
 * With n pages in use, those numbered n and above move, contents and counts, to the free ones below
 * n, lowest to lowest; *live is n. The pages from n on are free then, and may be given up. table_out
 * [B, width] and refs_out [pages] are the new ones; entries that name no page, or a free one, become
 * -1. The old table, and the contents that it names, stay as they are. kv_len and page are not used
 * (page must be valid). Only the rows of this table are rewritten: other holders of a page follow it
 * by themselves.
 */
int sparsp_pages_compact(const sparsp_pages* pages, const sparsp_page_buffer* buffers, int32_t count,
                         int32_t* table_out, int32_t* refs_out, int32_t* live, void* workspace,
                         int64_t workspace_bytes, void* stream);

/*
 * Page src[k] of every buffer to page dst[k], k < moves (device int32 arrays); a number outside [0,
 * pages) copies nothing. No page may be both a source and a destination, or a destination twice (it
 * would hold any of the contents).
 */
int sparsp_pages_copy(const sparsp_page_buffer* buffers, int32_t count, int32_t pages,
                      const int32_t* src, const int32_t* dst, int32_t moves, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SPARSP_BOUNDED_H */
