/*
 * sparsp_bounded.h - C ABI of libsparsp for a paged cache (sparsp_cache.h) that is kept bounded: a
 * sliding window bounds what a token reads of it.
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
 * sinks >= 0. A launch costs what the window holds, not what the cache does.
 */
int sparsp_paged_attn_window(const sparsp_cache* cache, int32_t tokens, const sparsp_rows* Q,
                             const sparsp_rows* O, int32_t out_dtype, float* lse, int32_t window,
                             int32_t sinks, float softmax_scale, int32_t max_new, int32_t max_kv,
                             void* workspace, int64_t workspace_bytes, void* stream);

/* Workspace bytes that sparsp_paged_attn_window can use (>= 0), or a negative status. Host only. */
int64_t sparsp_paged_attn_window_workspace_bytes(const sparsp_cache* cache, int32_t tokens,
                                                 int32_t q_heads, int32_t window, int32_t sinks,
                                                 int32_t max_new, int32_t max_kv);

#ifdef __cplusplus
}
#endif

#endif /* SPARSP_BOUNDED_H */
