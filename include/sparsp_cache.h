/*
 * sparsp_cache.h - C ABI of libsparsp around a growing sequence: rotary
 * positions, a paged cache of keys and values, the attention of new tokens over
 * it, the attention weight its tokens receive, and its eviction by that weight.
 *
 * A step of a program that keeps a cache:
 *
 *   sparsp_paged_append    the new tokens' K and V into the cache, K (and Q) rotated
 *   sparsp_paged_attn      attention of the new tokens over the cache
 *   sparsp_paged_weights   attention weight per cached token, summed up
 *   sparsp_cache_evict     the cache cut to the tokens of most weight
 *
 * sparsp_rope alone rotates whole tensors: Q and K before sparsp_block_scores,
 * also in placed order, since every token brings its own position.
 *
 * The conventions of sparsp.h hold: device pointers owned by the caller, nothing
 * allocated, work enqueued on `stream`, argument errors found on the host before
 * anything is launched, sparsp_last_error() for the message. What lies in device
 * memory (lengths, offsets, page numbers) cannot be checked on the host; the
 * kernels bound every value they read from there as stated below, so that no
 * content of these arrays makes a kernel leave the buffers.
 *
 * Token tensors (sparsp_rows) are [heads, tokens, d] with d contiguous and any
 * strides between heads and tokens: both [H, L, d] and a projection's
 * [tokens, H, d] are read in place. Addresses and strides are multiples of 16
 * bytes, strides at least d; rows that a call writes must not overlap.
 *
 * The cache (sparsp_cache) holds K and V as [pages, H, page, d], contiguous:
 * `page` tokens of one head are one contiguous tile, page a power of two in
 * [16, 256]. Sequence b's cached token t is row t % page of page
 * table[b, t / page]. Its new tokens are the columns new_off[b] ..
 * new_off[b+1]-1 of the token tensors, and kv_len[b] counts its cached tokens
 * with the new ones: new token i of n is the cached token kv_len[b] - n + i. Offsets
 * are clamped to [0, tokens], an end below its start to the start, kv_len to
 * [0, width * page]. A page number outside [0, pages) holds no tokens: nothing is read from it
 * or written to it. new_off ascends: launches are sized for that, and where it does not, the outputs
 * in the columns of all sequences, and what is cached and weighed for them, hold any values. Columns
 * that no sequence claims, among them those before new_off[0] and behind new_off[B], keep their
 * outputs as they were whatever new_off holds.
 *
 * Limits: d <= 128 (rope alone: 256) and a multiple of 8 (bf16) or 4 (f32); H and
 * query heads <= 1024, query heads a multiple of H; B <= 65536, B * heads <= 2^20; width * page
 * <= 2^30; tokens <= 2^26, and tokens * (query heads / H) <= 2^30.
 */
#ifndef SPARSP_CACHE_H
#define SPARSP_CACHE_H

#include "sparsp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* [heads, tokens, d]; strides in elements. */
typedef struct {
    void* data;
    int64_t head_stride;
    int64_t token_stride;
    int32_t heads;
    int32_t reserved; /* 0 */
} sparsp_rows;

typedef enum { SPARSP_ROPE_HALF = 0, SPARSP_ROPE_INTERLEAVED = 1 } sparsp_rope_layout;

typedef enum {
    SPARSP_ROPE_PLAIN = 0,
    SPARSP_ROPE_LINEAR = 1, /* every frequency divided by the scale */
    SPARSP_ROPE_BASE = 2,   /* the base raised, so that the lowest frequency is divided by it */
    SPARSP_ROPE_PARTS = 3   /* long wavelengths divided, short ones kept, a ramp between */
} sparsp_rope_scaling;

/*
 * A rotation of the first rot_dim channels of a row. Pair p of rot_dim / 2 is
 * channels (p, p + rot_dim/2) in the HALF layout and (2p, 2p+1) in the
 * INTERLEAVED one. The first axis_pairs[0] pairs turn with the position on axis
 * 0, the next axis_pairs[1] with that on axis 1, and so on (a video token has
 * frame, row and column; text has one axis); they sum to rot_dim / 2.
 */
typedef struct {
    int32_t rot_dim;
    int32_t layout; /* sparsp_rope_layout */
    int32_t axes;   /* 1 .. 3 */
    int32_t axis_pairs[3];
    float factor;    /* multiplies the rotated channels */
    int32_t inverse; /* nonzero: the transposed matrix (turns back; a gradient's pass) */
} sparsp_rotary;

/*
 * The frequencies of one axis of rot_dim / 2 pairs, HOST arrays:
 *   PLAIN   f_p = theta^(-2p / rot_dim)
 *   LINEAR  f_p / scale
 *   BASE    PLAIN with theta * scale^(rot_dim / (rot_dim - 2))
 *   PARTS   with r = trained * f_p / (2 pi) turns over the trained length,
 *           g = clamp((r - low) / (high - low), 0, 1):  f_p (g + (1 - g) / scale),
 *           and *factor = 0.1 ln(scale) + 1
 * *factor is 1 otherwise. Computed in 64 bits, rounded to float32 once. scale >= 1;
 * PARTS needs trained > 0 and low < high; BASE needs rot_dim > 2. A frequency past float32's range
 * (theta far below 1) is an error. Pure host code.
 */
int sparsp_rope_frequencies(int32_t rot_dim, double theta, int32_t scaling, double scale,
                            double trained, double low, double high, float* inv_freq,
                            float* factor);

/*
 * Y_k = X_k rotated, for count (1 or 2) tensors of the same tokens (Q and K share
 * their angles). The angle of pair p of token t is positions[axis(p), t] *
 * inv_freq[p], taken modulo a turn in 64 bits; with c and s its cosine and sine
 * times factor, (x1, x2) becomes (x1 c - x2 s, x1 s + x2 c), or with `inverse`
 * (x1 c + x2 s, x2 c - x1 s). Products are float32, rounded once to the type.
 * Channels from rot_dim on are copied.
 *
 * positions: device [axes, tokens], int32 (position_bits 32) or int64 (64), any sign.
 * inv_freq: device float32 [rot_dim / 2]. x, y: HOST arrays of `count` row sets. Y_k may
 * be X_k itself (same address and strides), otherwise the tensors must not overlap.
 * tokens = 0 does nothing.
 */
int sparsp_rope(const sparsp_rotary* r, int32_t tokens, int32_t d, int32_t dtype,
                const sparsp_rows* x, const sparsp_rows* y, int32_t count, const void* positions,
                int32_t position_bits, const float* inv_freq, void* stream);

typedef struct {
    void* K;               /* [pages, H, page, d] */
    void* V;               /* the same; may be NULL for sparsp_paged_weights */
    float* weights;        /* [pages, H, page], or NULL where a call does not need it */
    const int32_t* table;  /* [B, width] page numbers */
    const int32_t* new_off; /* [B + 1]; unused by sparsp_cache_evict */
    const int32_t* kv_len; /* [B] */
    int32_t pages, H, page, d, dtype, width, B;
    int32_t reserved; /* 0 */
} sparsp_cache;

/*
 * Writes the new tokens' K and V [H, tokens, d] into the cache, and 0 into their
 * weights where cache.weights is given. With a rotation r, K is rotated on the way
 * (as by sparsp_rope), and so is Q into Q_out where Q is given (Q_out may be Q).
 * Without r, Q must be NULL. Q_out and Q apart, nothing that is written may overlap another
 * tensor, nor K of the cache its V. A token whose place has no page, or lies before the first
 * cached token (kv_len < n), is not written; its Q is rotated all the same. Places
 * that two tokens share (a page in two tables) hold either one's values.
 */
int sparsp_paged_append(const sparsp_cache* cache, int32_t tokens, const sparsp_rows* K,
                        const sparsp_rows* V, const sparsp_rotary* r, const void* positions,
                        int32_t position_bits, const float* inv_freq, const sparsp_rows* Q,
                        const sparsp_rows* Q_out, void* stream);

/*
 * Attention of the new tokens over the cache (Eq. 1 of the paper over a sequence's cached
 * tokens). Query head h reads key head h / (Q.heads / H). Token i of n of a sequence
 * sees the cached tokens t < kv_len, and with `causal` only t <= kv_len - n + i:
 *   O[h, token]   = sum_t softmax_t(scale q.k_t) v_t
 *   lse[h, token] = log sum_t exp(scale q.k_t)                (natural log)
 * A row that sees no token gets O = 0, lse = -inf.
 *
 * Q, O: [heads, tokens, d]; O in out_dtype (F32 always; BF16, rounded to nearest even,
 * for a bf16 cache). lse: float32 [heads, tokens] or NULL. (O as [heads, tokens, d] and
 * lse are what sparsp_lse_merge takes, so parts over several caches can be joined.)
 * bf16 products run on the matrix cores with float32 sums. Where max_new has at most 16 rows (tokens
 * times query heads of a key head; 32 for d <= 64) probabilities enter them to 2^-16 of
 * themselves, otherwise rounded to bf16; softmax statistics are float32. f32 products are
 * float32. The largest score of a row is subtracted from the others before anything is rounded to
 * its size, however large it is, in whole rows and in split ones; lse itself is one float32. Q,
 * and K and V where a row's sequence has tokens, must be finite; what lies in the cache outside a
 * sequence's tokens does not matter.
 *
 * max_new, max_kv: what the caller knows of the largest number of new tokens and of cached
 * tokens of a sequence (0: nothing). They size the launch; results are right for
 * any values.
 * workspace: 16-byte aligned device memory or NULL, contents irrelevant, not shared by calls
 * that overlap. With it a long cache is split among workgroups, whose float32 parts are
 * merged by a second kernel; sparsp_paged_attn_workspace_bytes says how much that uses.
 * A smaller one splits less. The split depends on the arguments only, never on timing.
 */
int sparsp_paged_attn(const sparsp_cache* cache, int32_t tokens, const sparsp_rows* Q,
                      const sparsp_rows* O, int32_t out_dtype, float* lse, int32_t causal,
                      float softmax_scale, int32_t max_new, int32_t max_kv, void* workspace,
                      int64_t workspace_bytes, void* stream);

/* Workspace bytes that sparsp_paged_attn can use (>= 0), or a negative status. Host only; the
 * cache's pointers are not read. */
int64_t sparsp_paged_attn_workspace_bytes(const sparsp_cache* cache, int32_t tokens,
                                          int32_t q_heads, int32_t max_new, int32_t max_kv);

/*
 * cache.weights[., h, .] of sequence b's cached token t gets
 *   sum over new tokens i that see t, and query heads of key head h, of
 *   exp(scale q.k_t - lse[head, token])
 * added (accumulate != 0) or written: the attention weight it received in this step,
 * with Q, lse, causal and scale as in sparsp_paged_attn. A row of lse = -inf adds
 * nothing. (lse is a float32, and a weight off by up to 2^-22 |lse| of itself.) Weights of
 * other places stay. Sums are float32 in an order that depends on the arguments only. A
 * sequence without new tokens gets 0 added. Pages must not be shared between sequences.
 */
int sparsp_paged_weights(const sparsp_cache* cache, int32_t tokens, const sparsp_rows* Q,
                         const float* lse, int32_t causal, float softmax_scale,
                         int32_t accumulate, int32_t max_new, int32_t max_kv, void* stream);

/*
 * Cuts every sequence of more than `keep` cached tokens to `keep`. Each head keeps
 * the sequence's first `first` tokens and its last `recent`, and of the others the
 * keep - first - recent of most weight (float32 order, -0 equal to +0, NaN below everything; equal
 * weights: lowest token first). They move, in their order, to places 0 .. keep-1, K, V
 * and weight; what lies behind is left as it was. A sequence of at most `keep` tokens keeps all.
 *
 * kept: int32 [B, H, keep], the kept tokens ascending, then -1. kv_len_out: int32 [B],
 * min(kv_len, keep); it may not be cache.kv_len (other workgroups still read that).
 * dst_table NULL: within the sequence's own pages. Otherwise int32 [B, dst_width] with
 * dst_width * page >= keep: the kept tokens go to those pages of the same cache, none of
 * which may be a page of `table`, and the old pages stay as they were. Pages must not be
 * shared between sequences, nor K with V (or rows would move twice). A token on a bad page weighs
 * as NaN and moves nothing. first + recent <= keep; keep >= 1.
 *
 * workspace: 16-byte aligned device memory or NULL, contents irrelevant, not shared by calls that
 * overlap. With sparsp_cache_evict_workspace_bytes bytes the choice in few long sequences is
 * shared out over more workgroups; the result is the same.
 */
int sparsp_cache_evict(const sparsp_cache* cache, int32_t keep, int32_t first, int32_t recent,
                       const int32_t* dst_table, int32_t dst_width, int32_t* kv_len_out,
                       int32_t* kept, void* workspace, int64_t workspace_bytes, void* stream);

/* Workspace bytes that sparsp_cache_evict can use for this cache's shape (0: none), or a negative
 * status. Host only; the cache's pointers are not read. */
int64_t sparsp_cache_evict_workspace_bytes(const sparsp_cache* cache);

#ifdef __cplusplus
}
#endif

#endif /* SPARSP_CACHE_H */
