// Host interface between the C ABI of the paged cache (api_cache.cpp) and its HIP
// translation units, as sparsp_launch.h is for the four steps. Arguments are checked
// before any launcher is called.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include "../../include/sparsp_cache.h"

namespace sparsp {

// Sets the calling thread's error message and returns code (defined beside
// sparsp_last_error).
int set_error(int code, const char* msg);

// Token rows of one tensor on their way: from src to dst, or into the cache's pages.
struct RowMove {
    const void* src = nullptr;
    int64_t src_head = 0, src_token = 0;
    void* dst = nullptr;  // a strided tensor, or the paged K or V
    int64_t dst_head = 0, dst_token = 0;
    int heads = 0;
    bool paged = false, rotate = false;
};

struct RotateArgs {
    RowMove move[3];
    int moves = 0;
    int tokens = 0, d = 0;
    bool bf16 = false;
    // Rotation; rot = 0 moves rows as they are.
    int rot = 0, layout = 0;
    int axis_end[3] = {};  // pairs before axis_end[a] turn with axis a or an earlier one
    float factor = 1.f;
    bool inverse = false;
    const void* positions = nullptr;
    bool wide = false;  // 64-bit positions
    const float* inv_freq = nullptr;
    sparsp_cache cache = {};  // for paged moves
};
hipError_t launch_rotate_rows(const RotateArgs& a, hipStream_t s);

// New tokens into a cache held in 4 bits, and what it holds of them back. cache.K and cache.V are
// codes, cache.dtype is the rows'.
struct FourArgs {
    RotateArgs rows;  // move[0]: K, move[1]: V; move[2]: Q
    uint8_t *k_scales = nullptr, *v_scales = nullptr;
};
hipError_t launch_four_append(const FourArgs& a, hipStream_t s);
hipError_t launch_four_read(const FourArgs& a, hipStream_t s);

struct PagedArgs {
    sparsp_cache cache;
    // Of a cache held in 4 bits, whose K and V are codes and whose dtype is that of the rows; or NULL.
    const uint8_t *k_scales, *v_scales;
    int tokens, q_heads;
    const void* Q;
    int64_t q_head, q_token;
    bool causal;
    float scale;
    int max_new, max_kv;
    int window, sinks;  // window 0: none
    // attention
    void* O;
    int64_t o_head, o_token;
    bool out_bf16;
    float* lse;
    void* ws;
    int64_t ws_bytes;
    // weights
    const float* lse_in;
    bool accumulate;
};
hipError_t launch_paged_attn(const PagedArgs& a, hipStream_t s);
int64_t paged_attn_workspace(const PagedArgs& a);
hipError_t launch_paged_weights(const PagedArgs& a, hipStream_t s);

hipError_t launch_cache_evict(const sparsp_cache& c, int keep, int first, int recent,
                              const int32_t* dst_table, int dst_width, int32_t* kv_len_out,
                              int32_t* kept, void* ws, int64_t ws_bytes, hipStream_t s);
// Bytes of workspace that its choice can use.
int64_t evict_workspace(const sparsp_cache& c);

// Pages of a cache: the tables and counts of a call, and the contents that it copies.
struct PageArgs {
    int32_t *refs, *table;          // written (the new ones, where there are old ones)
    const int32_t *old_refs, *old_table;
    const int32_t *kv_len, *new_off, *parents;
    int32_t* kv_out;
    int pages, page, width, rows, old_rows;
    int window, sinks;
    int32_t* left;    // [1]
    // workspace
    int32_t* moves;   // [1]
    int32_t* counts;  // of chunks
    int32_t *src, *dst, *to, *from;
};
constexpr int kMaxBuffers = 8;
struct PageBuffers {
    char* data[kMaxBuffers];
    int64_t bytes[kMaxBuffers];  // of a page
    int first[kMaxBuffers];      // of a page's copying units, each buffer's first
    int count, units;
};
constexpr int kPageUnit = 16384;  // bytes of a unit at most
hipError_t launch_pages_reserve(const PageArgs& a, hipStream_t s);
hipError_t launch_pages_release(const PageArgs& a, hipStream_t s);
hipError_t launch_pages_fork(const PageArgs& a, const PageBuffers& f, hipStream_t s);
hipError_t launch_pages_copy(const PageBuffers& f, const int32_t* src, const int32_t* dst, int count,
                             int pages, hipStream_t s);
hipError_t launch_pages_compact(const PageArgs& a, const PageBuffers& f, hipStream_t s);

}  // namespace sparsp
