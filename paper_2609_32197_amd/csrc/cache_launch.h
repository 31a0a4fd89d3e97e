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

struct PagedArgs {
    sparsp_cache cache;
    int tokens, q_heads;
    const void* Q;
    int64_t q_head, q_token;
    bool causal;
    float scale;
    int max_new, max_kv;
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

}  // namespace sparsp
