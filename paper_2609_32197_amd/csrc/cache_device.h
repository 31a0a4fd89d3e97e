// Device helpers of the paged cache: a sequence's bounds and its pages.
#pragma once

#include "cache_launch.h"
#include "sparsp_internal.h"

namespace sparsp {

// New tokens [q0, q0 + n) and cached tokens of sequence b, whatever the arrays hold.
struct Seq {
    int q0, n, kv;
};
__device__ __forceinline__ int cached_tokens(const sparsp_cache& c, int b) {
    return min(max(c.kv_len[b], 0), c.width * c.page);
}
__device__ __forceinline__ Seq sequence(const sparsp_cache& c, int tokens, int b) {
    const int lo = min(max(c.new_off[b], 0), tokens);
    const int hi = min(max(c.new_off[b + 1], lo), tokens);
    return {lo, hi - lo, cached_tokens(c, b)};
}

// Page number of page index j of sequence b, or -1.
__device__ __forceinline__ int page_of(const int32_t* table, int width, int pages, int b, int j) {
    if (j < 0 || j >= width) return -1;
    const int p = table[int64_t(b) * width + j];
    return p >= 0 && p < pages ? p : -1;
}

// x / d for 0 <= x < 2^31 by one multiplication: m = floor(2^32 / d) + 1 is exact while
// x * d < 2^32; a step corrects larger x.
struct Div {
    uint32_t d, m;
    __device__ __forceinline__ uint32_t quot(uint32_t x) const {
        uint32_t q = d == 1 ? x : __umulhi(x, m);
        if (q * d > x) --q;
        return q;
    }
};
inline Div make_div(uint32_t d) { return {d, uint32_t((uint64_t(1) << 32) / d) + 1}; }

}  // namespace sparsp
