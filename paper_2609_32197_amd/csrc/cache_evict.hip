// Eviction by accumulated attention weight: which cached tokens stay, and their move to
// the front of the sequence.
//
// select_kernel, one workgroup per (sequence, head). A weight is mapped to an unsigned key of
// the same order (NaN lowest, -0 equal to +0). The smallest kept key T is found by a radix
// search: three passes of 11, 11 and 10 bits count the keys that share the prefix found so far,
// and the digit where the running count from above reaches the number wanted is the
// next part of T. Tokens above T stay, and of those equal to T the lowest. The list is written
// in token order: each wave owns a run of tokens, counts what it keeps, and after
// one exchange of the counts writes at its place.
//
// move_kernel. The kept tokens are ascending, so place j receives a token at or behind
// j. Within the sequence's own pages a workgroup therefore moves chunks of rows in order,
// reading a whole chunk before it writes any of it: what a chunk overwrites lies before
// every token that is still to be read. To make that enough parallel work, a workgroup moves 128
// bytes of every row of K or V of a head. Into other pages the chunks are independent
// workgroups.
#include "cache_device.h"

namespace sparsp {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 2048;

__device__ __forceinline__ uint32_t weight_key(float w) {
    if (!(w == w)) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);  // -0 + 0 = +0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kThreads) void select_kernel(const sparsp_cache c, int keep, int first,
                                                          int recent, int32_t* kv_len_out,
                                                          int32_t* kept) {
    __shared__ uint32_t bins[kBins];
    __shared__ uint32_t wave_sum[kWaves];
    __shared__ uint32_t found[2];  // digit, keys above it
    __shared__ int wave_gt[kWaves], wave_eq[kWaves];
    const int b = blockIdx.x / c.H, h = blockIdx.x % c.H;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = cached_tokens(c, b);
    const int shift = __builtin_ctz(c.page);
    int32_t* list = kept + int64_t(blockIdx.x) * keep;
    if (h == 0 && tid == 0) kv_len_out[b] = min(n, keep);
    if (n <= keep) {
        for (int j = tid; j < keep; j += kThreads) list[j] = j < n ? j : -1;
        return;
    }
    for (int j = tid; j < first; j += kThreads) list[j] = j;
    for (int j = tid; j < recent; j += kThreads) list[keep - recent + j] = n - recent + j;
    const int lo = first, hi = n - recent;
    int want = keep - first - recent;  // of hi - lo > want tokens
    if (want == 0) return;

    auto key_at = [&](int t) -> uint32_t {
        const int p = page_of(c.table, c.width, c.pages, b, t >> shift);
        return p < 0 ? 0u
                     : weight_key(c.weights[(int64_t(p) * c.H + h) * c.page + (t & (c.page - 1))]);
    };

    uint32_t T = 0;
    int high = 32;  // bits of T not yet known
    for (int pass = 0; pass < 3; ++pass) {
        const int bits = pass < 2 ? 11 : 10, low = high - bits;
        for (int e = tid; e < kBins; e += kThreads) bins[e] = 0;
        __syncthreads();
        for (int t = lo + tid; t < hi; t += kThreads) {
            const uint32_t k = key_at(t);
            if (high == 32 || (k >> high) == (T >> high))
                atomicAdd(&bins[(k >> low) & ((1u << bits) - 1)], 1u);
        }
        __syncthreads();
        // Keys above each digit: thread i holds the digits 2 i and 2 i + 1 from the top.
        const int top = (1 << bits) - 1;
        const int d0 = top - 2 * tid, d1 = d0 - 1;
        const uint32_t n0 = d0 >= 0 ? bins[d0] : 0, n1 = d1 >= 0 ? bins[d1] : 0;
        uint32_t sum = n0 + n1;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t y = __shfl_up(sum, off);
            if (lane >= off) sum += y;
        }
        if (lane == 63) wave_sum[wave] = sum;
        __syncthreads();
        uint32_t before = 0;
        for (int w = 0; w < wave; ++w) before += wave_sum[w];
        const uint32_t above0 = before + sum - n0 - n1, above1 = above0 + n0;
        if (above0 < uint32_t(want) && uint32_t(want) <= above0 + n0) {
            found[0] = uint32_t(d0);
            found[1] = above0;
        }
        if (above1 < uint32_t(want) && uint32_t(want) <= above1 + n1) {
            found[0] = uint32_t(d1);
            found[1] = above1;
        }
        __syncthreads();
        T |= found[0] << low;
        want -= int(found[1]);
        high = low;
        __syncthreads();  // found and the bins are rewritten by the next pass
    }
    // want tokens equal to T stay.

    const int run = (((hi - lo) + kWaves - 1) / kWaves + 63) / 64 * 64;
    const int r0 = lo + wave * run, r1 = min(hi, r0 + run);
    int gt = 0, eq = 0;
    for (int t = r0; t < r1; t += 64) {
        const uint32_t k = t + lane < r1 ? key_at(t + lane) : 0;
        const bool in = t + lane < r1;
        gt += __popcll(__ballot(in && k > T));
        eq += __popcll(__ballot(in && k == T));
    }
    if (lane == 0) {
        wave_gt[wave] = gt;
        wave_eq[wave] = eq;
    }
    __syncthreads();
    int at = first, eq_before = 0;
    for (int w = 0; w < wave; ++w) {
        at += wave_gt[w] + max(0, min(wave_eq[w], want - eq_before));
        eq_before += wave_eq[w];
    }
    for (int t = r0; t < r1; t += 64) {
        const bool in = t + lane < r1;
        const uint32_t k = in ? key_at(t + lane) : 0;
        const uint64_t eqs = __ballot(in && k == T);
        const uint64_t below = (uint64_t(1) << lane) - 1;
        const bool take =
            in && (k > T || (k == T && eq_before + __popcll(eqs & below) < want));
        const uint64_t takes = __ballot(take);
        if (take) list[at + __popcll(takes & below)] = t + lane;
        at += __popcll(takes);
        eq_before += __popcll(eqs);
    }
}

constexpr int kSlice = 128;                       // bytes of a row that a workgroup moves
constexpr int kParts = kSlice / 16;               // lanes of a row
constexpr int kRows = kThreads / kParts;          // rows of one access of all threads
constexpr int kDeep = 4;                          // accesses of a thread in flight
constexpr int kChunk = kRows * kDeep;

// Grid: (sequence, head) x (K slices, V slices) x chunk workgroups (one where dst_table is
// not given).
__global__ __launch_bounds__(kThreads) void move_kernel(const sparsp_cache c, int keep,
                                                        const int32_t* kept,
                                                        const int32_t* dst_table, int dst_width,
                                                        int slices, int chunk_groups, int row_bytes) {
    const int group = blockIdx.x % chunk_groups;
    const int piece = blockIdx.x / chunk_groups % (2 * slices);
    const int bh = blockIdx.x / chunk_groups / (2 * slices);
    const int b = bh / c.H, h = bh % c.H;
    const bool inside = dst_table == nullptr;
    const int32_t* to_table = inside ? c.table : dst_table;
    const int to_width = inside ? c.width : dst_width;
    const int n = cached_tokens(c, b);
    if (inside && n <= keep) return;
    const int count = min(n, keep);
    char* base = static_cast<char*>(piece < slices ? c.K : c.V);
    const int at = (piece % slices) * kSlice + int(threadIdx.x % kParts) * 16;
    const bool mine = at < row_bytes;
    const bool weights = piece == 0 && threadIdx.x % kParts == 0;
    const int shift = __builtin_ctz(c.page), mask = c.page - 1;
    const int32_t* list = kept + int64_t(bh) * keep;
    for (int j0 = group * kChunk; j0 < count; j0 += chunk_groups * kChunk) {
        uint4 x[kDeep];
        float w[kDeep];
        int64_t to[kDeep];
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            const int j = j0 + u * kRows + int(threadIdx.x) / kParts;
            to[u] = -1;
            x[u] = make_uint4(0, 0, 0, 0);
            w[u] = 0.f;
            if (j >= count) continue;
            const int t = list[j];
            if (t < 0 || (inside && t == j)) continue;
            const int p = page_of(c.table, c.width, c.pages, b, t >> shift);
            const int q = page_of(to_table, to_width, c.pages, b, j >> shift);
            if (p < 0 || q < 0) continue;
            const int64_t from = (int64_t(p) * c.H + h) * c.page + (t & mask);
            to[u] = (int64_t(q) * c.H + h) * c.page + (j & mask);
            if (mine) x[u] = *reinterpret_cast<const uint4*>(base + from * row_bytes + at);
            if (weights) w[u] = c.weights[from];
        }
        if (inside) {
            // Every row of the chunk is in registers before any is overwritten.
            __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            if (to[u] < 0) continue;
            if (mine) *reinterpret_cast<uint4*>(base + to[u] * row_bytes + at) = x[u];
            if (weights) c.weights[to[u]] = w[u];
        }
        // The chunks after this one read only places behind it.
    }
}

}  // namespace

hipError_t launch_cache_evict(const sparsp_cache& c, int keep, int first, int recent,
                              const int32_t* dst_table, int dst_width, int32_t* kv_len_out,
                              int32_t* kept, hipStream_t s) {
    select_kernel<<<c.B * c.H, kThreads, 0, s>>>(c, keep, first, recent, kv_len_out, kept);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const int row_bytes = c.d * (c.dtype == SPARSP_BF16 ? 2 : 4);
    const int slices = (row_bytes + kSlice - 1) / kSlice;
    int groups = 1;
    if (dst_table) {
        const int64_t pieces = int64_t(c.B) * c.H * 2 * slices;
        const int64_t most = (keep + kChunk - 1) / kChunk;
        groups = int(most < 4096 / pieces ? most : 4096 / pieces);
        if (groups < 1) groups = 1;
    }
    move_kernel<<<c.B * c.H * 2 * slices * groups, kThreads, 0, s>>>(
        c, keep, kept, dst_table, dst_width, slices, groups, row_bytes);
    return hipGetLastError();
}

}  // namespace sparsp
