// Eviction by accumulated attention weight: which cached tokens stay, and their move to
// the front of the sequence.
//
// select_kernel, one workgroup per (sequence, head). A weight is mapped to an unsigned key of
// the same order (NaN lowest, -0 equal to +0). The smallest kept key T is found by a radix
// search: the keys are counted by their first 11 bits, and the digit where the count from
// above reaches the number wanted is the beginning of T. The few keys that share it are
// collected in LDS, where passes of 11 and 10 bits find the rest (over all keys again, should
// they be more than fit). Tokens above T stay, and of those equal to T the lowest. The list is
// written in token order: each wave owns a run of tokens, and the counts of what the waves
// before it keep give it its place. So three passes read the weights, each with eight loads of
// a wave in flight and the page numbers in LDS (100,003 tokens took 235 us in five passes of
// one dependent load each, and take 116 us). Few long sequences are shared out over more
// workgroups, in three launches that hand their counts on through a workspace.
//
// move_kernel. The kept tokens are ascending, so place j receives a token at or behind
// j. Within the sequence's own pages a workgroup therefore moves chunks of rows in order,
// reading a whole chunk before it writes any of it: what a chunk overwrites lies before
// every token that is still to be read. To make that enough parallel work, a workgroup moves 128
// bytes of every row of K or V of a head. Into other pages the chunks are independent
// workgroups, which move whole rows.
#include <algorithm>

#include "cache_device.h"

namespace sparsp {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 2048;

typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t weight_key(float w) {
    if (!(w == w)) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);  // -0 + 0 = +0
    return u ^ (uint32_t(int32_t(u) >> 31) | 0x80000000u);
}

constexpr int kPages = 8192;       // page numbers held in LDS
constexpr int kCandidates = 4096;  // keys held in LDS
constexpr int kAhead = 8;          // loads of a lane in flight
constexpr int kSegments = 32;      // workgroups for a (sequence, head) at most

struct SelectLds {
    uint32_t bins[kBins];
    uint32_t wave_sum[kWaves];
    uint32_t found[2];  // digit, keys above it
    int wave_gt[kWaves], wave_eq[kWaves];
    int candidates;
    int pages[kPages];
};

__device__ __forceinline__ void clear_bins(SelectLds& l) {
    for (int e = threadIdx.x; e < kBins; e += kThreads) l.bins[e] = 0;
}

// The digit of `bits` bits in bins where the count from above reaches want, into found.
__device__ __forceinline__ void find_digit(SelectLds& l, int bits, int want) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    __syncthreads();
    // Thread i holds the digits 2 i and 2 i + 1 from the top.
    const int d0 = (1 << bits) - 1 - 2 * tid, d1 = d0 - 1;
    const uint32_t n0 = d0 >= 0 ? l.bins[d0] : 0, n1 = d1 >= 0 ? l.bins[d1] : 0;
    uint32_t sum = n0 + n1;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t y = __shfl_up(sum, off);
        if (lane >= off) sum += y;
    }
    if (lane == 63) l.wave_sum[wave] = sum;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < wave; ++w) before += l.wave_sum[w];
    const uint32_t above0 = before + sum - n0 - n1, above1 = above0 + n0;
    if (above0 < uint32_t(want) && uint32_t(want) <= above0 + n0) {
        l.found[0] = uint32_t(d0);
        l.found[1] = above0;
    }
    if (above1 < uint32_t(want) && uint32_t(want) <= above1 + n1) {
        l.found[0] = uint32_t(d1);
        l.found[1] = above1;
    }
    __syncthreads();
}

// The choice of one (sequence, head): `want` of the tokens [lo, hi), more than want of them.
struct Choice {
    int b, h, n, lo, hi, want;
};
// 0: nothing to choose (everything stays, or the first and recent tokens are all).
__device__ __forceinline__ bool choice_of(const sparsp_cache& c, int pair, int keep, int first,
                                          int recent, Choice* x) {
    x->b = pair / c.H;
    x->h = pair % c.H;
    x->n = cached_tokens(c, x->b);
    x->lo = first;
    x->hi = x->n - recent;
    x->want = keep - first - recent;
    return x->n > keep && x->want > 0;
}

// The tokens [lo, hi) of a choice that one of `segments` workgroups looks at, in whole groups of
// 64 tokens, a run of groups for each wave.
struct Segment {
    int lo, hi, run;  // of the workgroup; tokens of a wave's run
    int p0;           // page index of the first token
};
__device__ __forceinline__ Segment segment_of(const Choice& x, int segment, int segments, int shift) {
    const int base = x.lo & ~63, groups = ((x.hi + 63) >> 6) - (x.lo >> 6);
    const int each = (groups + segments - 1) / segments;
    Segment s;
    const int64_t from = base + int64_t(segment) * each * 64;
    s.lo = int(max(int64_t(x.lo), min(from, int64_t(x.hi))));
    s.hi = int(min(int64_t(x.hi), from + int64_t(each) * 64));
    s.run = (each + kWaves - 1) / kWaves * 64;
    s.p0 = s.lo >> shift;
    return s;
}
// Its page numbers, into LDS.
__device__ __forceinline__ void list_pages(const sparsp_cache& c, SelectLds& l, const Choice& x,
                                           const Segment& s, int shift) {
    const int pages = s.hi > s.lo ? ((s.hi - 1) >> shift) - s.p0 + 1 : 0;
    for (int e = threadIdx.x; e < min(pages, kPages); e += kThreads)
        l.pages[e] = page_of(c.table, c.width, c.pages, x.b, s.p0 + e);
}

// f(token, is there one, its key) for the tokens of the wave's run, 64 at a time in their order.
// WIDE: pages of 64 tokens and more, so 64 tokens are on one page.
template <bool WIDE, typename F>
__device__ __forceinline__ void walk(const sparsp_cache& c, const SelectLds& l, const Choice& x,
                                     const Segment& s, F f) {
    if (s.hi <= s.lo) return;  // (its list of pages is empty)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int shift = __builtin_ctz(c.page);
    const int r0 = (s.lo & ~63) + wave * s.run, r1 = min(s.hi, r0 + s.run);
    auto page_at = [&](int t) {
        const int e = (t >> shift) - s.p0;
        return e < kPages ? l.pages[e] : page_of(c.table, c.width, c.pages, x.b, s.p0 + e);
    };
    for (int t0 = r0; t0 < r1; t0 += 64 * kAhead) {
        float w[kAhead];
        bool page[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            // (groups behind the last are read as the last)
            const int t = min(t0 + 64 * u, (r1 - 1) & ~63);
            const int mine = min(max(t + lane, s.lo), s.hi - 1);
            int p = page_at(WIDE ? max(t, s.lo) : mine);
            if (WIDE) p = __builtin_amdgcn_readfirstlane(p);
            page[u] = p >= 0;
            const float* from = c.weights + (int64_t(max(p, 0)) * c.H + x.h) * c.page;
            w[u] = WIDE ? (from + (t & (c.page - 1)))[lane] : from[mine & (c.page - 1)];
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int t = t0 + 64 * u + lane;
            if (t0 + 64 * u < r1) f(t, t >= s.lo && t < r1, page[u] ? weight_key(w[u]) : 0u);
        }
    }
}

// Writes the kept tokens of the workgroup's segment, those above T and of those equal to T the first
// want - eq_before, to list + at. wave_gt and wave_eq hold what each wave has of both.
template <bool WIDE>
__device__ __forceinline__ void write_kept(const sparsp_cache& c, const SelectLds& l,
                                           const Choice& x, const Segment& s, uint32_t T, int want,
                                           int at, int eq_before, int32_t* list) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int w = 0; w < wave; ++w) {
        at += l.wave_gt[w] + max(0, min(l.wave_eq[w], want - eq_before));
        eq_before += l.wave_eq[w];
    }
    const uint64_t below = (uint64_t(1) << lane) - 1;
    walk<WIDE>(c, l, x, s, [&](int t, bool in, uint32_t k) {
        const uint64_t eqs = __ballot(in && k == T);
        const bool take = in && (k > T || (k == T && eq_before + __popcll(eqs & below) < want));
        const uint64_t takes = __ballot(take);
        if (take) list[at + __popcll(takes & below)] = t;
        at += __popcll(takes);
        eq_before += __popcll(eqs);
    });
}

// What stays without a choice, and the new length: once per (sequence, head).
__device__ __forceinline__ void write_forced(const Choice& x, int keep, int first, int recent,
                                             int32_t* kv_len_out, int32_t* list) {
    const int tid = threadIdx.x;
    if (x.h == 0 && tid == 0) kv_len_out[x.b] = min(x.n, keep);
    if (x.n <= keep) {
        for (int j = tid; j < keep; j += kThreads) list[j] = j < x.n ? j : -1;
        return;
    }
    for (int j = tid; j < first; j += kThreads) list[j] = j;
    for (int j = tid; j < recent; j += kThreads) list[keep - recent + j] = x.n - recent + j;
}

// One workgroup per (sequence, head).
template <bool WIDE>
__global__ __launch_bounds__(kThreads) void select_kernel(const sparsp_cache c, int keep, int first,
                                                          int recent, int32_t* kv_len_out,
                                                          int32_t* kept) {
    __shared__ SelectLds l;
    __shared__ uint32_t held_key[kCandidates];
    __shared__ uint8_t held_wave[kCandidates];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int32_t* list = kept + int64_t(blockIdx.x) * keep;
    Choice x;
    const bool choose = choice_of(c, blockIdx.x, keep, first, recent, &x);
    write_forced(x, keep, first, recent, kv_len_out, list);
    if (!choose) return;
    const int shift = __builtin_ctz(c.page);
    const Segment s = segment_of(x, 0, 1, shift);
    int want = x.want;
    list_pages(c, l, x, s, shift);
    clear_bins(l);
    if (tid == 0) l.candidates = 0;
    if (tid < kWaves) l.wave_gt[tid] = l.wave_eq[tid] = 0;
    __syncthreads();

    walk<WIDE>(c, l, x, s, [&](int, bool in, uint32_t k) {
        if (in) atomicAdd(&l.bins[k >> 21], 1u);
    });
    find_digit(l, 11, want);
    uint32_t T = l.found[0] << 21;
    want -= int(l.found[1]);
    clear_bins(l);
    int gt = 0;
    walk<WIDE>(c, l, x, s, [&](int, bool in, uint32_t k) {
        gt += __popcll(__ballot(in && k >> 21 > T >> 21));
        if (in && k >> 21 == T >> 21) {
            const int at = atomicAdd(&l.candidates, 1);
            if (at < kCandidates) {
                held_key[at] = k;
                held_wave[at] = uint8_t(wave);
            }
        }
    });
    __syncthreads();
    const int candidates = l.candidates;
    const bool held = candidates <= kCandidates;
    for (int pass = 0; pass < 2; ++pass) {
        const int high = pass ? 10 : 21, low = pass ? 0 : 10, bits = high - low;
        auto count = [&](uint32_t k) {
            if (k >> high == T >> high) atomicAdd(&l.bins[(k >> low) & ((1u << bits) - 1)], 1u);
        };
        if (held) {
            for (int e = tid; e < candidates; e += kThreads) count(held_key[e]);
        } else {
            walk<WIDE>(c, l, x, s, [&](int, bool in, uint32_t k) {
                if (in) count(k);
            });
        }
        find_digit(l, bits, want);
        T |= l.found[0] << low;
        want -= int(l.found[1]);
        clear_bins(l);
        __syncthreads();
    }

    if (held) {
        if (lane == 0) atomicAdd(&l.wave_gt[wave], gt);
        for (int e = tid; e < candidates; e += kThreads) {
            if (held_key[e] > T) atomicAdd(&l.wave_gt[held_wave[e]], 1);
            if (held_key[e] == T) atomicAdd(&l.wave_eq[held_wave[e]], 1);
        }
    } else {
        int above = 0, eq = 0;
        walk<WIDE>(c, l, x, s, [&](int, bool in, uint32_t k) {
            above += __popcll(__ballot(in && k > T));
            eq += __popcll(__ballot(in && k == T));
        });
        if (lane == 0) {
            l.wave_gt[wave] = above;
            l.wave_eq[wave] = eq;
        }
    }
    __syncthreads();
    write_kept<WIDE>(c, l, x, s, T, want, first, 0, list);
}

// The same by `segments` workgroups for each (sequence, head), in three launches. Workspace of
// a pair: the segments' counts by first digit [segments][2048], {the first digit of T, keys
// above it}, what a segment has {above the digit, at it} [segments][2], and the keys at it
// [segments][span].
struct SplitSpace {
    uint32_t* bins;
    uint32_t* digit;
    int* counts;
    uint32_t* keys;
    int span;  // keys of a segment at most
};
__host__ __device__ __forceinline__ int64_t split_words(int segments, int64_t span) {
    return segments * (int64_t(kBins) + 2 + span) + 2;
}
__device__ __forceinline__ SplitSpace split_space(uint32_t* ws, int pair, int segments, int span) {
    uint32_t* p = ws + pair * split_words(segments, span);
    uint32_t* digit = p + int64_t(segments) * kBins;
    return {p, digit, reinterpret_cast<int*>(digit + 2), digit + 2 + 2 * segments, span};
}

template <bool WIDE>
__global__ __launch_bounds__(kThreads) void count_kernel(const sparsp_cache c, int keep, int first,
                                                         int recent, int segments, int span,
                                                         uint32_t* ws, int32_t* kv_len_out,
                                                         int32_t* kept) {
    __shared__ SelectLds l;
    const int pair = blockIdx.x / segments, segment = blockIdx.x % segments;
    Choice x;
    const bool choose = choice_of(c, pair, keep, first, recent, &x);
    if (segment == 0)
        write_forced(x, keep, first, recent, kv_len_out, kept + int64_t(pair) * keep);
    if (!choose) return;
    const int shift = __builtin_ctz(c.page);
    const Segment s = segment_of(x, segment, segments, shift);
    list_pages(c, l, x, s, shift);
    clear_bins(l);
    __syncthreads();
    walk<WIDE>(c, l, x, s, [&](int, bool in, uint32_t k) {
        if (in) atomicAdd(&l.bins[k >> 21], 1u);
    });
    __syncthreads();
    const SplitSpace sp = split_space(ws, pair, segments, span);
    for (int e = threadIdx.x; e < kBins; e += kThreads) sp.bins[segment * kBins + e] = l.bins[e];
}

// The first digit of T from the segments' counts, into found.
__device__ __forceinline__ void first_digit(SelectLds& l, const SplitSpace& sp, int segments,
                                            int want) {
    static_assert(kBins == 2 * kThreads);
    const int e = 2 * threadIdx.x;
    u32x2_t sum = {};
    for (int g0 = 0; g0 < segments; g0 += 2 * kAhead) {  // (loads of 16 segments in flight)
        u32x2_t n[2 * kAhead];
#pragma unroll
        for (int u = 0; u < 2 * kAhead; ++u)
            n[u] = *reinterpret_cast<const u32x2_t*>(sp.bins +
                                                     min(g0 + u, segments - 1) * kBins + e);
#pragma unroll
        for (int u = 0; u < 2 * kAhead; ++u)
            if (g0 + u < segments) sum += n[u];
    }
    l.bins[e] = sum.x;
    l.bins[e + 1] = sum.y;
    find_digit(l, 11, want);
}

template <bool WIDE>
__global__ __launch_bounds__(kThreads) void gather_keys_kernel(const sparsp_cache c, int keep,
                                                               int first, int recent, int segments,
                                                               int span, uint32_t* ws) {
    __shared__ SelectLds l;
    const int pair = blockIdx.x / segments, segment = blockIdx.x % segments;
    Choice x;
    if (!choice_of(c, pair, keep, first, recent, &x)) return;
    const int shift = __builtin_ctz(c.page), lane = threadIdx.x & 63;
    const Segment s = segment_of(x, segment, segments, shift);
    list_pages(c, l, x, s, shift);
    if (threadIdx.x == 0) l.candidates = l.wave_gt[0] = 0;
    const SplitSpace sp = split_space(ws, pair, segments, span);
    first_digit(l, sp, segments, x.want);
    const uint32_t digit = l.found[0];
    int gt = 0;
    walk<WIDE>(c, l, x, s, [&](int, bool in, uint32_t k) {
        gt += __popcll(__ballot(in && k >> 21 > digit));
        if (in && k >> 21 == digit) {
            const int at = atomicAdd(&l.candidates, 1);
            sp.keys[int64_t(segment) * span + at] = k;
        }
    });
    if (lane == 0) atomicAdd(&l.wave_gt[0], gt);
    __syncthreads();
    if (threadIdx.x == 0) {
        sp.counts[2 * segment] = l.wave_gt[0];
        sp.counts[2 * segment + 1] = l.candidates;
        if (segment == 0) {
            sp.digit[0] = l.found[0];
            sp.digit[1] = l.found[1];
        }
    }
}

template <bool WIDE>
__global__ __launch_bounds__(kThreads) void place_kernel(const sparsp_cache c, int keep, int first,
                                                         int recent, int segments, int span,
                                                         uint32_t* ws, int32_t* kept) {
    __shared__ SelectLds l;
    __shared__ int before[2];  // kept or equal tokens of the segments before
    const int pair = blockIdx.x / segments, segment = blockIdx.x % segments;
    Choice x;
    if (!choice_of(c, pair, keep, first, recent, &x)) return;
    const int shift = __builtin_ctz(c.page), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Segment s = segment_of(x, segment, segments, shift);
    const SplitSpace sp = split_space(ws, pair, segments, span);
    uint32_t T = sp.digit[0] << 21;
    int want = x.want - int(sp.digit[1]);
    // A wave has the keys of two segments, the first 512 of each in registers, all asked for
    // at once.
    constexpr int OWN = kSegments / kWaves;
    int count[OWN];
    uint32_t key[OWN][kAhead];
#pragma unroll
    for (int j = 0; j < OWN; ++j) {
        const int g = wave + j * kWaves;
        count[j] = g < segments ? sp.counts[2 * g + 1] : 0;
    }
#pragma unroll
    for (int j = 0; j < OWN; ++j)
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            key[j][u] = lane + 64 * u < count[j]
                            ? sp.keys[int64_t(wave + j * kWaves) * span + lane + 64 * u]
                            : 0;
    auto every_key = [&](auto f) {  // f(is it of a segment before, key)
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
            const int g = wave + j * kWaves;
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (lane + 64 * u < count[j]) f(g < segment, key[j][u]);
            for (int e = 64 * kAhead + lane; e < count[j]; e += 64)
                f(g < segment, sp.keys[int64_t(g) * span + e]);
        }
    };
    list_pages(c, l, x, s, shift);
    clear_bins(l);
    __syncthreads();
    for (int pass = 0; pass < 2; ++pass) {
        const int high = pass ? 10 : 21, low = pass ? 0 : 10, bits = high - low;
        every_key([&](bool, uint32_t k) {
            if (k >> high == T >> high) atomicAdd(&l.bins[(k >> low) & ((1u << bits) - 1)], 1u);
        });
        find_digit(l, bits, want);
        T |= l.found[0] << low;
        want -= int(l.found[1]);
        clear_bins(l);
        __syncthreads();
    }
    if (threadIdx.x < 2) before[threadIdx.x] = 0;
    __syncthreads();
    every_key([&](bool earlier, uint32_t k) {
        if (earlier && k > T) atomicAdd(&before[0], 1);
        if (earlier && k == T) atomicAdd(&before[1], 1);
    });
    if (int(threadIdx.x) < segment) atomicAdd(&before[0], sp.counts[2 * threadIdx.x]);
    int above = 0, eq = 0;
    walk<WIDE>(c, l, x, s, [&](int, bool in, uint32_t k) {
        above += __popcll(__ballot(in && k > T));
        eq += __popcll(__ballot(in && k == T));
    });
    if (lane == 0) {
        l.wave_gt[wave] = above;
        l.wave_eq[wave] = eq;
    }
    __syncthreads();
    write_kept<WIDE>(c, l, x, s, T, want, first + before[0] + min(before[1], want), before[1],
                     kept + int64_t(pair) * keep);
}

constexpr int kSlice = 128;  // bytes of a row that a workgroup moves in place
constexpr int kDeep = 4;     // accesses of a thread in flight

// Grid: (sequence, head) x (K slices, V slices) x chunk workgroups (one in place). A row's slice
// is moved by `lanes` threads, a power of two.
template <bool INSIDE>
__global__ __launch_bounds__(kThreads) void move_kernel(const sparsp_cache c, int keep,
                                                        const int32_t* kept,
                                                        const int32_t* dst_table, int dst_width,
                                                        int slices, int lanes, int chunk_groups,
                                                        int row_bytes) {
    const int group = blockIdx.x % chunk_groups;
    const int piece = blockIdx.x / chunk_groups % (2 * slices);
    const int bh = blockIdx.x / chunk_groups / (2 * slices);
    const int b = bh / c.H, h = bh % c.H;
    const int32_t* to_table = INSIDE ? c.table : dst_table;
    const int to_width = INSIDE ? c.width : dst_width;
    const int n = cached_tokens(c, b);
    if (INSIDE && n <= keep) return;
    const int count = min(n, keep);
    char* base = static_cast<char*>(piece < slices ? c.K : c.V);
    const int lane_shift = __builtin_ctz(lanes), in_row = int(threadIdx.x) & (lanes - 1);
    const int rows = kThreads >> lane_shift, chunk = rows * kDeep;
    const int at = (piece % slices) * kSlice + in_row * 16;
    const bool mine = at < row_bytes;
    const bool weights = piece == 0 && in_row == 0;
    const int shift = __builtin_ctz(c.page), mask = c.page - 1;
    const int32_t* list = kept + int64_t(bh) * keep;
    // Three chunks at once, so that each waits once: the rows of this one are loaded beside the
    // page numbers of the next one and the list of the one after (24 sequences of 2,900 to 6,007
    // tokens: 142 us with three waits for a chunk, 130 us).
    const int step = chunk_groups * chunk, row0 = int(threadIdx.x) >> lane_shift;
    int t[kDeep], p[kDeep], q[kDeep];
    auto listed = [&](int j0, int u) {
        const int j = j0 + u * rows + row0;
        return j < count ? list[j] : -1;
    };
    auto source = [&](int u) {
        return t[u] < 0 ? -1 : page_of(c.table, c.width, c.pages, b, t[u] >> shift);
    };
    auto target = [&](int j0, int u) {
        const int j = j0 + u * rows + row0;
        return j < count ? page_of(to_table, to_width, c.pages, b, j >> shift) : -1;
    };
    int j0 = group * chunk;
#pragma unroll
    for (int u = 0; u < kDeep; ++u) t[u] = listed(j0, u);
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
        p[u] = source(u);
        q[u] = target(j0, u);
    }
    int next[kDeep];
#pragma unroll
    for (int u = 0; u < kDeep; ++u) next[u] = listed(j0 + step, u);
    for (; j0 < count; j0 += step) {
        u32x4_t x[kDeep];
        float w[kDeep];
        int64_t to[kDeep];
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            const int j = j0 + u * rows + row0;
            to[u] = -1;
            x[u] = u32x4_t{};
            w[u] = 0.f;
            const bool moves = p[u] >= 0 && q[u] >= 0 && !(INSIDE && t[u] == j);
            const int64_t from = (int64_t(p[u]) * c.H + h) * c.page + (t[u] & mask);
            if (moves) {
                to[u] = (int64_t(q[u]) * c.H + h) * c.page + (j & mask);
                if (mine) x[u] = *reinterpret_cast<const u32x4_t*>(base + from * row_bytes + at);
                if (weights) w[u] = c.weights[from];
            }
        }
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            t[u] = next[u];
            p[u] = source(u);
            q[u] = target(j0 + step, u);
        }
#pragma unroll
        for (int u = 0; u < kDeep; ++u) next[u] = listed(j0 + 2 * step, u);
        if (INSIDE) {
            // Every row of the chunk is in registers before any is overwritten.
            __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < kDeep; ++u) {
            if (to[u] < 0) continue;
            if (mine) store_nt(base + to[u] * row_bytes + at, __builtin_bit_cast(uint4, x[u]));
            if (weights) c.weights[to[u]] = w[u];
        }
        // The chunks after this one read only places behind it.
    }
}

}  // namespace

namespace {

// Workgroups for each (sequence, head): one where there are many pairs or the sequences cannot be
// long (one workgroup takes 17 us for 6,007 tokens and 116 us for 100,003, bound by its own
// instructions), else as many as fill half the GPU, with 4,096 tokens each and more.
int segments_of(const sparsp_cache& c) {
    const int64_t tokens = int64_t(c.width) * c.page, pairs = int64_t(c.B) * c.H;
    if (tokens <= 16384 || pairs > 64) return 1;
    return int(std::min<int64_t>({kSegments, 128 / pairs, tokens / 4096}));
}
int64_t segment_span(const sparsp_cache& c, int segments) {
    const int64_t groups = int64_t(c.width) * c.page / 64 + 2;
    return (groups + segments - 1) / segments * 64;
}

template <bool WIDE>
hipError_t launch_select(const sparsp_cache& c, int keep, int first, int recent, int32_t* kv_len_out,
                         int32_t* kept, void* ws, int64_t ws_bytes, hipStream_t s) {
    const int pairs = c.B * c.H, segments = segments_of(c);
    if (segments == 1 || !ws || ws_bytes < evict_workspace(c)) {
        select_kernel<WIDE><<<pairs, kThreads, 0, s>>>(c, keep, first, recent, kv_len_out, kept);
        return hipGetLastError();
    }
    const int span = int(segment_span(c, segments)), grid = pairs * segments;
    uint32_t* w = static_cast<uint32_t*>(ws);
    count_kernel<WIDE><<<grid, kThreads, 0, s>>>(c, keep, first, recent, segments, span, w,
                                                 kv_len_out, kept);
    gather_keys_kernel<WIDE><<<grid, kThreads, 0, s>>>(c, keep, first, recent, segments, span, w);
    place_kernel<WIDE><<<grid, kThreads, 0, s>>>(c, keep, first, recent, segments, span, w, kept);
    return hipGetLastError();
}

}  // namespace

int64_t evict_workspace(const sparsp_cache& c) {
    const int segments = segments_of(c);
    if (segments == 1) return 0;
    return int64_t(c.B) * c.H * split_words(segments, segment_span(c, segments)) * 4;
}

hipError_t launch_cache_evict(const sparsp_cache& c, int keep, int first, int recent,
                              const int32_t* dst_table, int dst_width, int32_t* kv_len_out,
                              int32_t* kept, void* ws, int64_t ws_bytes, hipStream_t s) {
    if (hipError_t e = c.page >= 64 ? launch_select<true>(c, keep, first, recent, kv_len_out, kept,
                                                          ws, ws_bytes, s)
                                    : launch_select<false>(c, keep, first, recent, kv_len_out, kept,
                                                           ws, ws_bytes, s);
        e != hipSuccess)
        return e;
    const int row_bytes = c.d * (c.dtype == SPARSP_BF16 ? 2 : 4);
    // (many pairs are work enough, and more workgroups would pass the size of a grid)
    const bool whole = dst_table || row_bytes < kSlice || c.B * c.H >= 1024;
    const int part = whole ? row_bytes : kSlice;
    const int slices = (row_bytes + part - 1) / part;
    int lanes = 1;
    while (lanes * 16 < part) lanes *= 2;
    const int64_t pieces = int64_t(c.B) * c.H * 2 * slices;
    if (!dst_table) {
        move_kernel<true><<<int(pieces), kThreads, 0, s>>>(c, keep, kept, nullptr, 0, slices, lanes,
                                                           1, row_bytes);
        return hipGetLastError();
    }
    const int chunk = kThreads / lanes * kDeep;
    const int64_t most = (keep + chunk - 1) / chunk;
    const int groups = int(std::max<int64_t>(1, std::min<int64_t>(most, 8192 / pieces)));
    move_kernel<false><<<int(pieces * groups), kThreads, 0, s>>>(c, keep, kept, dst_table, dst_width,
                                                                 slices, lanes, groups, row_bytes);
    return hipGetLastError();
}

}  // namespace sparsp
