// Pages of a cache shared, taken, given back, copied and moved together.
//
// refs[p] counts the table entries (and other holders) of page p; a page with none (or fewer) is
// free. Whatever takes pages takes the lowest free ones, in the order of the entries that want them,
// so that results depend on the arguments alone; the counts are changed by integer atomics, whose
// order does not matter.
//
// The tables are small: what bounds these kernels is latency, so they are few, and one workgroup does
// what one can. take_kernel ranks up to 65,536 pages and 1,024 sequences by scans, a thread 16 to 64
// pages in a row. For more of either, count_kernel's sums of each chunk go before, list_kernel lists
// the pages that are taken, and give_kernel's workgroups give them to a chunk of sequences each. (One
// new page each, a tenth of the pages free; one workgroup and several: 256 sequences, 16,000 pages 6.2
// and 13.3 us; 1,024, 60,000 12.4 and 15.9; 4,000, 60,000 25 and 17; 4,000 of a million 18 us.)
// Contents move in units of 16 KB, dealt to a grid that does not know how many there are (a cache of
// 1.7 GB of which a quarter moves: 158 us, 5.4 TB/s read and written).
#include <algorithm>

#include "cache_device.h"

namespace sparsp {
namespace {

constexpr int kTake = 1024;       // threads of a taking workgroup, and sequences of a chunk
constexpr int kEach = 16;         // pages of a thread and chunk
constexpr int kChunk = kTake * kEach;
constexpr int kAlone = 4;         // chunks that one workgroup takes from
constexpr int kUnit = kPageUnit;  // bytes of a copying workgroup's turn

// Sum of x over the threads before this one; *all: over all. N threads.
template <int N>
__device__ __forceinline__ int scan(int x, int* lds, int* all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int sum = x;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(sum, off);
        if (lane >= off) sum += y;
    }
    __syncthreads();  // the scan before has been read
    if (lane == 63) lds[wave] = sum;
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < N / 64; ++w) {
        const int y = lds[w];
        before += w < wave ? y : 0;
        total += y;
    }
    *all = total;
    return before + sum - x;
}

__device__ __forceinline__ int tokens_of(const PageArgs& a, int b) {
    return min(max(a.kv_len[b], 0), a.width * a.page);
}
__device__ __forceinline__ bool named(const PageArgs& a, int page) {
    return page >= 0 && page < a.pages;
}

// The entries of row b that may want a page.
struct Range {
    int begin, count;
};
__device__ __forceinline__ Range range_of(const PageArgs& a, int b) {
    if (b >= a.rows) return {0, 0};
    const int shift = __builtin_ctz(a.page);
    if (a.from)  // a fork: the last, partly filled page of a row that has to copy it
        return {(a.kv_out[b] - 1) >> shift, a.from[b] >= 0 ? 1 : 0};
    const int kv = tokens_of(a, b);
    const int n = min(max(a.new_off[b + 1], 0), 1 << 30) - min(max(a.new_off[b], 0), 1 << 30);
    const int begin = max(kv - n, 0) >> shift;
    return {begin, n > 0 ? ((kv + a.page - 1) >> shift) - begin : 0};
}

struct Lds {
    int sums[kTake / 64];
    int upto[kTake];  // of the chunk's sequences, the entries before the end of each
    int begin[kTake];
};

// Calls give(row, entry, rank) for the wanting entries of the 1,024 sequences from b0 on, rank
// counted from `rank`; returns how many there are. All threads.
template <typename Give>
__device__ __forceinline__ int each_want(const PageArgs& a, int b0, int rank, Lds& l, Give give) {
    const int t = threadIdx.x;
    const Range r = range_of(a, b0 + t);
    int all;
    const int before = scan<kTake>(r.count, l.sums, &all);
    l.upto[t] = before + r.count;
    l.begin[t] = r.begin - before;
    __syncthreads();
    int found = 0;
    for (int e0 = 0; e0 < all; e0 += kTake) {
        const int e = e0 + t;
        int s = 0, j = 0;
        bool want = e < all;
        if (want) {
#pragma unroll
            for (int step = kTake / 2; step; step >>= 1)
                if (l.upto[s + step - 1] <= e) s += step;
            j = l.begin[s] + e;
            want = a.from || !named(a, a.table[int64_t(b0 + s) * a.width + j]);
        }
        int sum;
        const int mine = scan<kTake>(want, l.sums, &sum);
        if (want) give(b0 + s, j, rank + found + mine);
        found += sum;
    }
    __syncthreads();  // upto and begin have been read
    return found;
}

// Four numbers of x from 4 i on, of `count` in all; `fill` behind them.
__device__ __forceinline__ int4 four_of(const int32_t* x, int i, int count, int fill) {
    const int at = 4 * i;
    if (at + 4 <= count && (reinterpret_cast<uintptr_t>(x) & 15) == 0)
        return *reinterpret_cast<const int4*>(x + at);
    return make_int4(at < count ? x[at] : fill, at + 1 < count ? x[at + 1] : fill,
                     at + 2 < count ? x[at + 2] : fill, at + 3 < count ? x[at + 3] : fill);
}

// The pages of a workgroup, kTake * N * kEach from `base` on: which of them are free (or in use), as
// bits of the thread that has N * kEach in a row. They are loaded four a thread as they lie (the
// sixteen of a thread at once would be as many cache lines a load as it has lanes: 31,000 pages and
// what a fork copies from, 21 us) and change hands in LDS.
template <int N>
struct PageBits {
    uint8_t quads[kTake * N * kEach / 4];
};
template <int N, typename Test>
__device__ __forceinline__ uint64_t page_bits(PageBits<N>& lds, int base, Test test) {
    const int t = threadIdx.x;
#pragma unroll
    for (int k = 0; k < N * kEach / 4; ++k) lds.quads[k * kTake + t] = test(base / 4 + k * kTake + t);
    __syncthreads();
    uint64_t bits = 0;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        uint32_t q = reinterpret_cast<const uint32_t*>(lds.quads)[t * N + n];  // a nibble a byte
        q = (q | q >> 4) & 0x00ff00ffu;
        bits |= uint64_t((q | q >> 8) & 0xffffu) << (n * kEach);
    }
    return bits;
}
// Free ones. What a fork copies from is not, though all that held it may have gone; what only rows that
// end have held is, so that a fork needs no more pages than the new rows.
template <int N>
__device__ __forceinline__ uint64_t free_pages(const PageArgs& a, PageBits<N>& lds, int base) {
    return page_bits<N>(lds, base, [&](int i) {
        const int4 x = four_of(a.refs, i, a.pages, 1);
        int free = (x.x <= 0) | (x.y <= 0) << 1 | (x.z <= 0) << 2 | (x.w <= 0) << 3;
        if (a.from) {
            const int4 y = four_of(a.to, i, a.pages, 0);
            free &= (y.x == 0) | (y.y == 0) << 1 | (y.z == 0) << 2 | (y.w == 0) << 3;
        }
        return uint8_t(free);
    });
}

// Free pages of each chunk, and behind them wanting entries of each chunk of sequences.
__global__ __launch_bounds__(kTake) void count_kernel(const PageArgs a, int chunks) {
    __shared__ Lds l;
    __shared__ PageBits<1> pages;
    const int c = blockIdx.x;
    int all;
    if (c < chunks)
        scan<kTake>(__popcll(free_pages<1>(a, pages, c * kChunk)), l.sums, &all);
    else
        all = each_want(a, (c - chunks) * kTake, 0, l, [](int, int, int) {});
    if (threadIdx.x == 0) a.counts[c] = all;
}

// Entry j of row b gets the page of its rank.
__device__ __forceinline__ void give_page(const PageArgs& a, int b, int j, int rank, int page) {
    a.table[int64_t(b) * a.width + j] = page;
    if (a.from) {
        a.src[rank] = a.from[b];
        a.dst[rank] = page;
    }
}

// The number of x's set bit that has k others below it.
__device__ __forceinline__ int bit_of(uint64_t x, int k) {
    int at = 0;
#pragma unroll
    for (int w = 32; w; w >>= 1) {
        const int below = __popcll(x >> at & ((uint64_t(1) << w) - 1));
        if (k >= below) {
            k -= below;
            at += w;
        }
    }
    return at;
}

// All of it by one workgroup, of N chunks of pages. An entry finds its page by its rank among the
// threads' free pages, so nothing is listed.
template <int N>
__global__ __launch_bounds__(kTake) void take_kernel(const PageArgs a) {
    __shared__ Lds l;
    __shared__ PageBits<N> pages;
    __shared__ uint64_t free[kTake];
    __shared__ int upto[kTake];
    const int t = threadIdx.x;
    const uint64_t bits = free_pages<N>(a, pages, 0);
    int all;
    const int rank = scan<kTake>(__popcll(bits), l.sums, &all);
    free[t] = bits;
    upto[t] = rank + __popcll(bits);
    // (each_want begins with a barrier)
    const int wants = each_want(a, 0, 0, l, [&](int b, int j, int r) {
        if (r >= all) return;
        int s = 0;
#pragma unroll
        for (int step = kTake / 2; step; step >>= 1)
            if (upto[s + step - 1] <= r) s += step;
        const uint64_t x = free[s];
        const int page = s * N * kEach + bit_of(x, r - upto[s] + __popcll(x));
        a.refs[page] = 1;
        give_page(a, b, j, r, page);
    });
    if (t == 0) {
        *a.left = all - wants;
        if (a.moves) *a.moves = min(all, wants);
    }
}

// The same in two steps for more: the free pages that are taken, in their order, and then each chunk
// of sequences its own of them. (Not in one, with each chunk of pages looking for the entries that
// want it: it would meet entries that others have filled already.)
__global__ __launch_bounds__(kTake) void list_kernel(const PageArgs a, int chunks, int groups) {
    __shared__ int sums[kTake / 64];
    __shared__ PageBits<1> pages;
    const int t = threadIdx.x, c = blockIdx.x;
    int x = 0, y = 0, z = 0, before, all, wants, mine;
    for (int k = t; k < chunks; k += kTake) {
        const int n = a.counts[k];
        x += k < c ? n : 0;
        y += n;
    }
    for (int k = t; k < groups; k += kTake) z += a.counts[chunks + k];
    scan<kTake>(x, sums, &before);
    scan<kTake>(y, sums, &all);
    scan<kTake>(z, sums, &wants);
    if (c == 0 && t == 0) {
        *a.left = all - wants;
        if (a.moves) *a.moves = min(all, wants);
    }
    if (before >= wants) return;
    const int first = c * kChunk + t * kEach;
    const uint32_t bits = uint32_t(free_pages<1>(a, pages, c * kChunk));
    int r = before + scan<kTake>(__popc(bits), sums, &mine);
    for (uint32_t m = bits; m && r < wants; m &= m - 1, ++r) {
        const int page = first + __builtin_ctz(m);
        a.dst[r] = page;
        a.refs[page] = 1;
    }
}
__global__ __launch_bounds__(kTake) void give_kernel(const PageArgs a, int chunks) {
    __shared__ Lds l;
    const int t = threadIdx.x, g = blockIdx.x;
    int x = 0, y = 0, rank, all;
    for (int k = t; k < chunks; k += kTake) y += a.counts[k];
    for (int k = t; k < g; k += kTake) x += a.counts[chunks + k];
    scan<kTake>(x, l.sums, &rank);
    scan<kTake>(y, l.sums, &all);
    each_want(a, g * kTake, rank, l, [&](int b, int j, int r) {
        if (r < all) give_page(a, b, j, r, a.dst[r]);
    });
}

hipError_t take(const PageArgs& a, hipStream_t s) {
    const int chunks = (a.pages + kChunk - 1) / kChunk, groups = (a.rows + kTake - 1) / kTake;
    if (chunks <= kAlone && groups == 1) {
        const auto kernel = chunks == 1 ? take_kernel<1> : chunks == 2 ? take_kernel<2> : take_kernel<4>;
        kernel<<<1, kTake, 0, s>>>(a);
        return hipGetLastError();
    }
    count_kernel<<<chunks + groups, kTake, 0, s>>>(a, chunks);
    list_kernel<<<chunks, kTake, 0, s>>>(a, chunks, groups);
    give_kernel<<<groups, kTake, 0, s>>>(a, chunks);
    return hipGetLastError();
}

// Entries whose pages no later token sees are given back.
__global__ __launch_bounds__(256) void release_kernel(const PageArgs a, int per_row) {
    const int b = blockIdx.x / per_row;
    const int kv = tokens_of(a, b);
    for (int j = blockIdx.x % per_row * 256 + threadIdx.x; j < a.width; j += per_row * 256) {
        const int64_t begin = int64_t(j) * a.page;
        const bool slid = a.window > 0 && begin >= a.sinks &&
                          begin + a.page <= int64_t(kv) - a.window + 1;
        if (begin < kv && !slid) continue;
        int32_t* at = a.table + int64_t(b) * a.width + j;
        const int page = *at;
        if (named(a, page)) atomicSub(a.refs + page, 1);
        *at = -1;
    }
}

// The rows of the new table; and the counts as they were, for fork_counts_kernel to change.
__global__ __launch_bounds__(256) void fork_rows_kernel(const PageArgs a) {
    const int i = blockIdx.x, t = threadIdx.x;
    if (i >= a.rows) {
        const int at = (i - a.rows) * 1024 + t * 4;
        for (int e = at; e < min(at + 4, a.pages); ++e) {
            a.refs[e] = a.old_refs[e];
            a.to[e] = 0;
        }
        return;
    }
    const int p = a.parents[i];
    const bool live = p >= 0 && p < a.old_rows;
    const int kv = live ? tokens_of(a, p) : 0;
    const int need = (kv + a.page - 1) / a.page;
    bool other = false;  // an earlier row continues the same one
    for (int k = t; k < i; k += 256) other |= a.parents[k] == p;
    other = __syncthreads_or(other);
    const int32_t* old = a.old_table + int64_t(live ? p : 0) * a.width;
    for (int j = t; j < a.width; j += 256) {
        int page = j < need ? old[j] : -1;
        if (!named(a, page)) page = -1;
        if (j == need - 1) {
            // A page that is not full goes to the first row, if nothing else holds it.
            const bool copy = page >= 0 && kv % a.page && (other || a.old_refs[page] != 1);
            a.from[i] = copy ? page : -1;
            if (copy) page = -1;
        }
        a.table[int64_t(i) * a.width + j] = page;
    }
    if (t == 0) {
        a.kv_out[i] = kv;
        if (need == 0) a.from[i] = -1;
    }
}

// What each old row's entries come to: one for each row that continues it, less its own.
__global__ __launch_bounds__(256) void fork_counts_kernel(const PageArgs a) {
    __shared__ int sums[4];
    const int p = blockIdx.x, t = threadIdx.x;
    int children = 0;
    for (int k = t; k < a.rows; k += 256) children += a.parents[k] == p;
    scan<256>(children, sums, &children);
    const int kv = tokens_of(a, p);
    for (int j = t; j < a.width; j += 256) {
        const int page = a.old_table[int64_t(p) * a.width + j];
        if (!named(a, page)) continue;
        const int64_t begin = int64_t(j) * a.page;
        int delta = -1;
        if (begin + a.page <= kv)
            delta = children - 1;
        else if (begin < kv && children > 0) {
            if (a.old_refs[page] == 1)
                delta = 0;
            else
                a.to[page] = 1;  // copied for every row
        }
        if (delta) atomicAdd(a.refs + page, delta);
    }
}

// One unit of the pages' contents: 16 KB of page `src` of one buffer to page `dst`.
__device__ __forceinline__ void copy_unit(const PageBuffers& f, int src, int dst, int u) {
    int n = 0;
    while (n + 1 < f.count && u >= f.first[n + 1]) ++n;
    const int64_t bytes = f.bytes[n], at = int64_t(u - f.first[n]) * kUnit;
    const char* from = f.data[n] + src * bytes + at;
    char* to = f.data[n] + dst * bytes + at;
    uint4 x[kUnit / 4096];
#pragma unroll
    for (int k = 0; k < kUnit / 4096; ++k) {
        const int off = k * 4096 + threadIdx.x * 16;
        if (at + off < bytes) x[k] = load_nt(from + off);
    }
#pragma unroll
    for (int k = 0; k < kUnit / 4096; ++k) {
        const int off = k * 4096 + threadIdx.x * 16;
        if (at + off < bytes) store_nt(to + off, x[k]);
    }
}

// Pages src[k] to dst[k], k below *moves (or `most`, where that is NULL).
__global__ __launch_bounds__(256) void copy_kernel(const PageBuffers f, const int32_t* src,
                                                   const int32_t* dst, const int32_t* moves, int most,
                                                   int pages) {
    const int64_t units = int64_t(moves ? *moves : most) * f.units;
    for (int64_t w = blockIdx.x; w < units; w += gridDim.x) {
        const int k = int(w / f.units);
        const int s = src[k], d = dst[k];
        if (s < 0 || s >= pages || d < 0 || d >= pages || s == d) continue;
        copy_unit(f, s, d, int(w % f.units));
    }
}

__device__ __forceinline__ uint8_t in_use(int4 x) {
    return uint8_t((x.x > 0) | (x.y > 0) << 1 | (x.z > 0) << 2 | (x.w > 0) << 3);
}
__global__ __launch_bounds__(kTake) void used_kernel(const PageArgs a) {
    __shared__ int sums[kTake / 64];
    int used = 0, all;
#pragma unroll
    for (int k = 0; k < kEach / 4; ++k)
        used += __popc(in_use(four_of(
            a.old_refs, blockIdx.x * (kChunk / 4) + k * kTake + threadIdx.x, a.pages, 0)));
    scan<kTake>(used, sums, &all);
    if (threadIdx.x == 0) a.counts[blockIdx.x] = all;
}

// With n pages in use, the k-th page in use from n on goes to the k-th free one below n: dst[k]. Of
// the pages in use from n on, src counts from the last, since that needs no count of those below n;
// to[page] is that number. *moves is how many there are. The counts of the pages below n that stay.
__global__ __launch_bounds__(kTake) void compact_kernel(const PageArgs a, int chunks) {
    __shared__ int sums[kTake / 64];
    __shared__ PageBits<1> pages;
    const int t = threadIdx.x, c = blockIdx.x, first = c * kChunk + t * kEach;
    int4 refs[kEach / 4];
#pragma unroll
    for (int k = 0; k < kEach / 4; ++k)
        refs[k] = four_of(a.old_refs, c * (kChunk / 4) + k * kTake + t, a.pages, 0);
    const uint32_t used = uint32_t(page_bits<1>(
        pages, 0, [&](int i) { return in_use(refs[i / kTake]); }));
    int mine, before = 0;
    int rank = scan<kTake>(__popc(used), sums, &mine);
    int n = mine;
    if (chunks > 1) {
        int x = 0, y = 0;
        for (int k = t; k < chunks; k += kTake) {
            const int m = a.counts[k];
            x += k < c ? m : 0;
            y += m;
        }
        scan<kTake>(x, sums, &before);
        scan<kTake>(y, sums, &n);
    }
    rank += before;  // pages in use before this thread's
    if (c == 0 && t == 0) {
        *a.left = n;
        if (n == a.pages) *a.moves = 0;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int p = first + i;
        const bool u = used >> i & 1;
        if (p == n && p < a.pages) *a.moves = n - rank;
        if (p < n) {
            if (!u) a.dst[p - rank] = p;
        } else if (u) {
            a.src[n - 1 - rank] = p;
            a.to[p] = n - 1 - rank;
        }
        rank += u;
    }
    // (free pages below n get their counts with their contents; until then any)
#pragma unroll
    for (int k = 0; k < kEach / 4; ++k) {
        const int at = 4 * (c * (kChunk / 4) + k * kTake + t);
        const int4 x = refs[k];
        const int y[4] = {at < n ? x.x : 0, at + 1 < n ? x.y : 0, at + 2 < n ? x.z : 0,
                          at + 3 < n ? x.w : 0};
        if (at + 4 <= a.pages && (reinterpret_cast<uintptr_t>(a.refs) & 15) == 0) {
            *reinterpret_cast<int4*>(a.refs + at) = make_int4(y[0], y[1], y[2], y[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (at + i < a.pages) a.refs[at + i] = y[i];
        }
    }
}

// The first workgroups rewrite the table, the others move contents and counts.
__global__ __launch_bounds__(256) void compact_move_kernel(const PageArgs a, const PageBuffers f,
                                                           int tables) {
    const int moves = *a.moves, n = *a.left;
    if (int(blockIdx.x) < tables) {
        const int64_t entries = int64_t(a.rows) * a.width;
        for (int64_t e = blockIdx.x * 256 + threadIdx.x; e < entries; e += tables * 256) {
            int page = a.old_table[e];
            if (!named(a, page) || a.old_refs[page] <= 0)
                page = -1;
            else if (page >= n)
                page = a.dst[moves - 1 - a.to[page]];
            a.table[e] = page;
        }
        return;
    }
    const int each = max(f.units, 1);  // (no contents: the counts alone)
    const int64_t units = int64_t(moves) * each;
    for (int64_t w = blockIdx.x - tables; w < units; w += gridDim.x - tables) {
        const int k = int(w / each), u = int(w % each);
        const int src = a.src[moves - 1 - k], dst = a.dst[k];
        if (u == 0 && threadIdx.x == 0) a.refs[dst] = a.old_refs[src];
        if (f.units > 0) copy_unit(f, src, dst, u);
    }
}

int copy_grid(int64_t units) {
    return int(std::min<int64_t>(std::max<int64_t>(units, 1), 8 * 256));
}

}  // namespace

hipError_t launch_pages_reserve(const PageArgs& a, hipStream_t s) { return take(a, s); }

hipError_t launch_pages_release(const PageArgs& a, hipStream_t s) {
    const int per_row = std::min((a.width + 255) / 256, 16);
    release_kernel<<<a.rows * per_row, 256, 0, s>>>(a, per_row);
    return hipGetLastError();
}

hipError_t launch_pages_fork(const PageArgs& a, const PageBuffers& f, hipStream_t s) {
    fork_rows_kernel<<<a.rows + (a.pages + 1023) / 1024, 256, 0, s>>>(a);
    fork_counts_kernel<<<a.old_rows, 256, 0, s>>>(a);
    const hipError_t e = take(a, s);
    if (e != hipSuccess || f.count == 0) return e;
    copy_kernel<<<copy_grid(int64_t(a.rows) * f.units), 256, 0, s>>>(f, a.src, a.dst, a.moves, 0,
                                                                     a.pages);
    return hipGetLastError();
}

hipError_t launch_pages_copy(const PageBuffers& f, const int32_t* src, const int32_t* dst, int count,
                             int pages, hipStream_t s) {
    copy_kernel<<<copy_grid(int64_t(count) * f.units), 256, 0, s>>>(f, src, dst, nullptr, count, pages);
    return hipGetLastError();
}

hipError_t launch_pages_compact(const PageArgs& a, const PageBuffers& f, hipStream_t s) {
    const int chunks = (a.pages + kChunk - 1) / kChunk;
    if (chunks > 1) used_kernel<<<chunks, kTake, 0, s>>>(a);
    compact_kernel<<<chunks, kTake, 0, s>>>(a, chunks);
    const int tables = int(std::min<int64_t>((int64_t(a.rows) * a.width + 255) / 256, 256));
    compact_move_kernel<<<tables + copy_grid(int64_t(a.pages / 2) * std::max(f.units, 1)), 256, 0, s>>>(
        a, f, tables);
    return hipGetLastError();
}

}  // namespace sparsp
