// Attention weight per cached token: w[t] = sum over the rows that see t of
// exp(scale q.k_t - lse). A row is (token, head of the group). No two waves add to the same
// weight, so there are no atomics and the order of a sum depends on the sizes alone.
//
// weights_rows_kernel, for up to 32 rows a sequence (a decoding step): Q and lse stay in
// registers, the workgroup walks a part of the sequence's keys, and what bounds it is reading
// K. Its waves take the tiles of S^T = K Q^T (paged_tiles.h) in turn, the next one loading
// while one is computed; each lane sums the exponentials of its keys over its columns of
// rows, and the sixteen lanes that hold a key's columns are added in a rotation.
// 64 sequences of 9,000 tokens: 5.3 TB/s, and 4.85 TB/s with a wave per tile and no next one;
// 64 of 400 to 9,001: 82, 78, 77 and 80 us in parts for 8, 16, 32 and 64 workgroups per CU.
//
// weights_keys_kernel, for more rows, float32 or few keys: a wave's keys stay in registers and it
// walks the rows, 16 at a time, the next ones loading while some are computed. The rows
// come from cache; float32 is bound by the matrix pipe. SPLIT shares the rows out to the four
// waves instead of the keys: four times the workgroups. bf16 does so where that makes up to two
// workgroups a CU, and goes to paged_weights_tiles.hip otherwise (32 heads of 128, 2,000 tokens
// over as many: 91 us, 178 us by its 64 workgroups; 1,000 over 4,000: 78 and 100 us; 16 heads
// of 4 sequences, 1,000 over 1,000, four a CU: 45 and 32 us). float32 does where the keys do not
// fill the GPU, and for 2,048 rows and more, whose tail it evens out (32 heads, 300 tokens over
// 300: 26 us, 76 us; 2,000 over 2,000: 373 and 511 us; 64 over 8,000: 87 and 80 us).
#include <algorithm>

#include "paged_tiles.h"

namespace sparsp {
namespace {

constexpr int kCus = 256;
constexpr int kSegment = 16384;  // keys whose page numbers are held at once

// Sum over the 16 lanes of a group, the same in all of them.
__device__ __forceinline__ float group_sum(float x) {
#define SPARSP_ROW_ROR(n) \
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + n, 0xf, 0xf, false))
    SPARSP_ROW_ROR(8);
    SPARSP_ROW_ROR(4);
    SPARSP_ROW_ROR(2);
    SPARSP_ROW_ROR(1);
#undef SPARSP_ROW_ROR
    return x;
}

// A row's place in Q, its lse in log2 units and the end of the keys it sees (0: none).
struct Row {
    int64_t at;
    float lse2;
    int limit;
};
__device__ __forceinline__ Row row_of(const PagedArgs& a, const Seq& s, int hk, int G, int r) {
    Row x = {0, 0.f, 0};
    if (r < s.n * G) {
        const int i = r / G, h = hk * G + r % G;
        const float lse = a.lse_in[int64_t(h) * a.tokens + s.q0 + i];
        x.at = int64_t(h) * a.q_head + int64_t(s.q0 + i) * a.q_token;
        x.lse2 = lse * kLog2e;
        x.limit = lse == -INFINITY ? 0 : a.causal ? min(s.kv, s.kv - s.n + i + 1) : s.kv;
    }
    return x;
}

template <typename T, int D, int NC>
__global__ __launch_bounds__(256) void weights_rows_kernel(const PagedArgs a, const PagedPlan plan) {
    using M = TileMath<T, D>;
    constexpr int KEYS = M::KEYS, JUMP = 4 * KEYS;
    __shared__ int page_list[kSegment / 16];
    const sparsp_cache& c = a.cache;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = lane & 15, g = lane >> 4;
    const auto [bh, part] = unit_of(blockIdx.x, c.B * c.H);
    const int b = bh / c.H, hk = bh % c.H;
    const int G = a.q_heads / c.H;
    const Seq s = sequence(c, a.tokens, b);
    const int keys = part_keys(plan, s.kv);
    if (part * int64_t(keys) >= s.kv) return;
    const int lo = part * keys, end = min(s.kv - lo, keys) + lo;
    const float c2 = a.scale * kLog2e;
    const int shift = __builtin_ctz(c.page), mask = c.page - 1;

    // Rows beyond the registers (the caller's max_new was too small) take further rounds, which
    // add to what the first has written.
    for (int r0 = 0; r0 == 0 || r0 < s.n * G; r0 += 16 * NC) {
        const bool add = a.accumulate || r0 > 0;
        typename M::QTile q[NC];
        Row row[NC];
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            const int r = r0 + 16 * n + col;
            row[n] = row_of(a, s, hk, G, r);
            M::load_row(q[n], a.Q, row[n].at, r < s.n * G, c.d, lane);
        }
        struct Stage {
            typename M::KTile k;
            float* to;  // the weight that this lane writes, or NULL
            float old;
        };
        auto load = [&](Stage& st, int t0, int p0) {
            M::load_k(c, st.k, page_list[((t0 + M::k_group(lane)) >> shift) - p0], hk, t0, lane);
            st.to = nullptr;
            st.old = 0.f;
            const int key = t0 + M::key_of(g, col);
            if (col < M::PER && key < end) {
                const int p = page_list[(key >> shift) - p0];
                if (p >= 0) {
                    st.to = c.weights + (int64_t(p) * c.H + hk) * c.page + (key & mask);
                    if (add) st.old = *st.to;
                }
            }
        };
        auto compute = [&](const Stage& st, int t0) {
            float w[M::PER] = {};
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                floatx4 sc[M::U];
                M::scores(st.k, q[n], sc);
#pragma unroll
                for (int v = 0; v < M::PER; ++v) {
                    const float x = __builtin_amdgcn_exp2f(fmaf(sc[v / 4][v % 4], c2, -row[n].lse2));
                    w[v] += t0 + M::key_of(g, v) < row[n].limit ? x : 0.f;
                }
            }
            float mine = 0.f;
#pragma unroll
            for (int v = 0; v < M::PER; ++v) {
                const float sum = group_sum(w[v]);
                mine = v == col ? sum : mine;
            }
            if (st.to) *st.to = st.old + mine;
        };
        for (int seg = lo; seg < end; seg += kSegment) {
            const int seg_end = min(end, seg + kSegment), p0 = seg >> shift;
            const int entries = ((((seg_end + JUMP - 1) & -JUMP) - 1) >> shift) - p0 + 1;
            __syncthreads();  // the list before has been read
            for (int e = threadIdx.x; e < entries; e += 256)
                page_list[e] = page_of(c.table, c.width, c.pages, b, p0 + e);
            __syncthreads();
            int t0 = seg + wave * KEYS;
            if (t0 >= seg_end) continue;
            Stage A, B;
            load(A, t0, p0);
            for (;;) {
                if (t0 + JUMP < seg_end) load(B, t0 + JUMP, p0);
                compute(A, t0);
                t0 += JUMP;
                if (t0 >= seg_end) break;
                if (t0 + JUMP < seg_end) load(A, t0 + JUMP, p0);
                compute(B, t0);
                t0 += JUMP;
                if (t0 >= seg_end) break;
            }
        }
    }
}

// SPLIT: the waves share their keys and take the groups of 16 rows in turn; their sums are added
// in LDS in the waves' order.
template <typename T, int D, int NK, bool SPLIT>
__global__ __launch_bounds__(256) void weights_keys_kernel(const PagedArgs a, int strides,
                                                           const Div group) {
    using M = TileMath<T, D>;
    constexpr int KEYS = M::KEYS, MINE = NK * KEYS, ALL = SPLIT ? MINE : 4 * MINE;
    __shared__ float sums[4][MINE];
    const sparsp_cache& c = a.cache;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = lane & 15, g = lane >> 4;
    const int bh = blockIdx.x / strides, first = blockIdx.x % strides;
    const int b = bh / c.H, hk = bh % c.H;
    const int G = int(group.d);
    const Seq s = sequence(c, a.tokens, b);
    const int rows = s.n * G;
    const float c2 = a.scale * kLog2e;
    const int shift = __builtin_ctz(c.page), mask = c.page - 1;
    constexpr int JUMP = SPLIT ? 64 : 16;  // rows of a turn
    for (int w0 = first * ALL; w0 < s.kv; w0 += strides * ALL) {
        const int t0 = w0 + (SPLIT ? 0 : wave * MINE);
        typename M::KTile k[NK];
        float w[NK][M::PER];
#pragma unroll
        for (int m = 0; m < NK; ++m) {
            const int from = t0 + m * KEYS;
            const int page =
                page_of(c.table, c.width, c.pages, b, (from + M::k_group(lane)) >> shift);
            M::load_k(c, k[m], page, hk, from, lane);
#pragma unroll
            for (int v = 0; v < M::PER; ++v) w[m][v] = 0.f;
        }
        struct Stage {
            typename M::QTile q;
            float lse;
            int limit;  // end of the keys that the row sees
        };
        auto load = [&](Stage& st, int r0) {
            const bool live = r0 + col < rows;
            const int r = live ? r0 + col : 0, i = int(group.quot(uint32_t(r)));
            const int h = hk * G + r - i * G;
            st.lse = a.lse_in[int64_t(h) * a.tokens + s.q0 + i];
            st.limit = !live ? 0 : a.causal ? min(s.kv, s.kv - s.n + i + 1) : s.kv;
            M::load_row(st.q, a.Q, int64_t(h) * a.q_head + int64_t(s.q0 + i) * a.q_token, live, c.d,
                        lane);
        };
        auto compute = [&](const Stage& st) {
            const float neg = -st.lse * kLog2e;
            const int limit = st.lse == -INFINITY ? 0 : st.limit;
#pragma unroll
            for (int m = 0; m < NK; ++m) {
                floatx4 sc[M::U];
                M::scores(k[m], st.q, sc);
#pragma unroll
                for (int v = 0; v < M::PER; ++v) {
                    const float x = __builtin_amdgcn_exp2f(fmaf(sc[v / 4][v % 4], c2, neg));
                    w[m][v] += t0 + m * KEYS + M::key_of(g, v) < limit ? x : 0.f;
                }
            }
        };
        // Rows before see none of these keys.
        int r0 = a.causal ? max(0, t0 - (s.kv - s.n)) * G / 16 * 16 : 0;
        if (SPLIT) r0 += 16 * wave;
        if (r0 < rows) {
            Stage A, B;
            load(A, r0);
            for (;;) {
                if (r0 + JUMP < rows) load(B, r0 + JUMP);
                compute(A);
                r0 += JUMP;
                if (r0 >= rows) break;
                if (r0 + JUMP < rows) load(A, r0 + JUMP);
                compute(B);
                r0 += JUMP;
                if (r0 >= rows) break;
            }
        }
        __syncthreads();  // the sums before have been read
#pragma unroll
        for (int m = 0; m < NK; ++m)
#pragma unroll
            for (int v = 0; v < M::PER; ++v) {
                const float sum = group_sum(w[m][v]);
                if (col == v) sums[wave][m * KEYS + M::key_of(g, v)] = sum;
            }
        __syncthreads();
        const int mine = SPLIT ? int(threadIdx.x) : lane, key = t0 + mine;
        if (mine < MINE && key < s.kv) {
            float sum = sums[SPLIT ? 0 : wave][mine];
            if (SPLIT)
#pragma unroll
                for (int o = 1; o < 4; ++o) sum += sums[o][mine];
            const int at = page_of(c.table, c.width, c.pages, b, key >> shift);
            if (at >= 0) {
                float* to = c.weights + (int64_t(at) * c.H + hk) * c.page + (key & mask);
                *to = a.accumulate ? *to + sum : sum;
            }
        }
    }
}

template <typename T, int NK, bool SPLIT>
hipError_t launch_keys(const PagedArgs& a, int most_kv, hipStream_t s) {
    const int keys = (sizeof(T) == 2 ? 32 : 16) * NK * (SPLIT ? 1 : 4);
    const int pairs = a.cache.B * a.cache.H;
    const int strides = std::max(1, std::min((most_kv + keys - 1) / keys, (1 << 22) / pairs));
    const Div group = make_div(uint32_t(a.q_heads / a.cache.H));
    if (a.cache.d <= 64)
        weights_keys_kernel<T, 64, NK, SPLIT><<<pairs * strides, 256, 0, s>>>(a, strides, group);
    else
        weights_keys_kernel<T, 128, NK, SPLIT><<<pairs * strides, 256, 0, s>>>(a, strides, group);
    return hipGetLastError();
}

template <typename T, int NC>
hipError_t launch_rows(const PagedArgs& a, int most_kv, hipStream_t s) {
    const int pairs = a.cache.B * a.cache.H;
    const int round = sizeof(T) == 2 ? 128 : 64;  // keys
    PagedPlan p = {};
    p.tiles = 1;
    p.parts = std::max(1, std::min((most_kv + round - 1) / round,
                                   std::max(1, 32 * kCus / std::min(pairs, 32 * kCus))));
    p.step = std::max(round, ((most_kv + p.parts - 1) / p.parts + round - 1) / round * round);
    if (a.cache.d <= 64)
        weights_rows_kernel<T, 64, NC><<<pairs * p.parts, 256, 0, s>>>(a, p);
    else
        weights_rows_kernel<T, 128, NC><<<pairs * p.parts, 256, 0, s>>>(a, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_weights(const PagedArgs& a, hipStream_t s) {
    const int most_new = a.max_new > 0 && a.max_new < a.tokens ? a.max_new : a.tokens;
    const int span = a.cache.width * a.cache.page;
    const int most_kv = a.max_kv > 0 && a.max_kv < span ? a.max_kv : span;
    const int64_t rows = int64_t(most_new) * (a.q_heads / a.cache.H);
    const bool bf16 = a.cache.dtype == SPARSP_BF16;
    if (rows <= 16)
        return bf16 ? launch_rows<uint16_t, 1>(a, most_kv, s) : launch_rows<float, 1>(a, most_kv, s);
    if (rows <= 32)
        return bf16 ? launch_rows<uint16_t, 2>(a, most_kv, s) : launch_rows<float, 2>(a, most_kv, s);
    // Workgroups of 64 keys.
    const int64_t units = int64_t(a.cache.B) * a.cache.H * ((int64_t(most_kv) + 63) / 64);
    if (bf16)
        return units <= 2 * kCus ? launch_keys<uint16_t, 2, true>(a, most_kv, s)
                                 : launch_weights_tiles(a, s);
    return units < kCus || rows >= 2048 ? launch_keys<float, 1, true>(a, most_kv, s)
                                        : launch_keys<float, 1, false>(a, most_kv, s);
}

}  // namespace sparsp
