// Attention of new tokens over the paged cache (Eq. 1 over a sequence's cached tokens).
//
// Rows. The query heads of one key head share its keys, so a row is (token, head of the
// group), token-major: n new tokens of a group of G heads are n G rows, packed 16 to an
// operand. A decoding step of G = 4 thus reads K and V once for four rows.
//
// paged_rows_kernel, for few rows a sequence and for float32: a workgroup takes 16 NC rows and
// a part of the sequence's keys; its four waves walk the key tiles in turn (wave w the tiles
// w, w+4, ...), each with a softmax of its own, the next tile loading while one is computed.
// The waves' results are merged in LDS through their running maxima. What bounds it is reading
// K and V, so every tile goes straight to operand registers (paged_tiles.h). More bf16 rows go
// to paged_attn_tiles.hip.
//
// Long caches are split: each part (a multiple of `step` keys) writes its normalised
// output, its sum of exponentials and the score they are relative to, float32, to the workspace,
// and a merge kernel joins a row's parts in their order. A sequence short enough for one part writes
// its output directly.
#include <algorithm>
#include <cmath>

#include "paged_tiles.h"

namespace sparsp {
namespace {

constexpr int kCus = 256;
constexpr int kSegment = 16384;  // keys whose page numbers are held at once

template <typename T, int D, int NC>
__global__ __launch_bounds__(256, 2) void paged_rows_kernel(const PagedArgs a, const PagedPlan plan) {
    using M = TileMath<T, D>;
    constexpr int KEYS = M::KEYS, DV = M::DV, PITCH = D + 4;
    __shared__ float merge_o[4][16][PITCH];
    __shared__ float merge_m[4][16], merge_l[4][16];
    __shared__ int page_list[kSegment / 16];
    const sparsp_cache& c = a.cache;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = lane & 15, g = lane >> 4;
    const int G = a.q_heads / c.H;
    Work work;
    if (!work_of<16 * NC>(plan, c, a.tokens, G, &work)) return;
    const int b = work.b, hk = work.hk, part = work.part;
    const Seq s = sequence(c, a.tokens, b);
    const int rows = s.n * G;
    const int keys = part_keys(plan, s.kv);
    const bool whole = s.kv <= keys;
    if (part > 0 && part * int64_t(keys) >= s.kv) return;
    const int lo = part * keys, part_end = min(s.kv - lo, keys) + lo;
    const float c2 = a.scale * kLog2e;
    const int shift = __builtin_ctz(c.page);

    for (int tile = work.tile; tile * int64_t(16 * NC) < rows; tile += work.stride) {
        typename M::QTile q[NC];
        int limit[NC], lowest = 1 << 30;  // keys before limit are seen
        int end = 0;
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            const int r = (tile * NC + n) * 16 + col;
            const bool live = r < rows;
            const int i = live ? r / G : 0, h = hk * G + (live ? r % G : 0);
            limit[n] = a.causal ? min(s.kv, s.kv - s.n + i + 1) : s.kv;
            if (!live) limit[n] = 1 << 30;
            lowest = min(lowest, limit[n]);
            M::load_row(q[n], a.Q, int64_t(h) * a.q_head + int64_t(s.q0 + i) * a.q_token, live,
                        c.d, lane);
        }
        {
            const int last = min(rows, (tile + 1) * 16 * NC) - 1;
            end = a.causal ? min(s.kv, s.kv - s.n + last / G + 1) : s.kv;
            end = min(end, part_end);
        }

        floatx4 acc[NC][DV];
        float m[NC], l[NC];
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            m[n] = -INFINITY;
            l[n] = 0.f;
#pragma unroll
            for (int d = 0; d < DV; ++d) acc[n][d] = floatx4{};
        }

        struct Stage {
            typename M::KTile k;
            typename M::VTile v;
            int kp, vp;
        };
        auto load_k = [&](Stage& st, int t0, int p0) {
            st.kp = page_list[((t0 + M::k_group(lane)) >> shift) - p0];
            M::load_k(c, st.k, st.kp, hk, t0, lane);
        };
        auto load_v = [&](Stage& st, int t0, int p0) {
            st.vp = page_list[((t0 + M::v_group(lane)) >> shift) - p0];
            M::load_v(c, st.v, st.vp, hk, t0, lane);
        };
        // after_scores: what is done once K has been used.
        auto compute = [&](Stage& st, int t0, auto after_scores) {
            const bool masked =
                __ballot(t0 + KEYS > lowest || t0 + KEYS > end || st.kp < 0 || st.vp < 0) != 0;
            if (masked) {
                // What lies behind the sequence may be anything, NaN included: rows of V there
                // are zeroed, not multiplied by a probability of zero.
                const int live = st.vp < 0 ? 0 : part_end - (t0 + M::v_group(lane));
                M::clear_v(st.v, live);
            }
            typename M::P pr[NC];
            floatx4 sc[NC][M::U];
#pragma unroll
            for (int n = 0; n < NC; ++n) M::scores(st.k, q[n], sc[n]);
            after_scores();
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                float p[M::PER];
#pragma unroll
                for (int v = 0; v < M::PER; ++v) p[v] = sc[n][v / 4][v % 4];
                if (masked) {
                    const int lim = st.vp < 0 ? 0 : min(limit[n], part_end);
#pragma unroll
                    for (int v = 0; v < M::PER; ++v)
                        p[v] = t0 + M::key_of(g, v) < lim ? p[v] : -INFINITY;
                }
                float mx = p[0];
#pragma unroll
                for (int v = 1; v < M::PER; ++v) mx = fmaxf(mx, p[v]);
                mx = row_max(mx);
                if (__ballot(mx > m[n]) != 0) {
                    const float top = fmaxf(m[n], mx);
                    const float alpha =
                        top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m[n] - top) * c2);
                    m[n] = top;
                    l[n] *= alpha;
#pragma unroll
                    for (int d = 0; d < DV; ++d) acc[n][d] *= alpha;
                }
                const float base = m[n] == -INFINITY ? 0.f : m[n];
#pragma unroll
                for (int v = 0; v < M::PER; ++v) {
                    p[v] = __builtin_amdgcn_exp2f((p[v] - base) * c2);
                    l[n] += p[v];
                }
                pr[n] = M::pack(p);
            }
            M::template output<NC>(st.v, pr, acc);
        };

        // Two tiles in flight: one is computed while the next is loaded. (With 32 rows the
        // registers hold one tile: the next one's K is loaded once the scores are there, its V
        // behind the output.) The page numbers of the next 16,384 keys lie in LDS: a load of
        // them would return in order with the rows asked for before.
        constexpr int JUMP = 4 * KEYS;
        for (int seg = lo; seg < end; seg += kSegment) {
            const int seg_end = min(end, seg + kSegment), p0 = seg >> shift;
            const int entries = ((((seg_end + JUMP - 1) & -JUMP) - 1) >> shift) - p0 + 1;
            __syncthreads();  // the list before has been read
            for (int e = threadIdx.x; e < entries; e += 256)
                page_list[e] = page_of(c.table, c.width, c.pages, b, p0 + e);
            __syncthreads();
            int t0 = seg + wave * KEYS;
            if (t0 >= seg_end) continue;
            Stage A;
            load_k(A, t0, p0);
            load_v(A, t0, p0);
            if constexpr (NC == 1) {
                Stage B;
                auto next = [&](Stage& st) {
                    if (t0 + JUMP >= seg_end) return;
                    load_k(st, t0 + JUMP, p0);
                    load_v(st, t0 + JUMP, p0);
                };
                for (;;) {
                    next(B);
                    compute(A, t0, [] {});
                    t0 += JUMP;
                    if (t0 >= seg_end) break;
                    next(A);
                    compute(B, t0, [] {});
                    t0 += JUMP;
                    if (t0 >= seg_end) break;
                }
            } else {
                for (;;) {
                    const bool more = t0 + JUMP < seg_end;
                    compute(A, t0, [&] {
                        if (more) load_k(A, t0 + JUMP, p0);
                    });
                    if (!more) break;
                    t0 += JUMP;
                    load_v(A, t0, p0);
                }
            }
        }

#pragma unroll
        for (int n = 0; n < NC; ++n) {
            const float sum = row_sum(l[n]);
            __syncthreads();  // the rows before have been read
#pragma unroll
            for (int d = 0; d < DV; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) merge_o[wave][col][DV * (4 * g + e) + d] = acc[n][d][e];
            if (g == 0) {
                merge_m[wave][col] = m[n];
                merge_l[wave][col] = sum;
            }
            __syncthreads();
            for (int e = threadIdx.x; e < 16 * (D / 4); e += 256) {
                const int row = e / (D / 4), ch = e % (D / 4) * 4;
                const int r = (tile * NC + n) * 16 + row;
                if (r >= rows || ch >= c.d) continue;
                float top = -INFINITY;
#pragma unroll
                for (int w = 0; w < 4; ++w) top = fmaxf(top, merge_m[w][row]);
                float x[4] = {}, total = 0.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float mw = merge_m[w][row];
                    const float f =
                        mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mw - top) * c2);
                    total += f * merge_l[w][row];
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) x[q4] += f * merge_o[w][row][ch + q4];
                }
                const bool any = total > 0.f;
                const float inv = any ? 1.f / total : 0.f;
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) x[q4] = any ? x[q4] * inv : 0.f;
                const int i = r / G, h = hk * G + r % G;
                const int64_t at = int64_t(h) * a.tokens + s.q0 + i;
                if (whole) {
                    store4(a.O, int64_t(h) * a.o_head + int64_t(s.q0 + i) * a.o_token + ch,
                           a.out_bf16, x);
                    if (ch == 0 && a.lse)
                        a.lse[at] = any ? fmaf(top, a.scale, __logf(total)) : -INFINITY;
                } else {
                    store4(plan.part_o, (at * plan.parts + part) * c.d + ch, false, x);
                    if (ch == 0) {
                        plan.part_sum[at * plan.parts + part] = total;
                        plan.part_ref[at * plan.parts + part] = top;
                    }
                }
            }
        }
    }
}

// Joins the parts of rows (token, head). 32 lanes hold a row, four channels a lane. SHARED, for few
// rows: the eight groups of a workgroup take one row's parts in turn and are added in LDS in
// their order. Otherwise each group has a row of its own (16,384 rows of two parts: 27 us with
// the attention, 50 us with a workgroup for each row).
template <bool SHARED>
__global__ __launch_bounds__(256) void paged_merge_kernel(const PagedArgs a, const PagedPlan plan,
                                                          int per_head) {
    __shared__ float part_x[8][128];
    __shared__ float part_w[8];
    const sparsp_cache& c = a.cache;
    const int bh = blockIdx.x / per_head;
    const int b = bh / a.q_heads, h = bh % a.q_heads;
    const Seq s = sequence(c, a.tokens, b);
    const int keys = part_keys(plan, s.kv);
    if (s.kv <= keys) return;
    const int parts = (s.kv + keys - 1) / keys;
    const float c2 = a.scale * kLog2e;
    const int group = threadIdx.x >> 5, lane = threadIdx.x & 31, ch = lane * 4;
    const int first = SHARED ? group : 0, stride = SHARED ? 8 : 1;  // of a group's parts
    constexpr int ROWS = SHARED ? 1 : 8, DEEP = 4;                  // DEEP parts in flight
    for (int i0 = blockIdx.x % per_head * ROWS; i0 < s.n; i0 += per_head * ROWS) {
        const int i = SHARED ? i0 : min(i0 + group, s.n - 1);
        const int64_t at = int64_t(h) * a.tokens + s.q0 + i;
        const float *sum = plan.part_sum + at * plan.parts, *ref = plan.part_ref + at * plan.parts;
        float top = -INFINITY;
        for (int p = lane; p < parts; p += 32) top = fmaxf(top, ref[p]);
#pragma unroll
        for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
        const float base = top == -INFINITY ? 0.f : top;
        float x[4] = {}, total = 0.f;
        const float* from = plan.part_o + at * plan.parts * c.d + (ch < c.d ? ch : 0);
        for (int p0 = first; p0 < parts; p0 += stride * DEEP) {
            floatx4 y[DEEP];
            float part[DEEP], mass[DEEP];
#pragma unroll
            for (int u = 0; u < DEEP; ++u) {
                const int p = min(p0 + stride * u, parts - 1);
                y[u] = *reinterpret_cast<const floatx4*>(from + int64_t(p) * c.d);
                part[u] = ref[p];
                mass[u] = sum[p];
            }
#pragma unroll
            for (int u = 0; u < DEEP; ++u) {
                const float w = p0 + stride * u < parts
                                    ? mass[u] * __builtin_amdgcn_exp2f((part[u] - base) * c2)
                                    : 0.f;
                total += w;
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) x[q4] += w * y[u][q4];
            }
        }
        if constexpr (SHARED) {
            __syncthreads();  // the row before has been read
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) part_x[group][ch + q4] = x[q4];
            if (ch == 0) part_w[group] = total;
            __syncthreads();
            if (group > 0) continue;
            total = 0.f;
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) x[q4] = 0.f;
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                total += part_w[w];
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) x[q4] += part_x[w][ch + q4];
            }
        } else if (i0 + group >= s.n) {
            continue;
        }
        const bool any = total > 0.f;
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) x[q4] = any ? x[q4] / total : 0.f;
        if (ch < c.d)
            store4(a.O, int64_t(h) * a.o_head + int64_t(s.q0 + i) * a.o_token + ch, a.out_bf16, x);
        if (ch == 0 && a.lse)
            a.lse[at] = any ? fmaf(top, a.scale, __logf(total)) : -INFINITY;
    }
}

// The launch for what is known of the lengths. bf16 rows of more than 16 a sequence go to
// the kernel of 128-row tiles (d = 128: 32 sequences of 8,000, 32 rows each: 237 us 32 rows at
// a time from registers, 198 us; one of 2,000 with 24 rows 13.0 and 15.3 us). At d <= 64, where
// a row's operands take half the registers, those of more than 32 do (64 sequences of 400 to
// 4,000, 24 rows each: 34.6 us from registers, 38.0 us by the tiles). float32 rows are taken 16
// or 32 at a time.
//
// Parts of the keys, in rounds (a round of a workgroup's waves is 128 keys, 64 of float32). What
// at most two workgroups a CU do is latency: a round costs about 1 us, the merge kernel 4 us and
// about 0.1 us for each part of a row, least in sum at sqrt(10 rounds) parts (one sequence of
// 8 key heads, 1,500 tokens: 13.1 us in 3 parts, 9.5 us in 12; 9,000: 15.8 us in 18, 19.5 us
// in 71). Up to three rounds stay whole, and tiles of 128 rows, whose partial rows are many, up
// to seven (512 new tokens of 32 heads over 512: 20 us whole, 26 us in 4 parts).
//
// More workgroups than that makes are split until two a CU have work, into parts of four rounds
// and more if there are over eight (1,000 tokens of 16 heads over 8,000: 212 us whole, 81 us in
// 4 parts, which is that, and 93 us in 8); into four times as many where that leaves a quarter
// of the GPU empty (675 tokens of 32 heads over 24,153: 172 tiles, 283 us in 2 parts, 242 us in
// 8). Few rows a sequence, and float32, whose products take 8 times as long as bf16's while a
// merge costs the same, are split further, into parts of sixteen rounds (float32: eight), so
// that a ragged batch fills the GPU to the end: 64 sequences of 400 to 9,001 tokens, 4 rows each,
// take 195 us whole and 140 us in 5 parts, with 40 rows 221 us in one and 162 us in 5 (32 of
// 8,000 each, which gain nothing by it, 192 and 198 us); float32, 710 to 279 tokens of 5
// sequences over 5,671 to 9,606: 1,330 us whole, 984 us. bf16 rows of more than 64, whose partial
// rows cost more, take parts of 32 rounds where their workgroups are two a CU at most and that
// is twice as many parts (16 heads of 64, 796 and 284 tokens over 45,429 and 12,913: 365 us in 3
// parts, 231 us in 12; 84 heads of 128, 109 to 55 over 10,471 to 2,812: 168 us in 2, 189 us in
// 3). There are no more parts than the workspace holds.
struct Shape {
    PagedPlan plan;
    int rows;       // of a tile
    int64_t bytes;  // of workspace used
};

Shape shape(const PagedArgs& a, int64_t ws_bytes) {
    const sparsp_cache& c = a.cache;
    const int G = a.q_heads / c.H;
    const int span = c.width * c.page;
    const int most_new = a.max_new > 0 && a.max_new < a.tokens ? a.max_new : a.tokens;
    const int most_kv = a.max_kv > 0 && a.max_kv < span ? a.max_kv : span;
    Shape r = {};
    const int64_t rows = int64_t(most_new) * G;
    r.rows = rows <= 16 ? 16 : c.dtype == SPARSP_F32 || (rows <= 32 && c.d <= 64) ? 32 : 128;
    int64_t tiles = (rows + r.rows - 1) / r.rows;
    const int64_t pairs = int64_t(c.B) * c.H;
    // (a grid holds fewer than 2^32 threads, and units are rounded up to the eight XCDs)
    const int64_t room = std::max<int64_t>(1, (int64_t(1) << 22) / std::max<int64_t>(pairs, 8));
    tiles = std::min(tiles, room);
    const int round = c.dtype == SPARSP_F32 ? 64 : 128;  // keys
    const int64_t rounds = (int64_t(most_kv) + round - 1) / round;
    // Row tiles that can have work.
    const int64_t flat = a.tokens * int64_t(G) / r.rows + c.B;
    const int64_t live = std::min(pairs * tiles, c.H * flat);
    int64_t parts = std::min(rounds, int64_t(std::sqrt(10.0 * double(rounds))));
    if (rounds <= 3 + (r.rows == 128 ? std::min<int64_t>(4, live * parts / 128) : 0)) parts = 1;
    if (live * parts > 2 * kCus) {
        int64_t fill = 2 * kCus / std::min<int64_t>(live, 2 * kCus);
        if (rounds >= 16 && live < 2 * kCus && live * fill < 3 * kCus / 2) fill *= 4;
        const int64_t level = 16 * kCus / std::min<int64_t>(live, 16 * kCus);
        const bool tall = r.rows == 128 && rows > 64;
        const int64_t least = c.dtype == SPARSP_F32 ? 8 : tall ? 32 : 16;  // rounds of a part
        parts = std::max(fill, std::min(level, (rounds + least - 1) / least));
        if (tall && (live > 2 * kCus || parts < 2 * fill)) parts = fill;
        parts = rounds <= 8 ? 1 : std::min(parts, (rounds + 3) / 4);
    }
    const int64_t all_rows = int64_t(a.q_heads) * a.tokens, part_bytes = all_rows * (c.d + 2) * 4;
    parts = std::max<int64_t>(1, std::min(parts, ws_bytes / part_bytes));
    // Each workgroup finds its tile among those that have work, where they are few of pairs *
    // tiles: one long sequence among many, whose empty workgroups would cost more (32 heads of
    // 128, 256 sequences of one new token and one of 1,024 over 2,000 each: 900 us, 386 us; the
    // two kinds by themselves: 356 and 58 us). And where key heads leave XCDs less to do than
    // others (2 of 128, 2,000 tokens over 6,000: 203 us, 115 us; 5 of 64: 187 and 138 us; 4
    // sequences of 806 to 2,000 tokens, 2 heads: 184 and 115 us), but not like sequences that
    // fill all eight (4 of 2,000 tokens, 2 heads: 53 and 60 us).
    const bool even = a.tokens == int64_t(c.B) * most_new && parts == 1 && pairs % 8 == 0;
    if (pairs * tiles > 2 * live || (tiles >= 8 && c.H % 8 != 0 && pairs * parts < 64 && !even &&
                                     c.H * flat * parts <= 1 << 20))
        r.plan.flat = int(flat);
    r.plan.step = int((rounds + parts - 1) / parts) * round;
    r.plan.tiles = int(tiles);
    r.plan.parts = int(parts);
    // (in whole units of d + 1 numbers for every row)
    const int64_t unit = all_rows * (c.d + 1) * 4;
    r.bytes = parts > 1 ? (parts * part_bytes + unit - 1) / unit * unit : 0;
    return r;
}

template <typename T, int D, int NC>
hipError_t launch_rows(const PagedArgs& a, const PagedPlan& p, hipStream_t s) {
    paged_rows_kernel<T, D, NC><<<workgroups(p, a.cache), 256, 0, s>>>(a, p);
    return hipGetLastError();
}

hipError_t launch_few(const PagedArgs& a, const Shape& r, hipStream_t s) {
    const bool small = a.cache.d <= 64, few = r.rows == 16;
    if (a.cache.dtype == SPARSP_BF16)
        return !small ? launch_rows<uint16_t, 128, 1>(a, r.plan, s)
               : few  ? launch_rows<uint16_t, 64, 1>(a, r.plan, s)
                      : launch_rows<uint16_t, 64, 2>(a, r.plan, s);
    if (few)
        return small ? launch_rows<float, 64, 1>(a, r.plan, s)
                     : launch_rows<float, 128, 1>(a, r.plan, s);
    return small ? launch_rows<float, 64, 2>(a, r.plan, s) : launch_rows<float, 128, 2>(a, r.plan, s);
}

}  // namespace

int64_t paged_attn_workspace(const PagedArgs& a) {
    return shape(a, int64_t(1) << 40).bytes;
}

hipError_t launch_paged_attn(const PagedArgs& a, hipStream_t s) {
    Shape r = shape(a, a.ws ? a.ws_bytes : 0);
    if (r.plan.parts > 1) {
        r.plan.part_o = static_cast<float*>(a.ws);
        const int64_t rows = int64_t(a.q_heads) * a.tokens * r.plan.parts;
        r.plan.part_sum = r.plan.part_o + rows * a.cache.d;
        r.plan.part_ref = r.plan.part_sum + rows;
    }
    const hipError_t e = r.rows == 128 ? launch_paged_tiles(a, r.plan, s) : launch_few(a, r, s);
    if (e != hipSuccess || r.plan.parts == 1) return e;
    const int most_new = a.max_new > 0 && a.max_new < a.tokens ? a.max_new : a.tokens;
    const int64_t pairs = int64_t(a.cache.B) * a.q_heads;
    const bool shared = pairs * most_new <= 16 * kCus;
    const int64_t runs = shared ? most_new : (most_new + 7) / 8;  // workgroups of a head
    const int per = int(std::min(runs, std::max<int64_t>(1, (int64_t(1) << 15) / pairs)));
    if (shared)
        paged_merge_kernel<true><<<int(pairs) * per, 256, 0, s>>>(a, r.plan, per);
    else
        paged_merge_kernel<false><<<int(pairs) * per, 256, 0, s>>>(a, r.plan, per);
    return hipGetLastError();
}

}  // namespace sparsp
