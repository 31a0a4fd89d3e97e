// Attention of few new tokens over a cache held in 4 bits.
//
// Rows, tiles, waves and parts are those of paged_rows_kernel (paged_attn.hip): 16 NC rows and a part
// of the keys a workgroup, four waves that walk tiles of 32 keys in turn with a softmax each, the next
// tile loading while one is computed, joined in LDS. A tile is a quarter of the bytes of bf16, and
// making bf16 of it costs vector instructions (32 conversions and 32 permutations a lane for a tile of
// d = 128), so everything else in the loop is kept from the vector unit. A tile's page is the same for
// all lanes, so its address is scalar, and lanes add constants. The reference of a row's exponentials
// moves only where they grow past it, as in paged_attn_tiles.hip, so a tile takes no maximum and
// rescales nothing. 64 sequences of 400 to 9,001 tokens, 8 key heads, one new token each: 46 us (184
// MB, 4.0 TB/s), 59 us as one more tile type of paged_rows_kernel. Neither issue (38% of it) nor reading
// is full then: parts of 1,920 keys make 968 workgroups of 1 to 15 rounds of 128 keys for the 768 that
// the registers and LDS let reside. Sequences of 9,000 each: 4.9 TB/s in 5 parts, 5.4 whole, 192 of them
// 5.4 and 5.7. One tile in flight and four waves a SIMD spill (64 of 9,000: 172 us), two waves and three
// tiles gain nothing (126.8 and 126.8 us).
#include "paged_four.h"

namespace sparsp {
namespace {

constexpr int kSegment = 16384;  // keys whose page numbers are held at once

template <int TERMS, int C, int NC, bool WINDOW, bool HALVES>
__global__ __launch_bounds__(256, 2) void paged_four_kernel(const PagedArgs a, const PagedPlan plan) {
    constexpr int D = C <= 64 ? 64 : 128;
    using M = TileMath<Four<TERMS, C>, D>;
    constexpr int KEYS = M::KEYS, DV = M::DV, PITCH = D + 4, JUMP = 4 * KEYS;
    __shared__ float merge_o[4][16][PITCH];
    __shared__ float merge_m[4][16], merge_l[4][16], merge_f[4][16];
    __shared__ int page_list[kSegment / 16];  // of each 16 keys
    const sparsp_cache& c = a.cache;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int G = a.q_heads / c.H;
    Work work;
    if (!work_of<16 * NC>(plan, c, a.tokens, G, &work)) return;
    // (the same for all lanes, which addresses have to show)
    const int b = __builtin_amdgcn_readfirstlane(work.b);
    const int hk = __builtin_amdgcn_readfirstlane(work.hk);
    const int part = __builtin_amdgcn_readfirstlane(work.part);
    const Seq s = sequence(c, a.tokens, b);
    const int rows = s.n * G;
    Span span = {0, 0, s.kv, 0};
    int keys = part_keys(plan, s.kv);
    bool whole = s.kv <= keys;
    if (!WINDOW && part > 0 && part * int64_t(keys) >= s.kv) return;
    int lo = part * keys, part_end = min(s.kv - lo, keys) + lo;
    const float c2 = a.scale * kLog2e;
    const int shift = __builtin_ctz(c.page);
    const typename M::template Source<HALVES> source(a, hk, lane);

    for (int tile = __builtin_amdgcn_readfirstlane(work.tile); tile * int64_t(16 * NC) < rows;
         tile += work.stride) {
        if constexpr (WINDOW) {
            span = span_of(a, s, G, tile * 16 * NC, min(rows, (tile + 1) * 16 * NC) - 1, KEYS);
            keys = part_keys(plan, span.len);
            whole = span.len <= keys;
            if (part > 0 && part * int64_t(keys) >= span.len) continue;
            lo = part * keys;
            part_end = min(span.len - lo, keys) + lo;
        }
        typename M::QTile q[NC];
        int limit[NC], lowest = 1 << 30;  // keys before limit are seen
        int first[NC], latest = 0;        // with a window, those from first on and the sinks
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            const int r = (tile * NC + n) * 16 + col;
            const bool live = r < rows;
            const int i = live ? r / G : 0, h = hk * G + (live ? r % G : 0);
            limit[n] = a.causal ? min(s.kv, s.kv - s.n + i + 1) : s.kv;
            if constexpr (WINDOW) {
                limit[n] -= span.skip;
                first[n] = live ? limit[n] - a.window : 0;
                latest = max(latest, first[n]);
            }
            if (!live) limit[n] = 1 << 30;
            lowest = min(lowest, limit[n]);
            M::load_row(q[n], a.Q, int64_t(h) * a.q_head + int64_t(s.q0 + i) * a.q_token, live,
                        c.d, lane);
        }
        int end;
        {
            const int last = min(rows, (tile + 1) * 16 * NC) - 1;
            end = a.causal ? min(s.kv, s.kv - s.n + last / G + 1) : s.kv;
            end = min(end - span.skip, part_end);
        }

        // l: a lane's sum of exponentials. lim: what its eight may sum to before the reference moves;
        // kSeen, or -1: the row has seen nothing yet, or kFar. base: minus the reference in log2
        // units, or with kFar the reference as a score.
        constexpr float kSeen = 256.f, kFar = -2.f;
        floatx4 acc[NC][DV];
        float l[NC], lim[NC], base[NC];
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            lim[n] = limit[n] > 0 ? -1.f : INFINITY;  // (a row that sees nothing never asks)
            l[n] = base[n] = 0.f;
#pragma unroll
            for (int d = 0; d < DV; ++d) acc[n][d] = floatx4{};
        }

        struct Stage {
            typename M::KTile k;
            typename M::VTile v;
            int page, second;
        };
        auto load = [&](Stage& st, int t0, int p0) {
            const int e = (t0 - p0) >> 4;
            st.page = __builtin_amdgcn_readfirstlane(page_list[e]);
            st.second = __builtin_amdgcn_readfirstlane(page_list[e + 1]);
            source.load(st.k, st.v, st.page, st.second, WINDOW ? span.cached(t0) : t0);
        };
        auto compute = [&](Stage& st, int t0) {
            const bool masked = __ballot(t0 + KEYS > lowest || t0 + KEYS > end || st.page < 0 ||
                                         st.second < 0 ||
                                         (WINDOW && t0 < latest && t0 + KEYS > a.sinks)) != 0;
            const bool gone = (g < 2 ? st.page : st.second) < 0;  // this lane's eight keys
            if (masked) {
                // What lies behind the sequence may be anything, NaN included: rows of V there
                // are zeroed, not multiplied by a probability of zero.
                M::clear_v(st.v, gone ? 0 : part_end - (t0 + M::v_group(lane)));
            }
            floatx4 sc[NC][M::U];
#pragma unroll
            for (int n = 0; n < NC; ++n) M::scores(st.k, q[n], sc[n]);
            float p[NC][M::PER], sum[NC];
            auto add = [&](int n) {
                sum[n] = p[n][0];
#pragma unroll
                for (int v = 1; v < M::PER; ++v) sum[n] += p[n][v];
            };
            bool moves = false;
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                if (masked) {
                    const int upto = gone ? 0 : min(limit[n], part_end);
#pragma unroll
                    for (int v = 0; v < M::PER; ++v) {
                        const int key = t0 + M::key_of(g, v);
                        const bool seen =
                            key < upto && (!WINDOW || key >= first[n] || key < a.sinks);
                        if (!seen) sc[n][v / 4][v % 4] = -INFINITY;
                    }
                }
#pragma unroll
                for (int v = 0; v < M::PER; ++v)
                    p[n][v] = __builtin_amdgcn_exp2f(fmaf(sc[n][v / 4][v % 4], c2, base[n]));
                add(n);
                moves |= sum[n] > lim[n];
            }
            if (__ballot(moves) != 0) {
#pragma unroll
                for (int n = 0; n < NC; ++n) {
                    float mx = sc[n][0][0];
#pragma unroll
                    for (int v = 1; v < M::PER; ++v) mx = fmaxf(mx, sc[n][v / 4][v % 4]);
                    mx = row_max(mx);
                    // (far references as in paged_attn_tiles.hip)
                    const bool was_far = lim[n] == kFar;
                    const float before = lim[n] == kSeen ? -base[n] : -INFINITY;
                    const float top = fmaxf(before, mx * c2);
                    const bool far = was_far || (mx > -INFINITY && !(fabsf(top) < 0x1p24f));
                    const float ref = was_far ? fmaxf(base[n], mx) : mx;
                    float alpha = far ? fmaf(-ref, c2, before) : before - top;
                    if (was_far) alpha = (base[n] - ref) * c2;
                    alpha = !far && top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(alpha);
                    l[n] *= alpha;
                    lim[n] = far               ? kFar
                             : top > -INFINITY ? kSeen
                             : limit[n] > 0    ? -1.f
                                               : INFINITY;
                    base[n] = far ? ref : top == -INFINITY ? 0.f : -top;
#pragma unroll
                    for (int d = 0; d < DV; ++d) acc[n][d] *= alpha;
#pragma unroll
                    for (int v = 0; v < M::PER; ++v) {
                        const float x = sc[n][v / 4][v % 4];
                        p[n][v] = __builtin_amdgcn_exp2f(far ? (x - base[n]) * c2
                                                             : fmaf(x, c2, base[n]));
                    }
                    add(n);
                }
            }
            typename M::P pr[NC];
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                l[n] += sum[n];
                pr[n] = M::pack(p[n]);
            }
            M::template output<NC>(st.v, pr, acc);
        };

        for (int seg = lo; seg < end; seg += kSegment) {
            const int seg_end = min(end, seg + kSegment);
            const int entries = (((seg_end + JUMP - 1) & -JUMP) - seg) >> 4;
            __syncthreads();  // the list before has been read
            for (int e = threadIdx.x; e < entries; e += 256) {
                const int key = seg + 16 * e;
                const bool seen = !WINDOW || span.sees(key, a.sinks);
                const int j = (WINDOW ? span.cached(key) : key) >> shift;
                page_list[e] = seen ? page_of(c.table, c.width, c.pages, b, j) : -1;
            }
            __syncthreads();
            const int t0 = seg + wave * KEYS;
            const int turns = __builtin_amdgcn_readfirstlane((seg_end - t0 + JUMP - 1) / JUMP);
            if (turns <= 0) continue;
            // Two tiles in flight. Every turn loads, the last ones their own tile again, and the loop
            // has one way out: where loads are a choice, the wait for one tile's is one for the
            // next one's too.
            auto at = [&](int turn) { return t0 + min(turn, turns - 1) * JUMP; };
            Stage A, B;
            load(A, t0, seg);
            for (int turn = 0; turn < turns; turn += 2) {
                load(B, at(turn + 1), seg);
                compute(A, t0 + turn * JUMP);
                load(A, at(turn + 2), seg);
                if (turn + 1 < turns) compute(B, t0 + (turn + 1) * JUMP);
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
                // The reference as a score, rounded, and what the sums are multiplied by for it.
                const bool far = lim[n] == kFar, none = !(sum > 0.f);
                const float ref = far ? base[n] : -base[n] / c2;
                merge_m[wave][col] = none ? -INFINITY : ref;
                merge_l[wave][col] = sum;
                merge_f[wave][col] = far ? 1.f : __builtin_amdgcn_exp2f(fmaf(-ref, c2, -base[n]));
            }
            __syncthreads();
            for (int e = threadIdx.x; e < 16 * (D / 4); e += 256) {
                const int row = e / (D / 4), ch = e % (D / 4) * 4;
                const int r = (tile * NC + n) * 16 + row;
                if (r >= rows || ch >= C) continue;
                float top = -INFINITY;
#pragma unroll
                for (int w = 0; w < 4; ++w) top = fmaxf(top, merge_m[w][row]);
                float x[4] = {}, total = 0.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float mw = merge_m[w][row];
                    const float f = mw == -INFINITY ? 0.f
                                                    : merge_f[w][row] *
                                                          __builtin_amdgcn_exp2f((mw - top) * c2);
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

template <int TERMS, int C, int NC>
hipError_t launch(const PagedArgs& a, const PagedPlan& p, hipStream_t s) {
    const auto kernel =
        a.cache.page == 16 ? (a.window ? paged_four_kernel<TERMS, C, NC, true, true>
                                       : paged_four_kernel<TERMS, C, NC, false, true>)
                           : (a.window ? paged_four_kernel<TERMS, C, NC, true, false>
                                       : paged_four_kernel<TERMS, C, NC, false, false>);
    kernel<<<workgroups(p, a.cache), 256, 0, s>>>(a, p);
    return hipGetLastError();
}
template <int C>
hipError_t launch_channels(const PagedArgs& a, const PagedPlan& p, hipStream_t s) {
    if (a.cache.dtype == SPARSP_BF16) {
        if constexpr (C <= 64)
            if (p.rows == 32) return launch<1, C, 2>(a, p, s);
        return launch<1, C, 1>(a, p, s);
    }
    if constexpr (C <= 64)
        if (p.rows == 32) return launch<3, C, 2>(a, p, s);
    return launch<3, C, 1>(a, p, s);
}

}  // namespace

hipError_t launch_four_few(const PagedArgs& a, const PagedPlan& p, hipStream_t s) {
    return a.cache.d == 32   ? launch_channels<32>(a, p, s)
           : a.cache.d == 64 ? launch_channels<64>(a, p, s)
           : a.cache.d == 96 ? launch_channels<96>(a, p, s)
                             : launch_channels<128>(a, p, s);
}

}  // namespace sparsp
