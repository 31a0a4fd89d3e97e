// Attention weight per cached token: w[t] = sum over the rows that see t of
// exp(scale q.k_t - lse). One wave owns 32 keys (16 of float32) whose K rows stay in its
// registers as the A operand of the score product S^T = K Q^T, and walks the rows
// 16 at a time; each lane sums the exponentials of its keys over its column of rows,
// and the sixteen columns are added once at the end. No two waves add to the same
// weight, so there are no atomics and the order of a sum depends on the sizes alone.
#include "paged_plan.h"
#include "paged_tiles.h"

namespace sparsp {
namespace {

template <typename T, int D>
__global__ __launch_bounds__(256) void paged_weights_kernel(const PagedArgs a, int strides) {
    using M = TileMath<T, D>;
    const sparsp_cache& c = a.cache;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = lane & 15, g = lane >> 4;
    const int bh = blockIdx.x / strides, first = blockIdx.x % strides;
    const int b = bh / c.H, hk = bh % c.H;
    const int G = a.q_heads / c.H;
    const Seq s = sequence(c, a.tokens, b);
    const int rows = s.n * G;
    const float c2 = a.scale * kLog2e;
    constexpr int KEYS = M::KEYS;
    for (int t0 = (first * 4 + wave) * KEYS; t0 < s.kv; t0 += strides * 4 * KEYS) {
        typename M::KTile k;
        const int page = page_of(c.table, c.width, c.pages, b,
                                 (t0 + M::k_group(lane)) >> __builtin_ctz(c.page));
        M::load_k(c, k, page, hk, t0, lane);
        float w[M::PER] = {};
        // Rows before r_first see none of these keys.
        const int r_first = a.causal ? max(0, t0 - (s.kv - s.n)) * G : 0;
        for (int r0 = r_first / 16 * 16; r0 < rows; r0 += 16) {
            const int r = r0 + col;
            typename M::QTile q;
            int limit = 0;
            float lse2 = 0.f;
            int64_t q_at = 0;
            if (r < rows) {
                const int i = r / G, h = hk * G + r % G;
                q_at = int64_t(h) * a.q_head + int64_t(s.q0 + i) * a.q_token;
                limit = a.causal ? min(s.kv, s.kv - s.n + i + 1) : s.kv;
                const float l = a.lse_in[int64_t(h) * a.tokens + s.q0 + i];
                if (l == -INFINITY) limit = 0;
                lse2 = l * kLog2e;
            }
            M::load_row(q, a.Q, q_at, r < rows, c.d, lane);
            floatx4 sc[M::U];
            M::scores(k, q, sc);
#pragma unroll
            for (int v = 0; v < M::PER; ++v) {
                const int key = t0 + M::key_of(g, v);
                const float x = __builtin_amdgcn_exp2f(fmaf(sc[v / 4][v % 4], c2, -lse2));
                w[v] += key < limit ? x : 0.f;
            }
        }
#pragma unroll
        for (int v = 0; v < M::PER; ++v)
#pragma unroll
            for (int off = 1; off < 16; off <<= 1) w[v] += __shfl_xor(w[v], off);
        if (col < M::PER) {
            const int key = t0 + M::key_of(g, col);
            float mine = 0.f;
#pragma unroll
            for (int v = 0; v < M::PER; ++v) mine = v == col ? w[v] : mine;
            if (key < s.kv) {
                const int at = page_of(c.table, c.width, c.pages, b, key >> __builtin_ctz(c.page));
                if (at >= 0) {
                    float* to = c.weights + (int64_t(at) * c.H + hk) * c.page + (key & (c.page - 1));
                    *to = a.accumulate ? *to + mine : mine;
                }
            }
        }
    }
}

template <typename T>
hipError_t launch_t(const PagedArgs& a, int strides, hipStream_t s) {
    const int grid = a.cache.B * a.cache.H * strides;
    if (a.cache.d <= 64)
        paged_weights_kernel<T, 64><<<grid, 256, 0, s>>>(a, strides);
    else
        paged_weights_kernel<T, 128><<<grid, 256, 0, s>>>(a, strides);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_weights(const PagedArgs& a, hipStream_t s) {
    const int most_new = a.max_new > 0 && a.max_new < a.tokens ? a.max_new : a.tokens;
    if (a.cache.dtype == SPARSP_BF16 && int64_t(most_new) * (a.q_heads / a.cache.H) > 32)
        return launch_weights_tiles(a, s);
    const int span = a.cache.width * a.cache.page;
    const int keys = a.max_kv > 0 && a.max_kv < span ? a.max_kv : span;
    const int per = 4 * (a.cache.dtype == SPARSP_BF16 ? 32 : 16);
    const int64_t pairs = int64_t(a.cache.B) * a.cache.H;
    int64_t strides = (keys + per - 1) / per;
    const int64_t most = (int64_t(1) << 22) / pairs;
    if (strides > most) strides = most < 1 ? 1 : most;
    return a.cache.dtype == SPARSP_BF16 ? launch_t<uint16_t>(a, int(strides), s)
                                        : launch_t<float>(a, int(strides), s);
}

}  // namespace sparsp
