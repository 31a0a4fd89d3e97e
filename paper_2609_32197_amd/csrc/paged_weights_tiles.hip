// Attention weight per cached token for many rows, bf16: w[t] = sum over the rows that see t of
// exp(scale q.k_t - lse).
//
// A workgroup owns 256 keys, each of its four waves 64 of them, whose K rows stay in registers
// as the A operand of S^T = K Q^T. Q passes through LDS in tiles of 64 rows, shared by the
// waves: a lane's 1 KB of Q operand feeds four products of 16 keys. What bounds it is the
// vector unit: a score costs one FMA, one exponential and one addition beside a product of
// 2 d operations. Rows that do not exist, and rows of lse = -inf, get an exponent of -inf and
// add nothing; the causal limit is tested in the tiles it crosses only.
//
// The next tile's rows are loaded into registers while a tile is computed and written to the
// other LDS buffer behind it, one barrier a tile. LDS rows carry the XOR swizzle of K in
// paged_attn_tiles.hip's form: the 16 rows read together land on their own 16 bytes of 256.
#include <type_traits>

#include "paged_plan.h"

namespace sparsp {
namespace {

constexpr int kRows = 64;   // rows of a tile
constexpr int kKeys = 256;  // keys of a workgroup

// The XOR of a row's 16-byte chunk number: 16 consecutive rows at one chunk cover 256 bytes.
template <int D>
__device__ __forceinline__ int q_swizzle(int row) {
    return D == 128 ? row & 15 : (row >> 1) & 7;
}

// EVEN: the group's heads divide a tile's rows, so that a thread's rows keep their head.
template <int D, bool EVEN>
__global__ __launch_bounds__(256, 2) void weights_tiles_kernel(const PagedArgs a, int strides,
                                                               const Div group) {
    constexpr int NCH = D / 8, KT = D / 32;
    constexpr int LOADS = kRows * NCH / 256;  // 16-byte loads of a thread and tile
    __shared__ __attribute__((aligned(16))) uint16_t lds[2][kRows * D];
    __shared__ float row_neg[2][kRows];  // -lse in log2 units
    __shared__ int row_limit[2][kRows];
    const sparsp_cache& c = a.cache;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int bh = blockIdx.x / strides, first = blockIdx.x % strides;
    const int b = bh / c.H, hk = bh % c.H;
    const int G = int(group.d);
    const Seq s = sequence(c, a.tokens, b);
    const int rows = s.n * G;
    const float c2 = a.scale * kLog2e;
    const int shift = __builtin_ctz(c.page), mask = c.page - 1;
    const int heads_ahead = kRows % G;
    const int64_t ahead = (int64_t(heads_ahead) * a.q_head + int64_t(kRows / G) * a.q_token) * 2;
    const int64_t wrap = (a.q_token - int64_t(G) * a.q_head) * 2;

    for (int w0 = first * kKeys; w0 < s.kv; w0 += strides * kKeys) {
        const int t0 = w0 + wave * 64;
        // K rows of the wave's 64 keys: key 16 u + col of tile u, channels 32 kt + 8 g ..
        // (zeros behind d).
        bf16x8 k[4][KT];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int key = t0 + 16 * u + col;
            const int p = page_of(c.table, c.width, c.pages, b, key >> shift);
            const uint16_t* from =
                static_cast<const uint16_t*>(c.K) +
                ((int64_t(max(p, 0)) * c.H + hk) * c.page + (key & mask)) * c.d;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const int ch = 32 * kt + 8 * g;
                uint4 x = *reinterpret_cast<const uint4*>(from + (ch < c.d ? ch : 0));
                if (ch >= c.d) x = make_uint4(0, 0, 0, 0);
                k[u][kt] = __builtin_bit_cast(bf16x8, x);
            }
        }

        float w[4][4] = {};
        // Rows before r_first see none of the workgroup's keys, rows from r_clear on all of the
        // wave's.
        int r_first = 0, r_clear = 0;
        if (a.causal) {
            r_first = max(0, w0 - (s.kv - s.n)) * G / kRows * kRows;
            r_clear = max(0, t0 + 63 - (s.kv - s.n)) * G;
        }
        r_clear = __builtin_amdgcn_readfirstlane(r_clear);

        // A thread's rows of a tile, and their places in Q: 64 rows on, the token is 64 / G
        // further and the head of the group 64 % G, or that less G and a token more.
        const char* from[LOADS];
        int head[LOADS];
        const int ch = tid % NCH * 8;
        const char* q0 = static_cast<const char*>(a.Q) +
                         (int64_t(hk) * G * a.q_head + int64_t(s.q0) * a.q_token +
                          (ch < c.d ? ch : 0)) * 2;
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int r = r_first + (u * 256 + tid) / NCH;
            const int i = int(group.quot(uint32_t(r)));
            head[u] = r - i * G;
            from[u] = q0 + (head[u] * a.q_head + i * a.q_token) * 2;
        }
        u32x4_t next[LOADS];
        float next_lse = 0.f;
        int next_limit = 0;
        auto load = [&](int r0) {
            const bool whole = r0 + kRows <= rows;
#pragma unroll
            for (int u = 0; u < LOADS; ++u) {
                // (a row behind the last is read as the first: its exponent is -inf)
                if (!whole && r0 + (u * 256 + tid) / NCH >= rows) from[u] = q0;
                next[u] = *reinterpret_cast<const u32x4_t*>(from[u]);
                from[u] += ahead;
                if constexpr (!EVEN) {
                    head[u] += heads_ahead;
                    if (head[u] >= G) {
                        head[u] -= G;
                        from[u] += wrap;
                    }
                }
            }
            // (what the load brings is first looked at in keep, behind the tile's products)
            const int r = min(r0 + lane, rows - 1);
            const int i = int(group.quot(uint32_t(r))), h = hk * G + r - i * G;
            next_lse = a.lse_in[int64_t(h) * a.tokens + s.q0 + i];
            next_limit = r0 + lane >= rows ? -1 : a.causal ? min(s.kv, s.kv - s.n + i + 1) : s.kv;
        };
        auto keep = [&](int buf) {
#pragma unroll
            for (int u = 0; u < LOADS; ++u) {
                const int e = u * 256 + tid, row = e / NCH;
                *reinterpret_cast<u32x4_t*>(
                    &lds[buf][row * D + ((tid % NCH ^ q_swizzle<D>(row)) * 8)]) = next[u];
            }
            if (wave == 0) {
                row_neg[buf][lane] =
                    next_lse == -INFINITY || next_limit < 0 ? -INFINITY : -next_lse * kLog2e;
                row_limit[buf][lane] = next_limit;
            }
        };
        // One tile of rows; CROSSED: some rows do not see all of the wave's keys.
        auto tile = [&](int buf, auto crossed_c) {
            constexpr bool CROSSED = decltype(crossed_c)::value;
            floatx4 sc[2][4];
            auto products = [&](int n) {
                const int row = 16 * n + col;
                const uint16_t* at = &lds[buf][row * D];
#pragma unroll
                for (int u = 0; u < 4; ++u) sc[n & 1][u] = floatx4{};
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    const bf16x8 q = *reinterpret_cast<const bf16x8*>(
                        at + (((4 * kt + g) ^ q_swizzle<D>(row)) * 8));
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        sc[n & 1][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            k[u][kt], q, sc[n & 1][u], 0, 0, 0);
                }
            };
            products(0);
#pragma unroll
            for (int n = 0; n < kRows / 16; ++n) {
                const int row = 16 * n + col;
                if (n + 1 < kRows / 16) products(n + 1);
                const float neg = row_neg[buf][row];
                const int limit = CROSSED ? row_limit[buf][row] - (t0 + 4 * g) : 0;
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float x = __builtin_amdgcn_exp2f(fmaf(sc[n & 1][u][e], c2, neg));
                        if (CROSSED) x = 16 * u + e < limit ? x : 0.f;
                        w[u][e] += x;
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
        };

        __syncthreads();  // the keys before have been computed
        if (r_first < rows) {
            load(r_first);
            keep(0);
        }
        int buf = 0;
        for (int r0 = r_first; r0 < rows; r0 += kRows) {
            __syncthreads();  // this tile is in LDS, the one before has been read
            const bool more = r0 + kRows < rows;
            if (more) load(r0 + kRows);
            if (r0 < r_clear)
                tile(buf, std::true_type{});
            else
                tile(buf, std::false_type{});
            buf ^= 1;
            if (more) keep(buf);
        }

        // Lane l's results are keys 16 u + 4 g + e of its column of rows: add the columns.
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int off = 1; off < 16; off <<= 1) w[u][e] += __shfl_xor(w[u][e], off);
        // Lane col of a group writes key 16 (col / 4) + 4 g + col % 4.
        float mine = 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) mine = col == 4 * u + e ? w[u][e] : mine;
        const int key = t0 + 16 * (col >> 2) + 4 * g + (col & 3);
        if (key < s.kv) {
            const int p = page_of(c.table, c.width, c.pages, b, key >> shift);
            if (p >= 0) {
                float* to = c.weights + (int64_t(p) * c.H + hk) * c.page + (key & mask);
                *to = a.accumulate ? *to + mine : mine;
            }
        }
    }
}

}  // namespace

hipError_t launch_weights_tiles(const PagedArgs& a, hipStream_t s) {
    const int span = a.cache.width * a.cache.page;
    const int keys = a.max_kv > 0 && a.max_kv < span ? a.max_kv : span;
    const int64_t pairs = int64_t(a.cache.B) * a.cache.H;
    int64_t strides = (keys + kKeys - 1) / kKeys;
    const int64_t most = (int64_t(1) << 22) / pairs;
    if (strides > most) strides = most < 1 ? 1 : most;
    const Div group = make_div(uint32_t(a.q_heads / a.cache.H));
    const int grid = int(pairs * strides);
    const bool even = kRows % group.d == 0;
    if (a.cache.d <= 64) {
        if (even)
            weights_tiles_kernel<64, true><<<grid, 256, 0, s>>>(a, int(strides), group);
        else
            weights_tiles_kernel<64, false><<<grid, 256, 0, s>>>(a, int(strides), group);
    } else {
        if (even)
            weights_tiles_kernel<128, true><<<grid, 256, 0, s>>>(a, int(strides), group);
        else
            weights_tiles_kernel<128, false><<<grid, 256, 0, s>>>(a, int(strides), group);
    }
    return hipGetLastError();
}

}  // namespace sparsp
