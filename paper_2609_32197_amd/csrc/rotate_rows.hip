// Rows of new tokens on their way to where attention reads them: rotated to their
// positions (Q, K), copied (V), into a strided tensor or into the pages of the cache.
//
// Pair p of a row at position x turns by the angle x f_p: (x1, x2) -> (x1 c - x2 s,
// x1 s + x2 c). The angle is reduced to a fraction of a turn in 64 bits (at a position of
// 10^6 a float32 product is off by 0.03 rad), sine and cosine are float32 of that
// fraction, and the rotated pair is rounded to the row's type once.
//
// Memory-bound: every row is read once and written once, and all heads of a token, of up
// to three tensors, share its angles. A workgroup takes `per` tokens: it finds where
// their rows go, computes cos and sin of their pairs into LDS, and then walks (token, head,
// unit) items; a unit is one access of V elements, or for rotated rows in the HALF layout
// the two accesses that hold a pair's ends, so a row may be rotated in place.
#include "cache_device.h"

namespace sparsp {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxPer = 16;         // tokens of a workgroup at most
constexpr int kTableFloats = 2048;  // float2 entries of cos and sin

struct Move {
    const char* src;
    int64_t src_head, src_token;  // bytes
    char* dst;
    int64_t dst_head, dst_token;
    Div heads, units;
    int paged, rotate;
};

struct Params {
    Move move[3];
    int moves, tokens, per, d, P, layout, inverse, wide;
    int axis_end[3];
    float factor;
    const void* positions;
    const float* inv_freq;
    sparsp_cache cache;
};

template <typename T>
__device__ __forceinline__ float up(T x);
template <>
__device__ __forceinline__ float up<float>(float x) { return x; }
template <>
__device__ __forceinline__ float up<uint16_t>(uint16_t x) { return bf16_bits_to_f32(x); }
template <typename T>
__device__ __forceinline__ T down(float x);
template <>
__device__ __forceinline__ float down<float>(float x) { return x; }
template <>
__device__ __forceinline__ uint16_t down<uint16_t>(float x) { return uint16_t(f32_to_bf16_bits(x)); }

template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
    T e[V];
};

// A workgroup's places: for each token the byte offset of its row in the pages, or -1.
// new_off is ascending, so the sequence of token t is the number of ends new_off[1..B] at
// or before t, counted by all threads at once.
template <typename T>
__device__ __forceinline__ void find_places(const Params& p, int t0, int count, int64_t* place,
                                            int* ends) {
    const sparsp_cache& c = p.cache;
    for (int k = 0; k < count; ++k) {
        int mine = 0;
        for (int b = threadIdx.x; b < c.B; b += kThreads) mine += c.new_off[b + 1] <= t0 + k;
        for (int off = 32; off; off >>= 1) mine += __shfl_xor(mine, off);
        if ((threadIdx.x & 63) == 0) ends[k * (kThreads / 64) + (threadIdx.x >> 6)] = mine;
    }
    __syncthreads();
    if (int(threadIdx.x) < count) {
        const int k = threadIdx.x;
        int b = 0;
        for (int w = 0; w < kThreads / 64; ++w) b += ends[k * (kThreads / 64) + w];
        int64_t at = -1;
        if (b < c.B) {
            const Seq s = sequence(c, p.tokens, b);
            const int i = t0 + k - s.q0, slot = s.kv - s.n + i;
            if (i >= 0 && i < s.n && slot >= 0) {
                const int page = page_of(c.table, c.width, c.pages, b, slot / c.page);
                if (page >= 0)
                    at = (int64_t(page) * c.H * c.page + slot % c.page) * c.d;
            }
        }
        place[k] = at < 0 ? -1 : at * int64_t(sizeof(T));
        if (at >= 0 && c.weights) {
            const int64_t row = at / c.d;  // (page * H) * rows of a page + row of the page
            for (int h = 0; h < c.H; ++h) c.weights[row + int64_t(h) * c.page] = 0.f;
        }
    }
}

template <typename T, int V, bool HALF, bool PAGED>
__global__ __launch_bounds__(kThreads) void rotate_rows_kernel(const Params p) {
    __shared__ float2 turn[kTableFloats];
    __shared__ int64_t place[kMaxPer];
    __shared__ int ends[kMaxPer * (kThreads / 64)];
    const int t0 = blockIdx.x * p.per, count = min(p.per, p.tokens - t0);
    if (PAGED) find_places<T>(p, t0, count, place, ends);
    for (int e = threadIdx.x; e < count * p.P; e += kThreads) {
        const int k = e / p.P, pr = e % p.P;
        const int axis = (pr >= p.axis_end[0]) + (pr >= p.axis_end[1]);
        const int64_t at = int64_t(axis) * p.tokens + t0 + k;
        const double x = p.wide ? double(static_cast<const int64_t*>(p.positions)[at])
                                : double(static_cast<const int32_t*>(p.positions)[at]);
        constexpr double kInvTurn = 0.15915494309189533576888;  // 1 / (2 pi)
        double r = x * double(p.inv_freq[pr]) * kInvTurn;
        r -= rint(r);
        float s, c;
        sincospif(float(2.0 * r), &s, &c);
        turn[e] = make_float2(c * p.factor, (p.inverse ? -s : s) * p.factor);
    }
    __syncthreads();

    for (int m = 0; m < p.moves; ++m) {
        const Move& mv = p.move[m];
        const uint32_t heads = mv.heads.d, units = mv.units.d;
        const uint32_t items = uint32_t(count) * heads * units;
        for (uint32_t it = threadIdx.x; it < items; it += kThreads) {
            const uint32_t row = mv.units.quot(it), u = it - row * units;
            const uint32_t k = mv.heads.quot(row), h = row - k * heads;
            const char* src = mv.src + int64_t(h) * mv.src_head + int64_t(t0 + k) * mv.src_token;
            char* dst = mv.dst;
            if (PAGED && mv.paged) {
                if (place[k] < 0) continue;
                dst += place[k] + int64_t(h) * p.cache.page * p.d * int64_t(sizeof(T));
            } else {
                dst += int64_t(h) * mv.dst_head + int64_t(t0 + k) * mv.dst_token;
            }
            using Unit = Vec<T, V>;
            const Unit* in = reinterpret_cast<const Unit*>(src);
            Unit* out = reinterpret_cast<Unit*>(dst);
            const uint32_t turned = mv.rotate ? p.P * (HALF ? 1 : 2) / V : 0;  // units that rotate
            if (u >= turned) {
                const uint32_t at = u + (HALF ? turned : 0);
                out[at] = in[at];
                continue;
            }
            const float2* cs = turn + k * p.P;
            if (HALF) {
                const Unit a = in[u], b = in[u + turned];
                Unit ya, yb;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float2 t = cs[u * V + e];
                    const float x1 = up<T>(a.e[e]), x2 = up<T>(b.e[e]);
                    ya.e[e] = down<T>(x1 * t.x - x2 * t.y);
                    yb.e[e] = down<T>(x1 * t.y + x2 * t.x);
                }
                out[u] = ya;
                out[u + turned] = yb;
            } else if constexpr (V >= 2) {
                const Unit a = in[u];
                Unit y;
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    const float2 t = cs[(u * V + e) / 2];
                    const float x1 = up<T>(a.e[e]), x2 = up<T>(a.e[e + 1]);
                    y.e[e] = down<T>(x1 * t.x - x2 * t.y);
                    y.e[e + 1] = down<T>(x1 * t.y + x2 * t.x);
                }
                out[u] = y;
            }
        }
    }
}

template <typename T, int V, bool HALF>
hipError_t launch_v(const RotateArgs& a, Params& p, bool paged, hipStream_t s) {
    for (int m = 0; m < p.moves; ++m) {
        const RowMove& r = a.move[m];
        const bool two = r.rotate && HALF;  // a rotating unit covers two accesses
        p.move[m].units = make_div(uint32_t(two ? (a.d - a.rot / 2) / V : a.d / V));
    }
    const int grid = (a.tokens + p.per - 1) / p.per;
    if (paged)
        rotate_rows_kernel<T, V, HALF, true><<<grid, kThreads, 0, s>>>(p);
    else
        rotate_rows_kernel<T, V, HALF, false><<<grid, kThreads, 0, s>>>(p);
    return hipGetLastError();
}

template <typename T, int V>
hipError_t launch_layout(const RotateArgs& a, Params& p, bool paged, hipStream_t s) {
    if (a.rot && a.layout == SPARSP_ROPE_HALF) return launch_v<T, V, true>(a, p, paged, s);
    return launch_v<T, V, false>(a, p, paged, s);
}

}  // namespace

hipError_t launch_rotate_rows(const RotateArgs& a, hipStream_t s) {
    const int size = a.bf16 ? 2 : 4;
    Params p = {};
    p.moves = a.moves;
    bool paged = false;
    int heads = 0;
    for (int m = 0; m < a.moves; ++m) {
        const RowMove& r = a.move[m];
        p.move[m] = {static_cast<const char*>(r.src), r.src_head * size, r.src_token * size,
                     static_cast<char*>(r.dst),       r.dst_head * size, r.dst_token * size,
                     make_div(uint32_t(r.heads)),     make_div(1),       r.paged,
                     r.rotate};
        paged |= r.paged;
        heads += r.heads;
    }
    p.tokens = a.tokens;
    p.d = a.d;
    p.P = a.rot / 2;
    p.layout = a.layout;
    p.inverse = a.inverse;
    p.wide = a.wide;
    for (int x = 0; x < 3; ++x) p.axis_end[x] = a.axis_end[x];
    p.factor = a.factor;
    p.positions = a.positions;
    p.inv_freq = a.inv_freq;
    p.cache = a.cache;
    // Tokens of a workgroup: enough to fill the GPU four times with one each, more only
    // where there are so many that the angles are better shared by longer runs.
    p.per = 1;
    while (p.per < kMaxPer && a.tokens / (2 * p.per) >= 1024 &&
           (p.P == 0 || 2 * p.per * p.P <= kTableFloats))
        p.per *= 2;
    // The widest access that divides the rotated part (its half, where a unit is two
    // accesses) and the rest.
    const int part = a.rot == 0 ? a.d : a.layout == SPARSP_ROPE_HALF ? a.rot / 2 : a.rot;
    const int all = part | a.d | (a.d - a.rot);
    if (a.bf16) {
        if (all % 8 == 0) return launch_layout<uint16_t, 8>(a, p, paged, s);
        if (all % 4 == 0) return launch_layout<uint16_t, 4>(a, p, paged, s);
        if (all % 2 == 0) return launch_layout<uint16_t, 2>(a, p, paged, s);
        return launch_layout<uint16_t, 1>(a, p, paged, s);
    }
    if (all % 4 == 0) return launch_layout<float, 4>(a, p, paged, s);
    if (all % 2 == 0) return launch_layout<float, 2>(a, p, paged, s);
    return launch_layout<float, 1>(a, p, paged, s);
}

}  // namespace sparsp
