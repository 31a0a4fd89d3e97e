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
    int tokens_first;  // a head's rows lie token after token
};

struct Params {
    Move move[3];
    int moves, tokens, d, P, inverse, wide, stream;
    Div per;  // tokens of a workgroup
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
// Rows that no cache can hold until they are read again leave none of themselves in one.
template <typename T, int V>
__device__ __forceinline__ Vec<T, V> get(const Vec<T, V>* p, bool stream) {
    if constexpr (sizeof(T) * V == 16)
        if (stream)
            return __builtin_bit_cast(Vec<T, V>, load_nt(reinterpret_cast<const char*>(p)));
    return *p;
}
template <typename T, int V>
__device__ __forceinline__ void put(Vec<T, V>* p, Vec<T, V> x, bool stream) {
    if constexpr (sizeof(T) * V == 16)
        if (stream) return store_nt(reinterpret_cast<char*>(p), __builtin_bit_cast(uint4, x));
    *p = x;
}

// A workgroup's places: for each token the byte offset of its row in the pages, or what place_of
// has for none. A wave takes a token.
template <typename T>
__device__ __forceinline__ void find_places(const Params& p, int t0, int count, int64_t* place) {
    const sparsp_cache& c = p.cache;
    const int lane = threadIdx.x & 63;
    for (int k = threadIdx.x >> 6; k < count; k += kThreads / 64) {
        const int64_t row = place_of(c, p.tokens, t0 + k, lane);
        if (lane == 0) place[k] = row < 0 ? row : row * c.d * int64_t(sizeof(T));
        if (row >= 0 && c.weights)
            for (int h = lane; h < c.H; h += 64) c.weights[row + int64_t(h) * c.page] = 0.f;
    }
}

template <typename T, int V, bool HALF, bool PAGED>
__global__ __launch_bounds__(kThreads) void rotate_rows_kernel(const Params p) {
    __shared__ float2 turn[kTableFloats];
    __shared__ int64_t place[kMaxPer];
    const int t0 = blockIdx.x * p.per.d, count = min(int(p.per.d), p.tokens - t0);
    if (PAGED) find_places<T>(p, t0, count, place);
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
    const bool stream = p.stream;

    for (int m = 0; m < p.moves; ++m) {
        const Move& mv = p.move[m];
        const uint32_t heads = mv.heads.d, units = mv.units.d;
        // Rows are walked in the order in which they lie.
        const uint32_t items = (mv.tokens_first ? p.per.d : uint32_t(count)) * heads * units;
        for (uint32_t it = threadIdx.x; it < items; it += kThreads) {
            const uint32_t row = mv.units.quot(it), u = it - row * units;
            uint32_t k, h;
            if (mv.tokens_first) {
                h = p.per.quot(row);
                k = row - h * p.per.d;
                if (k >= uint32_t(count)) continue;
            } else {
                k = mv.heads.quot(row);
                h = row - k * heads;
            }
            const char* src = mv.src + int64_t(h) * mv.src_head + int64_t(t0 + k) * mv.src_token;
            char* dst = mv.dst;
            if (PAGED && place[k] == kNoSequence) continue;
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
                put(out + at, get(in + at, stream), stream);
                continue;
            }
            const float2* cs = turn + k * p.P;
            if (HALF) {
                const Unit a = get(in + u, stream), b = get(in + u + turned, stream);
                Unit ya, yb;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float2 t = cs[u * V + e];
                    const float x1 = up<T>(a.e[e]), x2 = up<T>(b.e[e]);
                    ya.e[e] = down<T>(x1 * t.x - x2 * t.y);
                    yb.e[e] = down<T>(x1 * t.y + x2 * t.x);
                }
                put(out + u, ya, stream);
                put(out + u + turned, yb, stream);
            } else if constexpr (V >= 2) {
                const Unit a = get(in + u, stream);
                Unit y;
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    const float2 t = cs[(u * V + e) / 2];
                    const float x1 = up<T>(a.e[e]), x2 = up<T>(a.e[e + 1]);
                    y.e[e] = down<T>(x1 * t.x - x2 * t.y);
                    y.e[e + 1] = down<T>(x1 * t.y + x2 * t.x);
                }
                put(out + u, y, stream);
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
    const int grid = (a.tokens + int(p.per.d) - 1) / int(p.per.d);
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
                     r.rotate,                        r.src_token < r.src_head};
        paged |= r.paged;
        heads += r.heads;
    }
    p.tokens = a.tokens;
    p.d = a.d;
    p.P = a.rot / 2;
    p.inverse = a.inverse;
    p.wide = a.wide;
    for (int x = 0; x < 3; ++x) p.axis_end[x] = a.axis_end[x];
    p.factor = a.factor;
    p.positions = a.positions;
    p.inv_freq = a.inv_freq;
    p.cache = a.cache;
    // Tokens of a workgroup: enough to fill the GPU four times with one each, more only
    // where there are so many that the angles are better shared by longer runs.
    int per = 1;
    while (per < kMaxPer && a.tokens / (2 * per) >= 1024 &&
           (p.P == 0 || 2 * per * p.P <= kTableFloats))
        per *= 2;
    p.per = make_div(uint32_t(per));
    p.stream = int64_t(heads) * a.tokens * a.d * size > (int64_t(256) << 20);
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
