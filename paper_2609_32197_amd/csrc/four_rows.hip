// New tokens into a cache held in 4 bits, and back (the format is stated in paged_four.h).
//
// With a the largest magnitude of 32 channels the scale is 2^e, e = floor(log2 a) - 2, so that every
// magnitude is below 8 of it; a code is the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even one,
// 6 for what is larger. All that is exact: e comes from the exponents' bits alone, and a magnitude is
// rounded once, by the conversion instruction.
//
// K is rotated on the way in 64 bits. A code jumps by a third of its value where a value crosses a
// border, so that with 32 bits it would depend, once in some 10^6 values, on the rounding of a
// product; in 64 bits a value is as near to a border once in 10^10. Q, which stays in its own type,
// is rotated in float32 as by sparsp_rope.
//
// A thread takes eight channels, a dword of codes; four neighbours share a scale. A workgroup takes
// `per` tokens and shares their cosines and sines over all heads, as in rotate_rows.hip. Prompts of
// 8,461 tokens, 20 heads of Q, K and V of 128, half of each rotated: 56 us, 3.4 TB/s, the vector unit
// busy with the 64-bit rotation, which K's channels behind the rotated ones go through too, turned by
// nothing (with codes by comparisons in 64 bits instead of the conversion instruction 77 us); the same
// read back 25 us, 4.4 TB/s.
//
// `per` is chosen by the tokens alone, whatever the heads; many heads would have shorter runs and few
// longer ones. Append and read, us, the same data over and over, at most 4, 8 and 16 tokens:
//   20 heads of Q, K and V, 8,461 tokens    45 + 23    49 + 24    49 + 24 (the rule takes 8)
//   20 heads,              50,895 tokens   258 + 159  271 + 164  287 + 169
//   32 and 8 heads,       111,075 tokens   450 + 130  474 + 136  500 + 141
//   8 and 2 heads of 64,  111,075 tokens   126 + 34   104 + 30    94 + 26
//   one head,             111,075 tokens    96 + 34    78 + 30    69 + 26
#include "cache_device.h"
#include "paged_four.h"

namespace sparsp {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxPer = 16;        // tokens of a workgroup at most
constexpr int kTablePairs = 1152;  // cosines and sines held
constexpr int kStill = 8;          // behind a token's pairs: some that do not turn

struct Side {
    const char* src;
    int64_t head, token;  // bytes
    uint8_t *codes, *scales;
};
struct Params {
    Side kv[2];
    const char* q;
    char* q_out;
    int64_t q_head, q_token, out_head, out_token;
    int q_heads;
    int tokens, P, inverse, wide;
    Div per, units, q_units, q_heads_div, heads;
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
__device__ __forceinline__ uint16_t down<uint16_t>(float x) {
    return __builtin_bit_cast(uint16_t, __bf16(x));
}

template <typename T, int V>
struct alignas(sizeof(T) * V < 16 ? sizeof(T) * V : 16) Vec {
    T e[V];
};
template <typename T, int V>
__device__ __forceinline__ Vec<T, V> get(const char* row, int ch) {
    return *reinterpret_cast<const Vec<T, V>*>(row + ch * int(sizeof(T)));
}

// Codes of eight channels and the scale's exponent byte, which the four lanes of a group share. top:
// the largest magnitude's bits, with the exponent (of a float64) from bit `at` on; an infinity or a
// NaN gets the scale that stands for NaN.
template <int AT, int BIAS>
__device__ __forceinline__ int group_exponent(uint32_t top, uint32_t* scale) {
    top = max(top, uint32_t(__shfl_xor(int(top), 1)));
    top = max(top, uint32_t(__shfl_xor(int(top), 2)));
    const int e = min(max(int(top >> AT) - BIAS - 2, -125), 125);
    *scale = int(top >> AT) > 2 * BIAS ? 255u : uint32_t(e + 127);
    return e;
}
// The conversion divides by the scale, rounds to the nearest code, ties to the even one, and cuts to 6.
__device__ __forceinline__ uint32_t codes_of(const float (&y)[8], float scale) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
}
__device__ __forceinline__ uint32_t quantise(const float (&y)[8], uint32_t* scale) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(y[e]) & 0x7fffffffu);
    const int exponent = group_exponent<23, 127>(top, scale);
    const uint32_t codes = codes_of(y, __uint_as_float(uint32_t(exponent + 127) << 23));
    return *scale == 255 ? 0u : codes;
}
// A float64 over 2^e is cut to float32, with the last bit set if that leaves anything out: such a
// number is on the same side of every border as the float64. (Borders have few bits; what is below
// 2^-126 of the scale becomes 0.)
__device__ __forceinline__ uint32_t quantise(double (&y)[8], uint32_t* scale) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, uint32_t(__double2hiint(y[e])) & 0x7fffffffu);
    const int exponent = group_exponent<20, 1023>(top, scale);
    if (exponent == 125) {  // a row may be turned beyond what a float32 over 2^e holds
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = fmin(fmax(y[e], -0x1p130), 0x1p130);
    }
    const int shift = (1023 - 127 + exponent) << 20;
    float m[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t hi = uint32_t(__double2hiint(y[e])), lo = uint32_t(__double2loint(y[e]));
        const int high = max(int(hi & 0x7fffffffu) - shift, 0);  // exponent in place, 20 bits behind it
        const uint32_t left = min(lo & 0x1fffffffu, 1u);
        m[e] = __uint_as_float((hi & 0x80000000u) | __builtin_amdgcn_alignbit(high, lo, 29) | left);
    }
    const uint32_t codes = codes_of(m, 1.f);
    return *scale == 255 ? 0u : codes;
}

template <typename T, int V, bool HALF>
__global__ __launch_bounds__(kThreads) void four_append_kernel(const Params p) {
    __shared__ double2 turn[kTablePairs];
    __shared__ int64_t place[kMaxPer];
    const sparsp_cache& c = p.cache;
    const int t0 = blockIdx.x * p.per.d, count = min(int(p.per.d), p.tokens - t0);
    const int lane = threadIdx.x & 63, row_pairs = p.P + kStill;
    for (int k = threadIdx.x >> 6; k < count; k += kThreads / 64) {
        const int64_t row = place_of(c, p.tokens, t0 + k, lane);
        if (lane == 0) place[k] = row;
    }
    for (int e = threadIdx.x; p.P > 0 && e < count * row_pairs; e += kThreads) {
        const int k = e / row_pairs, pr = e % row_pairs;
        if (pr >= p.P) {
            turn[e] = make_double2(1.0, 0.0);
            continue;
        }
        const int axis = (pr >= p.axis_end[0]) + (pr >= p.axis_end[1]);
        const int64_t at = int64_t(axis) * p.tokens + t0 + k;
        const double x = p.wide ? double(static_cast<const int64_t*>(p.positions)[at])
                                : double(static_cast<const int32_t*>(p.positions)[at]);
        constexpr double kInvTurn = 0.15915494309189533576888;  // 1 / (2 pi)
        double r = x * double(p.inv_freq[pr]) * kInvTurn;
        r -= rint(r);
        double s, cs;
        sincospi(2.0 * r, &s, &cs);
        turn[e] = make_double2(cs * p.factor, (p.inverse ? -s : s) * p.factor);
    }
    __syncthreads();

    // Q: units of V pairs, then of V channels that stay.
    if (p.q) {
        const uint32_t turned = HALF ? p.P / V : 2 * p.P / V;
        const uint32_t items = uint32_t(count) * p.q_heads * p.q_units.d;
        for (uint32_t it = threadIdx.x; it < items; it += kThreads) {
            const uint32_t row = p.q_units.quot(it), u = it - row * p.q_units.d;
            const uint32_t k = p.q_heads_div.quot(row), h = row - k * p.q_heads;
            if (place[k] == kNoSequence) continue;
            const char* in = p.q + int64_t(h) * p.q_head + int64_t(t0 + k) * p.q_token;
            char* out = p.q_out + int64_t(h) * p.out_head + int64_t(t0 + k) * p.out_token;
            const double2* cs = turn + k * row_pairs;
            auto put = [&](int ch, const Vec<T, V>& x) {
                *reinterpret_cast<Vec<T, V>*>(out + ch * int(sizeof(T))) = x;
            };
            if (u >= turned) {
                const int ch = int(u + (HALF ? turned : 0)) * V;
                put(ch, get<T, V>(in, ch));
            } else if (HALF) {
                const int ch = int(u) * V;
                const Vec<T, V> a = get<T, V>(in, ch), b = get<T, V>(in, ch + p.P);
                Vec<T, V> ya, yb;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float tc = float(cs[ch + e].x), ts = float(cs[ch + e].y);
                    const float x1 = up<T>(a.e[e]), x2 = up<T>(b.e[e]);
                    ya.e[e] = down<T>(x1 * tc - x2 * ts);
                    yb.e[e] = down<T>(x1 * ts + x2 * tc);
                }
                put(ch, ya);
                put(ch + p.P, yb);
            } else if constexpr (V >= 2) {
                const int ch = int(u) * V;
                const Vec<T, V> a = get<T, V>(in, ch);
                Vec<T, V> y;
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    const double2 t = cs[(ch + e) / 2];
                    const float tc = float(t.x), ts = float(t.y);
                    const float x1 = up<T>(a.e[e]), x2 = up<T>(a.e[e + 1]);
                    y.e[e] = down<T>(x1 * tc - x2 * ts);
                    y.e[e + 1] = down<T>(x1 * ts + x2 * tc);
                }
                put(ch, y);
            }
        }
    }

    // K and V: units of eight channels; a row's units fill whole groups of four lanes.
    const uint32_t items = uint32_t(count) * c.H * p.units.d;
    for (uint32_t it = threadIdx.x; it < items; it += kThreads) {
        const uint32_t row = p.units.quot(it), u = it - row * p.units.d;
        const uint32_t k = p.heads.quot(row), h = row - k * c.H;
        const int64_t at = place[k];
        if (at < 0) continue;
        const char* kin = p.kv[0].src + int64_t(h) * p.kv[0].head + int64_t(t0 + k) * p.kv[0].token;
        const char* vin = p.kv[1].src + int64_t(h) * p.kv[1].head + int64_t(t0 + k) * p.kv[1].token;
        const int ch = int(u) * 8;
        const Vec<T, 8> x = get<T, 8>(kin, ch), w = get<T, 8>(vin, ch);
        uint32_t scale[2], codes[2];
        if (p.P > 0) {
            const double2* cs = turn + k * row_pairs;
            double y[8];
            if (HALF) {
#pragma unroll
                for (int e0 = 0; e0 < 8; e0 += V) {
                    const int first = ch + e0;
                    const bool turns = first < 2 * p.P, behind = turns && first >= p.P;
                    const int far_at = !turns ? first : behind ? first - p.P : first + p.P;
                    const Vec<T, V> far = get<T, V>(kin, far_at);
                    const double2* t = cs + (!turns ? p.P : behind ? far_at : first);
                    const uint32_t flip = behind ? 0u : 0x80000000u;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float z = __uint_as_float(__float_as_uint(up<T>(far.e[e])) ^ flip);
                        y[e0 + e] = double(up<T>(x.e[e0 + e])) * t[e].x + double(z) * t[e].y;
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const double2 t = cs[min((ch + e) / 2, p.P)];
                    const double x1 = double(up<T>(x.e[e])), x2 = double(up<T>(x.e[e + 1]));
                    y[e] = x1 * t.x - x2 * t.y;
                    y[e + 1] = x1 * t.y + x2 * t.x;
                }
            }
            codes[0] = quantise(y, scale);
        } else {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = up<T>(x.e[e]);
            codes[0] = quantise(y, scale);
        }
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = up<T>(w.e[e]);
        codes[1] = quantise(y, scale + 1);
        const int64_t to = at + int64_t(h) * c.page;  // (c.page a power of two, heads [page] rows)
        const int slot = int(to & (c.page - 1));
        const int64_t scale_at = (to - slot) * (c.d / 32) + int64_t(u / 4) * c.page + slot;
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            *reinterpret_cast<uint32_t*>(p.kv[side].codes + to * (c.d / 2) + 4 * u) = codes[side];
            if (u % 4 == 0) p.kv[side].scales[scale_at] = uint8_t(scale[side]);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void four_read_kernel(const Params p) {
    __shared__ int64_t place[kMaxPer];
    const sparsp_cache& c = p.cache;
    const int t0 = blockIdx.x * p.per.d, count = min(int(p.per.d), p.tokens - t0);
    const int lane = threadIdx.x & 63;
    for (int k = threadIdx.x >> 6; k < count; k += kThreads / 64) {
        const int64_t row = place_of(c, p.tokens, t0 + k, lane);
        if (lane == 0) place[k] = row;
    }
    __syncthreads();
    const uint32_t items = uint32_t(count) * c.H * p.units.d;
    for (uint32_t it = threadIdx.x; it < items; it += kThreads) {
        const uint32_t row = p.units.quot(it), u = it - row * p.units.d;
        const uint32_t k = p.heads.quot(row), h = row - k * c.H;
        const int64_t at = place[k];
        if (at == kNoSequence) continue;
        const int64_t from = max(at, int64_t(0)) + int64_t(h) * c.page;
        const int slot = int(from & (c.page - 1));
        const int64_t scale_at = (from - slot) * (c.d / 32) + int64_t(u / 4) * c.page + slot;
        uint32_t codes[2], scale[2];
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            codes[side] = scale[side] = 0;
            if (at < 0) continue;
            const Side& sd = p.kv[side];
            codes[side] = *reinterpret_cast<const uint32_t*>(sd.codes + from * (c.d / 2) + 4 * u);
            scale[side] = sd.scales[scale_at];
        }
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const Side& sd = p.kv[side];
            const uint4 x = four_octet(codes[side], __uint_as_float(scale[side] << 23));
            char* out = const_cast<char*>(sd.src) + int64_t(h) * sd.head + int64_t(t0 + k) * sd.token;
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<uint4*>(out + 16 * u) = x;
            } else {
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    uint4 y;
                    y.x = w[2 * e] << 16;
                    y.y = w[2 * e] & 0xffff0000u;
                    y.z = w[2 * e + 1] << 16;
                    y.w = w[2 * e + 1] & 0xffff0000u;
                    *reinterpret_cast<uint4*>(out + 32 * u + 16 * e) = y;
                }
            }
        }
    }
}

Params params(const FourArgs& f, int pairs) {
    const RotateArgs& a = f.rows;
    const int size = a.bf16 ? 2 : 4;
    Params p = {};
    for (int n = 0; n < 2; ++n)
        p.kv[n] = {static_cast<const char*>(a.move[n].src), a.move[n].src_head * size,
                   a.move[n].src_token * size,
                   static_cast<uint8_t*>(n == 0 ? a.cache.K : a.cache.V),
                   n == 0 ? f.k_scales : f.v_scales};
    p.tokens = a.tokens;
    p.P = pairs;
    p.cache = a.cache;
    p.units = make_div(uint32_t(a.cache.d / 8));
    p.heads = make_div(uint32_t(a.cache.H));
    // As in rotate_rows.hip: enough workgroups to fill the GPU four times, then longer runs (figures
    // at the top).
    int per = 1;
    while (per < kMaxPer && a.tokens / (2 * per) >= 1024 &&
           (pairs == 0 || 2 * per * (pairs + kStill) <= kTablePairs))
        per *= 2;
    p.per = make_div(uint32_t(per));
    return p;
}

template <typename T, int V>
void launch_append(const Params& p, bool half, hipStream_t s) {
    const int grid = (p.tokens + int(p.per.d) - 1) / int(p.per.d);
    if (half)
        four_append_kernel<T, V, true><<<grid, kThreads, 0, s>>>(p);
    else
        four_append_kernel<T, V, false><<<grid, kThreads, 0, s>>>(p);
}
template <typename T>
void launch_width(const Params& p, bool half, int width, hipStream_t s) {
    if (width == 8) return launch_append<T, 8>(p, half, s);
    if (width == 4) return launch_append<T, 4>(p, half, s);
    if (width == 2) return launch_append<T, 2>(p, half, s);
    launch_append<T, 1>(p, half, s);
}

}  // namespace

hipError_t launch_four_append(const FourArgs& f, hipStream_t s) {
    const RotateArgs& a = f.rows;
    const int size = a.bf16 ? 2 : 4;
    Params p = params(f, a.rot / 2);
    p.inverse = a.inverse;
    p.wide = a.wide;
    for (int x = 0; x < 3; ++x) p.axis_end[x] = a.axis_end[x];
    p.factor = a.factor;
    p.positions = a.positions;
    p.inv_freq = a.inv_freq;
    const bool half = a.rot && a.layout == SPARSP_ROPE_HALF;
    // The widest unit that divides the rotated part (its half, where a pair lies in two units).
    const int part = half ? a.rot / 2 : a.rot;
    int width = 8;
    while (part % width) width /= 2;
    if (a.moves == 3) {
        const RowMove& q = a.move[2];
        p.q = static_cast<const char*>(q.src);
        p.q_out = static_cast<char*>(q.dst);
        p.q_head = q.src_head * size;
        p.q_token = q.src_token * size;
        p.out_head = q.dst_head * size;
        p.out_token = q.dst_token * size;
        p.q_heads = q.heads;
        p.q_heads_div = make_div(uint32_t(q.heads));
        p.q_units = make_div(uint32_t((a.cache.d - (half ? a.rot / 2 : 0)) / width));
    }
    if (a.bf16)
        launch_width<uint16_t>(p, half, width, s);
    else
        launch_width<float>(p, half, width, s);
    return hipGetLastError();
}

hipError_t launch_four_read(const FourArgs& f, hipStream_t s) {
    const Params p = params(f, 0);
    const int grid = (p.tokens + int(p.per.d) - 1) / int(p.per.d);
    if (f.rows.bf16)
        four_read_kernel<uint16_t><<<grid, kThreads, 0, s>>>(p);
    else
        four_read_kernel<float><<<grid, kThreads, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace sparsp
