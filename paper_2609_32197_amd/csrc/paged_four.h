// What the attention kernels need of a cache held in 4 bits.
//
// A code is sign, two bits of exponent, one of mantissa (0, 0.5, 1, 1.5, 2, 3, 4, 6); 32 channels of a
// token share a power of two. What a code stands for is exact in bf16, so the products are those of
// a bf16 cache: v_cvt_scalef32_pk_bf16_fp4 makes two values of a byte, scale included (a scale of 255
// makes NaN), and the matrix cores take them from there.
//
// Codes lie as [pages, H, page, d / 2], the even channel in a byte's low half; scales as [pages, H,
// d / 32, page], so that the scales of consecutive keys, which a lane needs together, are one load.
#pragma once

#include "paged_tiles.h"

namespace sparsp {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));

// The scale byte e of w as the float that the conversion takes (its exponent).
__device__ __forceinline__ float four_scale(uint32_t w, int e) {
    return __uint_as_float(__builtin_amdgcn_ubfe(w, 8 * e, 8) << 23);
}
// Byte BYTE of w: two channels, bf16.
template <int BYTE>
__device__ __forceinline__ uint32_t four_pair(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, BYTE));
}
// Eight channels.
__device__ __forceinline__ uint4 four_octet(uint32_t w, float scale) {
    return make_uint4(four_pair<0>(w, scale), four_pair<1>(w, scale), four_pair<2>(w, scale),
                      four_pair<3>(w, scale));
}

// First row of head hk on `page` (-1: page 0, whose values the callers mask).
__device__ __forceinline__ int64_t four_head(const sparsp_cache& c, int page, int hk) {
    return int64_t(page < 0 ? 0 : page) * c.H + hk;
}

// Rows of Q in float32 (TERMS 3) enter the products as three bf16 each, which hold them whole, and so
// do probabilities; rows in bf16 (TERMS 1) as they are, and probabilities as two.
template <int TERMS>
struct Four {};

// Layout as for bf16 (paged_tiles.h), but for the order of the channels in a score's sum: lane group
// g takes D / 4 consecutive ones, 16 or 8 bytes of codes in one load and one scale.
template <int TERMS, int D>
struct TileMath<Four<TERMS>, D> {
    static constexpr int KEYS = 32, U = 2, PER = 8, KT = D / 32, DV = D / 16;
    static constexpr int PT = TERMS == 1 ? 2 : 3;  // terms of a probability
    struct KTile { uint32_t k[U][KT], scales[2]; };
    struct QTile { bf16x8 q[TERMS][KT]; };
    struct VTile { uint32_t r[8], scales[2]; };

    static __device__ __forceinline__ const PagedArgs& source(const PagedArgs& a) { return a; }
    static __device__ __forceinline__ int key_of(int g, int v) { return 8 * g + v; }
    static __device__ __forceinline__ int k_group(int lane) { return 8 * ((lane & 15) >> 2); }
    static __device__ __forceinline__ int v_group(int lane) { return 8 * (lane >> 4); }

    // The scales of eight keys from `key` on, of channel ch's 32.
    static __device__ __forceinline__ void load_scales(const sparsp_cache& c, const uint8_t* scales,
                                                       uint32_t (&to)[2], int64_t head, int ch,
                                                       int key) {
        const u32x2_t x = *reinterpret_cast<const u32x2_t*>(
            scales + (head * (c.d >> 5) + (ch >> 5)) * c.page + (key & (c.page - 1)));
        to[0] = x.x;
        to[1] = x.y;
    }
    static __device__ __forceinline__ void load_k(const PagedArgs& a, KTile& t, int page, int hk,
                                                  int t0, int lane) {
        const sparsp_cache& c = a.cache;
        const int own = (D / 4) * (lane >> 4), ch = own < c.d ? own : 0;
        const int key = t0 + k_group(lane);
        const int64_t head = four_head(c, page, hk);
        const uint8_t* p = static_cast<const uint8_t*>(c.K) +
                           ((head * c.page + (key & (c.page - 1)) + (lane & 3)) * c.d + ch) / 2;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if constexpr (KT == 4) {
                const uint4 x = *reinterpret_cast<const uint4*>(p + 2 * u * c.d);
                t.k[u][0] = x.x;
                t.k[u][1] = x.y;
                t.k[u][2] = x.z;
                t.k[u][3] = x.w;
            } else {
                const uint2 x = *reinterpret_cast<const uint2*>(p + 2 * u * c.d);
                t.k[u][0] = x.x;
                t.k[u][1] = x.y;
            }
        }
        load_scales(c, a.k_scales, t.scales, head, ch, key);
    }
    static __device__ __forceinline__ void load_row(QTile& t, const void* Q, int64_t at, bool live,
                                                    int d, int lane) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            const int ch = (D / 4) * (lane >> 4) + 8 * kt;
            if constexpr (TERMS == 1) {
                uint4 x = make_uint4(0, 0, 0, 0);
                if (live && ch < d)
                    x = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(Q) + at + ch);
                t.q[0][kt] = __builtin_bit_cast(bf16x8, x);
            } else {
                floatx8 x = {};
                if (live && ch < d)
                    x = *reinterpret_cast<const floatx8*>(static_cast<const float*>(Q) + at + ch);
                split<TERMS>(x, [&](int term, bf16x8 y) { t.q[term][kt] = y; });
            }
        }
    }
    template <int N, typename Put>
    static __device__ __forceinline__ void split(floatx8 x, Put put) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const bf16x8 y = __builtin_convertvector(x, bf16x8);
            put(n, y);
            x -= __builtin_convertvector(y, floatx8);
        }
    }
    static __device__ __forceinline__ void scores(const KTile& k, const QTile& q, floatx4 (&s)[U]) {
        const int own = __lane_id() & 3;
        float scale[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            s[u] = floatx4{};
            scale[u] = four_scale(k.scales[u], own);
        }
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bf16x8 x = __builtin_bit_cast(bf16x8, four_octet(k.k[u][kt], scale[u]));
#pragma unroll
                for (int n = TERMS - 1; n >= 0; --n)
                    s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q.q[n][kt], s[u], 0, 0, 0);
            }
    }
    static __device__ __forceinline__ void load_v(const PagedArgs& a, VTile& t, int page, int hk,
                                                  int t0, int lane) {
        const sparsp_cache& c = a.cache;
        const int own = DV * (lane & 15), ch = own < c.d ? own : 0;
        const int key = t0 + v_group(lane);
        const int64_t head = four_head(c, page, hk);
        const uint8_t* p = static_cast<const uint8_t*>(c.V) +
                           ((head * c.page + (key & (c.page - 1))) * c.d + ch) / 2;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            t.r[e] = DV == 8 ? *reinterpret_cast<const uint32_t*>(p + e * (c.d / 2))
                             : *reinterpret_cast<const uint16_t*>(p + e * (c.d / 2));
        load_scales(c, a.v_scales, t.scales, head, ch, key);
    }
    // Keys from `live` on (of this lane's eight) become zero: codes, and scales, which may say NaN.
    static __device__ __forceinline__ void clear_v(VTile& t, int live) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            t.r[e] = e < live ? t.r[e] : 0u;
            t.scales[e / 4] = e < live ? t.scales[e / 4] : t.scales[e / 4] & ~(255u << (e % 4 * 8));
        }
    }
    struct P { bf16x8 p[PT]; };
    static __device__ __forceinline__ P pack(const float (&p)[PER]) {
        floatx8 x;
#pragma unroll
        for (int v = 0; v < 8; ++v) x[v] = p[v];
        P r;
        split<PT>(x, [&](int term, bf16x8 y) { r.p[term] = y; });
        return r;
    }
    template <int NC>
    static __device__ __forceinline__ void output(const VTile& v, const P (&p)[NC],
                                                  floatx4 (&acc)[NC][DV]) {
        uint32_t r[8][DV / 2];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float scale = four_scale(v.scales[e / 4], e % 4);
            r[e][0] = four_pair<0>(v.r[e], scale);
            r[e][1] = four_pair<1>(v.r[e], scale);
            if constexpr (DV == 8) {
                r[e][2] = four_pair<2>(v.r[e], scale);
                r[e][3] = four_pair<3>(v.r[e], scale);
            }
        }
#pragma unroll
        for (int c = 0; c < DV; ++c) {
            uint4 x;
            const uint32_t sel = c & 1 ? 0x07060302u : 0x05040100u;
            x.x = __builtin_amdgcn_perm(r[1][c / 2], r[0][c / 2], sel);
            x.y = __builtin_amdgcn_perm(r[3][c / 2], r[2][c / 2], sel);
            x.z = __builtin_amdgcn_perm(r[5][c / 2], r[4][c / 2], sel);
            x.w = __builtin_amdgcn_perm(r[7][c / 2], r[6][c / 2], sel);
            const bf16x8 a = __builtin_bit_cast(bf16x8, x);
#pragma unroll
            for (int t = PT - 1; t >= 0; --t)
#pragma unroll
                for (int n = 0; n < NC; ++n)
                    acc[n][c] =
                        __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p[n].p[t], acc[n][c], 0, 0, 0);
        }
    }
};

// A workgroup's 256 threads on their way with a tile of 64 keys: each 16 bytes of codes of K and of V,
// which are 32 channels of a key and have one scale (D = 64: the first half of the threads K, the
// others V), through registers to bf16 rows in LDS.
template <int D>
struct FourStage {
    static constexpr int GROUPS = D / 32, SIDES = D == 128 ? 2 : 1;
    uint4 codes[SIDES];
    uint32_t scale[SIDES];
    int key, group, side;

    __device__ __forceinline__ void init(int tid) {
        side = D == 128 ? 0 : tid >> 7;
        group = tid % GROUPS;
        key = tid / GROUPS % 64;
    }
    // token: the tile's cached token of this thread's key, on `page` (-1: none).
    __device__ __forceinline__ void load(const PagedArgs& a, int page, int hk, int token) {
        const sparsp_cache& c = a.cache;
        const bool live = page >= 0 && 32 * group < c.d;
        const int64_t head = four_head(c, page, hk);
        const int row = token & (c.page - 1), g = 32 * group < c.d ? group : 0;
        const int64_t at = ((head * c.page + row) * c.d + 32 * g) / 2;
        const int64_t scale_at = (head * (c.d >> 5) + g) * c.page + row;
#pragma unroll
        for (int n = 0; n < SIDES; ++n) {
            const bool k = SIDES == 2 ? n == 0 : side == 0;
            codes[n] = make_uint4(0, 0, 0, 0);
            scale[n] = 0;
            if (live) {
                codes[n] = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(k ? c.K : c.V) + at);
                scale[n] = (k ? a.k_scales : a.v_scales)[scale_at];
            }
        }
    }
    // To rows of D channels at k and v; ks and vs: the swizzle of this thread's row.
    __device__ __forceinline__ void store(uint16_t* k, uint16_t* v, int ks, int vs) const {
#pragma unroll
        for (int n = 0; n < SIDES; ++n) {
            const bool is_k = SIDES == 2 ? n == 0 : side == 0;
            const float s = __uint_as_float(scale[n] << 23);
            uint16_t* row = (is_k ? k : v) + key * D;
            const int swizzle = is_k ? ks : vs;
            const uint32_t w[4] = {codes[n].x, codes[n].y, codes[n].z, codes[n].w};
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<uint4*>(row + ((4 * group + j) ^ swizzle) * 8) = four_octet(w[j], s);
        }
    }
};

}  // namespace
}  // namespace sparsp
