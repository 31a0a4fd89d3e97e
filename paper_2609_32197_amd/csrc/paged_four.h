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

// The conversion takes a scale's exponent from bits 30 to 23 of its operand and nothing else: byte
// `e` of w is shifted there, whatever comes with it. turn: 9 + 8 e.
__device__ __forceinline__ float four_scale(uint32_t w, int turn) {
    return __uint_as_float(__builtin_amdgcn_alignbit(w, w, turn));
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

// Rows of Q in float32 (TERMS 3) enter the products as three bf16 each, which hold them whole, and so
// do probabilities; rows in bf16 (TERMS 1) as they are, and probabilities as two. C: channels.
template <int TERMS, int C>
struct Four {};

// Layout as for bf16 (paged_tiles.h), but for the order of the channels in a score's sum: lane group
// g takes D / 4 consecutive ones, 16 or 8 bytes of codes in one load and one scale.
template <int TERMS, int C, int D>
struct TileMath<Four<TERMS, C>, D> {
    static constexpr int KEYS = 32, U = 2, PER = 8, KT = D / 32, DV = D / 16;
    static constexpr int PT = TERMS == 1 ? 2 : 3;  // terms of a probability
    struct KTile { uint32_t k[U][KT], scales[2]; };
    struct QTile { bf16x8 q[TERMS][KT]; };
    struct VTile { uint32_t r[8], scales[2]; };

    static __device__ __forceinline__ int key_of(int g, int v) { return 8 * g + v; }
    static __device__ __forceinline__ int k_group(int lane) { return 8 * ((lane & 15) >> 2); }
    static __device__ __forceinline__ int v_group(int lane) { return 8 * (lane >> 4); }

    // Where a wave reads. A tile's 32 keys lie on one page, whose address is the same for all lanes:
    // lanes add constants to it, through descriptors rooted at the tile, which costs the vector unit
    // nothing. With HALVES, for pages of 16, they lie on two.
    template <bool HALVES>
    struct Source {
        const uint8_t *k, *v, *ks, *vs;      // of the head on page 0
        uint32_t page_codes, page_scales;    // bytes of a page
        uint32_t row_mask;
        uint32_t k_at, v_at, ks_at, vs_at;   // a lane's place in a tile
        bool k_second, v_second;             // in its second 16 keys

        __device__ __forceinline__ Source(const PagedArgs& a, int hk, int lane) {
            const sparsp_cache& c = a.cache;
            row_mask = c.page - 1;
            page_codes = uint32_t(c.H * c.page) * (C / 2);
            page_scales = uint32_t(c.H * c.page) * (C / 32);
            const uint32_t head = uint32_t(hk * c.page);
            k = static_cast<const uint8_t*>(c.K) + head * (C / 2);
            v = static_cast<const uint8_t*>(c.V) + head * (C / 2);
            ks = a.k_scales + head * (C / 32);
            vs = a.v_scales + head * (C / 32);
            const int k_own = (D / 4) * (lane >> 4), k_ch = k_own < C ? k_own : 0;
            const int v_own = DV * (lane & 15), v_ch = v_own < C ? v_own : 0;
            k_at = ((k_group(lane) + (lane & 3)) * C + k_ch) / 2;
            v_at = (v_group(lane) * C + v_ch) / 2;
            ks_at = k_ch / 32 * c.page + k_group(lane);
            vs_at = v_ch / 32 * c.page + v_group(lane);
            k_second = k_group(lane) >= 16;
            v_second = v_group(lane) >= 16;
        }
        // page, second: of the tile's first and second 16 keys (-1: page 0, whose values the callers
        // mask). t0 is a multiple of 32.
        __device__ __forceinline__ void load(KTile& kt, VTile& vt, int page, int second, int t0) const {
            if constexpr (HALVES) {
                const uint64_t p = uint32_t(max(page, 0)), q = uint32_t(max(second, 0));
                const uint64_t codes = p * page_codes, scales = p * page_scales;
                const uint64_t codes2 = q * page_codes - 16 * (C / 2), scales2 = q * page_scales - 16;
                load_k(kt, k + (k_second ? codes2 : codes) + k_at,
                       ks + (k_second ? scales2 : scales) + ks_at);
                load_v(vt, v + (v_second ? codes2 : codes) + v_at,
                       vs + (v_second ? scales2 : scales) + vs_at);
            } else {
                const uint64_t row = uint32_t(t0) & row_mask;
                const uint64_t p = uint32_t(max(max(page, second), 0));  // (either may be masked)
                const uint64_t codes = p * page_codes + row * (C / 2), scales = p * page_scales + row;
                const int tile = KEYS * (C / 2), groups = (C / 32 - 1) * (row_mask + 1) + KEYS;
                const auto kd = rooted(k + codes, tile), vd = rooted(v + codes, tile);
                const auto ksd = rooted(ks + scales, groups), vsd = rooted(vs + scales, groups);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if constexpr (KT == 4) {
                        const u32x4_t x =
                            __builtin_amdgcn_raw_buffer_load_b128(kd, k_at + 2 * u * C, 0, 0);
#pragma unroll
                        for (int e = 0; e < 4; ++e) kt.k[u][e] = x[e];
                    } else {
                        const u32x2_t x =
                            __builtin_amdgcn_raw_buffer_load_b64(kd, k_at + 2 * u * C, 0, 0);
#pragma unroll
                        for (int e = 0; e < 2; ++e) kt.k[u][e] = x[e];
                    }
                }
                const u32x2_t x = __builtin_amdgcn_raw_buffer_load_b64(ksd, ks_at, 0, 0);
                kt.scales[0] = x.x;
                kt.scales[1] = x.y;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (DV == 8)
                        vt.r[e] = __builtin_amdgcn_raw_buffer_load_b32(vd, v_at + e * (C / 2), 0, 0);
                    else
                        vt.r[e] = uint16_t(
                            __builtin_amdgcn_raw_buffer_load_b16(vd, v_at + e * (C / 2), 0, 0));
                }
                const u32x2_t y = __builtin_amdgcn_raw_buffer_load_b64(vsd, vs_at, 0, 0);
                vt.scales[0] = y.x;
                vt.scales[1] = y.y;
            }
        }
        static __device__ __forceinline__ __amdgpu_buffer_rsrc_t rooted(const uint8_t* p, int bytes) {
            const uint64_t at = reinterpret_cast<uint64_t>(p);
            const uint64_t lo = uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(at)));
            const uint64_t hi = uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(at >> 32)));
            return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(hi << 32 | lo), 0,
                                                     __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
        }
        static __device__ __forceinline__ void load_k(KTile& t, const uint8_t* from,
                                                      const uint8_t* scales) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if constexpr (KT == 4) {
                    const u32x4_t x = *reinterpret_cast<const u32x4_t*>(from + 2 * u * C);
#pragma unroll
                    for (int e = 0; e < 4; ++e) t.k[u][e] = x[e];
                } else {
                    const u32x2_t x = *reinterpret_cast<const u32x2_t*>(from + 2 * u * C);
#pragma unroll
                    for (int e = 0; e < 2; ++e) t.k[u][e] = x[e];
                }
            }
            load_scales(t.scales, scales);
        }
        static __device__ __forceinline__ void load_v(VTile& t, const uint8_t* from,
                                                      const uint8_t* scales) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                t.r[e] = DV == 8 ? *reinterpret_cast<const uint32_t*>(from + e * (C / 2))
                                 : *reinterpret_cast<const uint16_t*>(from + e * (C / 2));
            load_scales(t.scales, scales);
        }
        // Of eight keys.
        static __device__ __forceinline__ void load_scales(uint32_t (&to)[2], const uint8_t* from) {
            const u32x2_t x = *reinterpret_cast<const u32x2_t*>(from);
            to[0] = x.x;
            to[1] = x.y;
        }
    };

    static __device__ __forceinline__ void load_row(QTile& t, const void* Q, int64_t at, bool live,
                                                    int, int lane) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            const int ch = (D / 4) * (lane >> 4) + 8 * kt;
            if constexpr (TERMS == 1) {
                uint4 x = make_uint4(0, 0, 0, 0);
                if (live && ch < C)
                    x = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(Q) + at + ch);
                t.q[0][kt] = __builtin_bit_cast(bf16x8, x);
            } else {
                floatx8 x = {};
                if (live && ch < C) {
                    const floatx4* p =
                        reinterpret_cast<const floatx4*>(static_cast<const float*>(Q) + at + ch);
                    x = __builtin_shufflevector(p[0], p[1], 0, 1, 2, 3, 4, 5, 6, 7);
                }
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
        const int turn = 9 + 8 * (__lane_id() & 3);
        float scale[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            s[u] = floatx4{};
            scale[u] = four_scale(k.scales[u], turn);
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
    // Keys from `live` on (of this lane's eight) become zero: codes, and scales, which may say NaN.
    static __device__ __forceinline__ void clear_v(VTile& t, int live) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            t.r[e] = e < live ? t.r[e] : 0u;
            t.scales[e / 4] = e < live ? t.scales[e / 4] : t.scales[e / 4] & ~(255u << (e % 4 * 8));
        }
    }
    static __device__ __forceinline__ uint32_t upper_halves(float x, float y) {
        return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
    }
    struct P { bf16x8 p[PT]; };
    static __device__ __forceinline__ P pack(const float (&p)[PER]) {
        floatx8 x;
#pragma unroll
        for (int v = 0; v < 8; ++v) x[v] = p[v];
        P r;
        if constexpr (PT == 2) {
            // The upper half of its bits, and what that leaves.
            floatx8 hi;
            uint4 w;
#pragma unroll
            for (int v = 0; v < 8; ++v)
                hi[v] = __uint_as_float(__float_as_uint(x[v]) & 0xffff0000u);
            w.x = upper_halves(x[0], x[1]);
            w.y = upper_halves(x[2], x[3]);
            w.z = upper_halves(x[4], x[5]);
            w.w = upper_halves(x[6], x[7]);
            r.p[0] = __builtin_bit_cast(bf16x8, w);
            r.p[1] = __builtin_convertvector(x - hi, bf16x8);
        } else {
            split<PT>(x, [&](int term, bf16x8 y) { r.p[term] = y; });
        }
        return r;
    }
    // Two output tiles at a time: a byte of each key's code, and the eight keys' halves of it.
    template <int W, int NC>
    static __device__ __forceinline__ void output_pair(const VTile& v, const float (&scale)[8],
                                                       const P (&p)[NC], floatx4 (&acc)[NC][DV]) {
        uint32_t r[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = four_pair<W>(v.r[e], scale[e]);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            uint4 x;
            const uint32_t sel = c ? 0x07060302u : 0x05040100u;
            x.x = __builtin_amdgcn_perm(r[1], r[0], sel);
            x.y = __builtin_amdgcn_perm(r[3], r[2], sel);
            x.z = __builtin_amdgcn_perm(r[5], r[4], sel);
            x.w = __builtin_amdgcn_perm(r[7], r[6], sel);
            const bf16x8 a = __builtin_bit_cast(bf16x8, x);
#pragma unroll
            for (int t = PT - 1; t >= 0; --t)
#pragma unroll
                for (int n = 0; n < NC; ++n)
                    acc[n][2 * W + c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        a, p[n].p[t], acc[n][2 * W + c], 0, 0, 0);
        }
    }
    template <int NC>
    static __device__ __forceinline__ void output(const VTile& v, const P (&p)[NC],
                                                  floatx4 (&acc)[NC][DV]) {
        float scale[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) scale[e] = four_scale(v.scales[e / 4], 9 + 8 * (e % 4));
        output_pair<0>(v, scale, p, acc);
        output_pair<1>(v, scale, p, acc);
        if constexpr (DV == 8) {
            output_pair<2>(v, scale, p, acc);
            output_pair<3>(v, scale, p, acc);
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
    uint32_t page_codes, page_scales;  // bytes of a page
    uint32_t code_at, scale_at;        // this thread's in the first row of page 0
    bool there;

    __device__ __forceinline__ void init(const sparsp_cache& c, int hk, int tid) {
        side = D == 128 ? 0 : tid >> 7;
        group = tid % GROUPS;
        key = tid / GROUPS % 64;
        there = 32 * group < c.d;
        const uint32_t g = there ? group : 0, groups = uint32_t(c.d) / 32;
        page_codes = uint32_t(c.H * c.page * (c.d / 2));
        page_scales = uint32_t(c.H * c.page) * groups;
        code_at = uint32_t(hk * c.page) * uint32_t(c.d / 2) + 16 * g;
        scale_at = (uint32_t(hk) * groups + g) * c.page;
    }
    // token: the tile's cached token of this thread's key, on `page` (-1: none).
    __device__ __forceinline__ void load(const PagedArgs& a, int page, int token) {
        const sparsp_cache& c = a.cache;
        const bool live = page >= 0 && there;
        const uint32_t row = token & (c.page - 1), p = max(page, 0);
        const uint64_t at = uint64_t(p) * page_codes + (code_at + row * uint32_t(c.d / 2));
        const uint64_t scales = uint64_t(p) * page_scales + (scale_at + row);
#pragma unroll
        for (int n = 0; n < SIDES; ++n) {
            const bool k = SIDES == 2 ? n == 0 : side == 0;
            codes[n] = make_uint4(0, 0, 0, 0);
            scale[n] = 0;
            if (live) {
                codes[n] = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(k ? c.K : c.V) + at);
                scale[n] = (k ? a.k_scales : a.v_scales)[scales];
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
            // Eight lanes write 16 bytes each to all 32 banks: lanes whose chunks the swizzle does not
            // keep apart take theirs in another order (attend4-chunks of perf/more_operators.py 659 us
            // in the same one, 8 cycles more a store, and 650 so; at d = 64, where a lane's side
            // decides as well, the choice costs more: 369 and 400 us).
            const int turn = D == 128 && (group & 2) ? (is_k ? 2 : 1) : 0;
            const int swizzle = (is_k ? ks : vs) ^ turn;
            const uint32_t w[4] = {codes[n].x, codes[n].y, codes[n].z, codes[n].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t c = turn == 2 ? w[j ^ 2] : turn == 1 ? w[j ^ 1] : w[j];
                *reinterpret_cast<uint4*>(row + ((4 * group + j) ^ swizzle) * 8) = four_octet(c, s);
            }
        }
    }
};

}  // namespace
}  // namespace sparsp
