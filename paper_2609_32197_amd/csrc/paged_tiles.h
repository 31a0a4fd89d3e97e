// One wave's products of a tile of cached keys with 16 query rows, straight from global
// memory to the matrix cores' operand registers.
//
// The score tile is computed transposed, S^T = K Q^T, and so is the output, O^T = V^T P^T:
// lane l holds row r = l % 16 of every result, and of the keys those that the P^T
// operand wants from it, so the probabilities never move between lanes.
//
// Lane l = 16 g + i (g = l / 16). 16x16x32 bf16: A lane l holds row i, k values
// 8 g .. 8 g + 7; B lane l column i, the same k values; lane l's four results are column i,
// rows 4 g .. 4 g + 3. 16x16x4 f32: A and B lane l hold one k value, g; results alike.
//
// bf16, 32 keys a tile: score tile u (0, 1) is fed key 8 (m / 4) + 4 u + m % 4 as its row m,
// so lane l's eight results are the consecutive keys 8 g .. 8 g + 7, which are its k values of
// P^T. For V^T a lane reads D / 16 consecutive channels of those eight keys and
// transposes the 8 x D/16 block in registers (one byte permutation per register); output
// tile c holds the channels (D/16) i + c, so a lane ends with 4 D/16 consecutive ones.
// f32, 16 keys a tile: row m is key m; step e of P^T V takes key 4 g + e from each lane.
//
// Head dimensions below D leave the last operand columns over: those lanes read channel 0
// again, Q holds zeros there and the output columns are not stored.
#pragma once

#include "paged_plan.h"

namespace sparsp {
namespace {

// Address of cached row `key` of head hk on `page` (page -1: page 0, whose values the
// callers mask).
template <typename T>
__device__ __forceinline__ const T* cached_row(const sparsp_cache& c, const void* base, int page,
                                               int hk, int key) {
    const int64_t row = (int64_t(page < 0 ? 0 : page) * c.H + hk) * c.page + (key & (c.page - 1));
    return static_cast<const T*>(base) + row * c.d;
}

template <typename T, int D>
struct TileMath;

template <int D>
struct TileMath<uint16_t, D> {
    static constexpr int KEYS = 32, U = 2, PER = 8, KT = D / 32, DV = D / 16;
    struct KTile { bf16x8 k[U][KT]; };
    struct QTile { bf16x8 q[KT]; };
    struct VTile { uint32_t r[8][DV / 2]; };

    static __device__ __forceinline__ int key_of(int g, int v) { return 8 * g + v; }
    static __device__ __forceinline__ int k_group(int lane) { return 8 * ((lane & 15) >> 2); }
    static __device__ __forceinline__ int v_group(int lane) { return 8 * (lane >> 4); }

    static __device__ __forceinline__ void load_k(const sparsp_cache& c, KTile& t, int page, int hk,
                                                  int t0, int lane) {
        const int g = lane >> 4;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint16_t* p = cached_row<uint16_t>(c, c.K, page, hk,
                                                     t0 + k_group(lane) + 4 * u + (lane & 3));
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const int ch = 32 * kt + 8 * g;
                t.k[u][kt] = *reinterpret_cast<const bf16x8*>(p + (ch < c.d ? ch : 0));
            }
        }
    }
    static __device__ __forceinline__ void load_row(QTile& t, const void* Q, int64_t at, bool live,
                                                    int d, int lane) {
        const int g = lane >> 4;
        const uint16_t* p = static_cast<const uint16_t*>(Q) + at;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            const int ch = 32 * kt + 8 * g;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (live && ch < d) x = *reinterpret_cast<const uint4*>(p + ch);
            t.q[kt] = __builtin_bit_cast(bf16x8, x);
        }
    }
    static __device__ __forceinline__ void scores(const KTile& k, const QTile& q, floatx4 (&s)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) s[u] = floatx4{};
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int u = 0; u < U; ++u)
                s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k.k[u][kt], q.q[kt], s[u], 0, 0, 0);
    }
    static __device__ __forceinline__ void load_v(const sparsp_cache& c, VTile& t, int page, int hk,
                                                  int t0, int lane) {
        const int ch = DV * (lane & 15), off = ch < c.d ? ch : 0;
        // (the eight keys are on one page: pages start at multiples of 16)
        const uint16_t* p = cached_row<uint16_t>(c, c.V, page, hk, t0 + v_group(lane)) + off;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (DV == 8) {
                const uint4 x = *reinterpret_cast<const uint4*>(p + e * c.d);
                t.r[e][0] = x.x;
                t.r[e][1] = x.y;
                t.r[e][2] = x.z;
                t.r[e][3] = x.w;
            } else {
                const uint2 x = *reinterpret_cast<const uint2*>(p + e * c.d);
                t.r[e][0] = x.x;
                t.r[e][1] = x.y;
            }
        }
    }
    // Rows from `live` on (of this lane's eight) become zero.
    static __device__ __forceinline__ void clear_v(VTile& t, int live) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int w = 0; w < DV / 2; ++w) t.r[e][w] = e < live ? t.r[e][w] : 0u;
    }
    // A probability enters the product as two bf16, its rounding and what that leaves, so it is off by
    // 2^-16 of itself. What waits for K and V has the matrix pipe to spare (64 sequences of 400 to
    // 9,001 tokens, one new each: 140.9 us with one bf16, 141.3 us; of 4,000 at d = 64, 24 rows each,
    // 116.0 and 116.5 us; one of 9,000: 18.0 and 18.5 us), and of 1,000 bf16 outputs 998 are the
    // exact ones rounded, 618 with one bf16.
    struct P { bf16x8 hi, lo; };
    static __device__ __forceinline__ P pack(const float (&p)[PER]) {
        floatx8 x;
#pragma unroll
        for (int v = 0; v < 8; ++v) x[v] = p[v];
        const bf16x8 hi = __builtin_convertvector(x, bf16x8);
        return {hi, __builtin_convertvector(x - __builtin_convertvector(hi, floatx8), bf16x8)};
    }
    template <int NC>
    static __device__ __forceinline__ void output(const VTile& v, const P (&p)[NC],
                                                  floatx4 (&acc)[NC][DV]) {
#pragma unroll
        for (int c = 0; c < DV; ++c) {
            uint4 x;
            const uint32_t sel = c & 1 ? 0x07060302u : 0x05040100u;
            x.x = __builtin_amdgcn_perm(v.r[1][c / 2], v.r[0][c / 2], sel);
            x.y = __builtin_amdgcn_perm(v.r[3][c / 2], v.r[2][c / 2], sel);
            x.z = __builtin_amdgcn_perm(v.r[5][c / 2], v.r[4][c / 2], sel);
            x.w = __builtin_amdgcn_perm(v.r[7][c / 2], v.r[6][c / 2], sel);
            const bf16x8 a = __builtin_bit_cast(bf16x8, x);
#pragma unroll
            for (int n = 0; n < NC; ++n)
                acc[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p[n].lo, acc[n][c], 0, 0, 0);
#pragma unroll
            for (int n = 0; n < NC; ++n)
                acc[n][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p[n].hi, acc[n][c], 0, 0, 0);
        }
    }
};

template <int D>
struct TileMath<float, D> {
    static constexpr int KEYS = 16, U = 1, PER = 4, KT = D / 16, DV = D / 16;
    struct KTile { floatx4 k[KT]; };
    struct QTile { floatx4 q[KT]; };
    struct VTile { float r[4][DV]; };

    static __device__ __forceinline__ int key_of(int g, int v) { return 4 * g + v; }
    static __device__ __forceinline__ int k_group(int) { return 0; }
    static __device__ __forceinline__ int v_group(int lane) { return 4 * (lane >> 4); }

    static __device__ __forceinline__ void load_k(const sparsp_cache& c, KTile& t, int page, int hk,
                                                  int t0, int lane) {
        const int g = lane >> 4;
        const float* p = cached_row<float>(c, c.K, page, hk, t0 + (lane & 15));
#pragma unroll
        for (int j = 0; j < KT; ++j) {
            const int ch = 16 * j + 4 * g;
            t.k[j] = *reinterpret_cast<const floatx4*>(p + (ch < c.d ? ch : 0));
        }
    }
    static __device__ __forceinline__ void load_row(QTile& t, const void* Q, int64_t at, bool live,
                                                    int d, int lane) {
        const int g = lane >> 4;
        const float* p = static_cast<const float*>(Q) + at;
#pragma unroll
        for (int j = 0; j < KT; ++j) {
            const int ch = 16 * j + 4 * g;
            t.q[j] = floatx4{};
            if (live && ch < d) t.q[j] = *reinterpret_cast<const floatx4*>(p + ch);
        }
    }
    static __device__ __forceinline__ void scores(const KTile& k, const QTile& q, floatx4 (&s)[U]) {
        s[0] = floatx4{};
#pragma unroll
        for (int j = 0; j < KT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                s[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.k[j][e], q.q[j][e], s[0], 0, 0, 0);
    }
    static __device__ __forceinline__ void load_v(const sparsp_cache& c, VTile& t, int page, int hk,
                                                  int t0, int lane) {
        const int ch = DV * (lane & 15);
        const float* p = cached_row<float>(c, c.V, page, hk, t0 + v_group(lane));
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int w = 0; w < DV; w += 4) {
                const floatx4 x = *reinterpret_cast<const floatx4*>(
                    p + e * c.d + (ch + w < c.d ? ch + w : 0));
#pragma unroll
                for (int q = 0; q < 4; ++q) t.r[e][w + q] = x[q];
            }
    }
    static __device__ __forceinline__ void clear_v(VTile& t, int live) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int w = 0; w < DV; ++w) t.r[e][w] = e < live ? t.r[e][w] : 0.f;
    }
    struct P { float p[4]; };
    static __device__ __forceinline__ P pack(const float (&p)[PER]) {
        return {{p[0], p[1], p[2], p[3]}};
    }
    template <int NC>
    static __device__ __forceinline__ void output(const VTile& v, const P (&p)[NC],
                                                  floatx4 (&acc)[NC][DV]) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int c = 0; c < DV; ++c)
#pragma unroll
                for (int n = 0; n < NC; ++n)
                    acc[n][c] =
                        __builtin_amdgcn_mfma_f32_16x16x4f32(v.r[e][c], p[n].p[e], acc[n][c], 0, 0, 0);
    }
};

}  // namespace
}  // namespace sparsp
