// What the kernels of the paged attention share: how a launch cuts a sequence's rows and keys,
// and how outputs leave.
#pragma once

#include "cache_device.h"

namespace sparsp {

// `tiles` workgroups stride over a sequence's row tiles, `parts` over its keys. With `flat` row
// tiles of all sequences at most, a workgroup finds its own among them instead.
struct PagedPlan {
    int tiles, parts, step, flat;
    float* part_o;  // [q_heads, tokens, parts, d], normalised
    // A part's sum of exponentials [q_heads, tokens, parts], and behind all of them the score, not
    // yet scaled, that they are relative to (-inf: the part has nothing). Not the log of one times
    // the other, which a float32 holds to 2^-24 of a row's largest score only: parts of one and of
    // three equal scores of 2^24 weighed the same.
    float *part_sum, *part_ref;
};

// Row tiles of 128 on LDS tiles, bf16 (paged_attn_tiles.hip).
hipError_t launch_paged_tiles(const PagedArgs& a, const PagedPlan& p, hipStream_t s);
// Weights of 256 keys a workgroup with Q through LDS, bf16 (paged_weights_tiles.hip).
hipError_t launch_weights_tiles(const PagedArgs& a, hipStream_t s);

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;

// Max and sum over the four lanes that hold a row, the same in all four.
__device__ __forceinline__ float row_max(float x) {
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float row_sum(float x) {
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The (sequence, head) pair and the part of unit u of pairs * parts. Units go to the eight XCDs
// in turn. Part by part, so that the parts that only long sequences have come last, and turned by
// the part, so that the parts of a pair do not share an XCD: with the parts of a pair in a
// row, short sequences of a ragged batch left most XCDs idle (64 sequences of 400 to 9,001
// tokens in 16 parts: 254 us).
struct Unit {
    int bh, part;
};
__device__ __forceinline__ Unit unit_of(int u, int pairs) {
    const int part = u / pairs;
    return {(u % pairs + pairs - part % pairs) % pairs, part};
}

// What a workgroup does: the row tiles tile, tile + stride, ... of a sequence and key head, and a
// part of the keys.
struct Work {
    int b, hk, part, tile, stride;
};
// Row tile number f of all sequences' tiles of ROWS rows. Each wave counts the tiles of 64
// sequences at a time.
template <int ROWS>
__device__ __forceinline__ bool find_tile(const sparsp_cache& c, int tokens, int G, int f, Work* w) {
    const int lane = threadIdx.x & 63;
    uint32_t before = 0;
    for (int b0 = 0; b0 < c.B; b0 += 64) {
        const int n = b0 + lane < c.B ? sequence(c, tokens, b0 + lane).n : 0;
        const uint32_t mine = uint32_t(n * G + ROWS - 1) / ROWS;
        uint32_t sum = mine;  // (exact up to the first lane that passes f, whatever new_off holds)
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t y = __shfl_up(sum, off);
            if (lane >= off) sum += y;
        }
        const uint64_t behind = __ballot(before + sum > uint32_t(f));
        if (behind) {
            const int l = __builtin_ctzll(behind);
            w->b = b0 + l;
            w->tile = f - int(before) - int(__builtin_amdgcn_readlane(sum - mine, l));
            return true;
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
}
// False: nothing. The row tiles of one part of the keys run on one XCD, one after another, so
// that all but the first find the keys in its L2. Flat tiles do so eight at a time, all heads'
// and parts' first eight before the next, and with parts, of which the later ones have less to
// do, the next eight on another XCD.
template <int ROWS>
__device__ __forceinline__ bool work_of(const PagedPlan& p, const sparsp_cache& c, int tokens, int G,
                                        Work* w) {
    const int xcd = blockIdx.x & 7, k = blockIdx.x >> 3;
    if (p.flat) {
        const int turn = (k >> 3) * 8 + xcd, units = c.H * p.parts;
        const int run = turn / units, f = run * 8 + (k & 7);
        const int unit = (turn + (p.parts > 1 ? run : 0)) % units;
        w->hk = unit % c.H;
        w->part = unit / c.H;
        w->stride = 1 << 30;
        return f < p.flat && find_tile<ROWS>(c, tokens, G, f, w);
    }
    const int unit = k / p.tiles * 8 + xcd;
    if (unit >= c.B * c.H * p.parts) return false;
    const auto [bh, part] = unit_of(unit, c.B * c.H);
    *w = {bh / c.H, bh % c.H, part, k % p.tiles, p.tiles};
    return true;
}
inline int workgroups(const PagedPlan& p, const sparsp_cache& c) {
    return p.flat ? ((p.flat + 7) / 8 * c.H * p.parts + 7) / 8 * 64
                  : (c.B * c.H * p.parts + 7) / 8 * 8 * p.tiles;
}

// Keys of a part of a sequence of kv cached tokens: a multiple of step, so many that
// `parts` of them cover kv.
__device__ __forceinline__ int part_keys(const PagedPlan& p, int kv) {
    const int64_t all = (int64_t(kv) + p.parts - 1) / p.parts;
    const int64_t k = (all + p.step - 1) / p.step * p.step;
    return int(k < p.step ? p.step : k);
}

__device__ __forceinline__ void store4(void* O, int64_t at, bool bf16, const float (&x)[4]) {
    if (bf16) {
        uint2 w;
        w.x = f32_to_bf16_bits(x[0]) | (f32_to_bf16_bits(x[1]) << 16);
        w.y = f32_to_bf16_bits(x[2]) | (f32_to_bf16_bits(x[3]) << 16);
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(O) + at) = w;
    } else {
        *reinterpret_cast<float4*>(static_cast<float*>(O) + at) =
            make_float4(x[0], x[1], x[2], x[3]);
    }
}

}  // namespace
}  // namespace sparsp
