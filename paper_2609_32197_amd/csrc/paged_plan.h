// What the kernels of the paged attention share: how a launch cuts a sequence's rows and keys,
// and how outputs leave.
#pragma once

#include "cache_device.h"

namespace sparsp {

// `tiles` workgroups stride over a sequence's row tiles, `parts` over its keys.
struct PagedPlan {
    int tiles, parts, step;
    float* part_o;    // [q_heads, tokens, parts, d]
    float* part_lse;  // [q_heads, tokens, parts]
};

// Row tiles of 128 on LDS tiles, bf16 (paged_attn_tiles.hip).
hipError_t launch_paged_tiles(const PagedArgs& a, const PagedPlan& p, hipStream_t s);
// Weights of 256 keys a workgroup with Q through LDS, bf16 (paged_weights_tiles.hip).
hipError_t launch_weights_tiles(const PagedArgs& a, hipStream_t s);

namespace {

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
