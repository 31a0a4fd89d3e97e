// Attention of many new tokens over the paged cache, bf16: 128 rows (token, head of the
// group) a workgroup, K and V tiles of 64 keys shared by its four waves through LDS.
//
// Each wave owns 32 rows against every key and runs one online softmax. Score and output
// tiles are computed transposed with v_mfma_f32_16x16x32_bf16, S^T = K Q^T and O^T = V^T P^T,
// and the keys are dealt to the rows of the score tiles so that a lane's probabilities are its
// operand of the second product (the layout is stated in paged_tiles.h; a wave's two column
// groups of 16 rows share every operand of K and V). V lies in LDS as it lies in the cache,
// one key a row; its transposed operand comes from ds_read_b64_tr_b16: in a group of 16
// lanes, lane i points at 4 channels of key i / 4, channels 4 (i % 4), and receives channel
// i of the four keys. Two such reads make the eight keys of an operand.
//
// Tiles are double-buffered: the copies of tile j+1 are issued right after the barrier that
// opens tile j. They are direct-to-LDS buffer loads; a wave copies 16 rows, which lie on one
// page, through a descriptor rooted at the first of them and ending with the sequence: rows
// behind it, rows of a page that does not exist and channels behind d become zeros. The page
// numbers of the next 16,384 keys are held in LDS, since a load of them in the loop would wait
// for the copies.
//
// Swizzle: 16-byte chunks of an LDS row are exchanged by an XOR with bits of the row, applied to
// the source addresses of the copies. K rows read together by 16 lanes (8 i + j + const,
// i, j < 4) land on their own 16 bytes of 256; V rows read together by 32 lanes (8 i + j +
// const, i < 2, j < 4) on their own 32 bytes.
#include <type_traits>

#include "paged_four.h"

namespace sparsp {
namespace {

typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4_t lds_short4;

constexpr float kLn2 = 0.6931471805599453f;

constexpr int kKeys = 64;        // keys of a tile
constexpr int kRowsTile = 128;   // rows of a workgroup
constexpr int kSegment = 16384;  // keys whose page numbers are held at once

// The XOR of a row's 16-byte chunk number, for K and for V.
template <int D>
__device__ __forceinline__ int k_swizzle(int row) {
    const int i = (row >> 3) & 3;
    return D == 128 ? (row & 3) | (i << 2) : ((row >> 1) & 1) | (i << 1);
}
template <int D>
__device__ __forceinline__ int v_swizzle(int row) {
    const int i = (row >> 3) & 1;
    return (D == 128 ? (row & 3) | (i << 2) : ((row >> 1) & 1) | (i << 1)) << 1;
}

// A wave's copies of one tile to LDS, 1 KB an instruction, to consecutive places. Inline
// assembly, because the compiler would guard every later LDS read with a wait for all copies in
// flight; the waits are explicit. M0 is restored, and a wait state separates each write of it
// from its use.
template <int NI>
__device__ __forceinline__ void copy_rows(const u32x4_t& desc, const int (&off)[NI], uint32_t to) {
    static_assert(NI == 2 || NI == 4, "copies of a wave");
#if defined(__HIP_DEVICE_COMPILE__)
    uint32_t saved;
    if constexpr (NI == 2)
        asm volatile(
            "s_mov_b32 %[sv], m0\n\ts_mov_b32 m0, %[to]\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %[o0], %[desc], 0 offen lds\n\t"
            "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %[o1], %[desc], 0 offen lds\n\t"
            "s_mov_b32 m0, %[sv]"
            : [sv] "=&s"(saved)
            : [to] "s"(to), [desc] "s"(desc), [o0] "v"(off[0]), [o1] "v"(off[1])
            : "memory", "scc");
    else
        asm volatile(
            "s_mov_b32 %[sv], m0\n\ts_mov_b32 m0, %[to]\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %[o0], %[desc], 0 offen lds\n\t"
            "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %[o1], %[desc], 0 offen lds\n\t"
            "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %[o2], %[desc], 0 offen lds\n\t"
            "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\t"
            "buffer_load_dwordx4 %[o3], %[desc], 0 offen lds\n\t"
            "s_mov_b32 m0, %[sv]"
            : [sv] "=&s"(saved)
            : [to] "s"(to), [desc] "s"(desc), [o0] "v"(off[0]), [o1] "v"(off[1]), [o2] "v"(off[2]),
              [o3] "v"(off[3])
            : "memory", "scc");
#endif
}

// D: channels of a row in LDS; those from C on are zero and left out of the products (d = 96,
// 32 heads, 675 tokens over 24,153: 283 us, with all 128 328 us).
template <int D, int C, bool WINDOW, bool FOUR>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2)))
void paged_tiles_kernel(const PagedArgs a, const PagedPlan plan) {
    constexpr int TILE = kKeys * D;
    constexpr int NCH = D / 8;         // 16-byte chunks of a row
    constexpr int RPI = 64 / NCH;      // rows of one copy instruction
    constexpr int NI = kKeys / 4 / RPI;  // copy instructions of a wave, each of K and V
    constexpr int KT = C / 32, DT = C / 16;
    __shared__ __attribute__((aligned(16))) uint16_t lds[2][2][TILE];  // [buffer][K, V]
    __shared__ int page_list[kSegment / 16];

    const sparsp_cache& c = a.cache;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int G = a.q_heads / c.H;
    Work work;
    if (!work_of<kRowsTile>(plan, c, a.tokens, G, &work)) return;
    const int b = work.b, hk = work.hk, part = work.part;
    const Seq s = sequence(c, a.tokens, b);
    const int rows = s.n * G;
    // Calls with a window or over 4 bits can have a tail, and find their part for each tile.
    constexpr bool EACH = WINDOW || FOUR;
    Span span = {0, 0, s.kv, 0};
    int keys = part_keys(plan, s.kv);
    bool whole = s.kv <= keys;
    if (!EACH && part > 0 && part * int64_t(keys) >= s.kv) return;
    int lo = part * keys, part_end = min(s.kv - lo, keys) + lo;
    const float c2 = a.scale * kLog2e;
    const int shift = __builtin_ctz(c.page);
    const int list_shift = WINDOW ? 4 : shift;  // (a window's gap is no multiple of a page)
    const uint32_t row_bytes = uint32_t(c.d) * 2, page_bytes = uint32_t(c.H * c.page) * row_bytes;
    // (48-bit addresses: the upper 16 bits of a descriptor's address word stay clear)
    const uint64_t head_at = uint64_t(uint32_t(hk * c.page)) * row_bytes;
    const uint64_t k_base = (reinterpret_cast<uint64_t>(c.K) & 0xffffffffffffull) + head_at;
    const uint64_t v_base = (reinterpret_cast<uint64_t>(c.V) & 0xffffffffffffull) + head_at;
    [[maybe_unused]] FourStage<D> stage;
    if constexpr (FOUR) stage.init(c, hk, tid);
    const uint32_t k_lds = __builtin_amdgcn_readfirstlane(
        uint32_t(reinterpret_cast<uintptr_t>(&lds[0][0][16 * wave * D])));

    // A wave copies the 16 rows from 16 * wave on, which lie on one page whatever its size.
    // Source offsets of this lane's copies from the first of them; channels behind d lie past
    // every descriptor.
    int koff[NI], voff[NI];
#pragma unroll
    for (int n = 0; n < NI; ++n) {
        const int sub = n * RPI + lane / NCH, row = 16 * wave + sub, pc = lane % NCH;
        const int kc = (pc ^ k_swizzle<D>(row)) * 8, vc = (pc ^ v_swizzle<D>(row)) * 8;
        koff[n] = kc < c.d ? int(sub * row_bytes) + kc * 2 : 0x7ffffff0;
        voff[n] = vc < c.d ? int(sub * row_bytes) + vc * 2 : 0x7ffffff0;
    }
    // Byte addresses of this lane's operands in a tile: the XOR with kt (dt) and the immediate
    // offsets of a tile's other rows are added where they are read.
    const int krow = 8 * (col >> 2) + (col & 3);
    const uint32_t k_at = uint32_t(krow * D * 2 + ((g ^ k_swizzle<D>(krow)) * 16));
    const int vrow = 8 * g + (col >> 2);
    const uint32_t v_at = uint32_t(vrow * D * 2 + (((col & 3) >> 1) ^ v_swizzle<D>(vrow)) * 16 +
                                   (col & 1) * 8);

    // Later row tiles see more keys: they come first.
    for (int turns = work.tile; turns * int64_t(kRowsTile) < rows; turns += work.stride) {
        const int n_tiles = (rows + kRowsTile - 1) / kRowsTile;
        const int tile = n_tiles - 1 - turns;
        if constexpr (EACH) {
            if constexpr (WINDOW)
                span = span_of(a, s, G, tile * kRowsTile, min(rows, (tile + 1) * kRowsTile) - 1, kKeys);
            // (of a workgroup's tiles, which are more where max_new was too small, the first is the tail's)
            const bool all = plan.tail && (work.tail < 0 || turns != work.tile);
            keys = all ? max(span.len, 1) : part_keys(plan, span.len);
            whole = span.len <= keys;
            if (part > 0 && part * int64_t(keys) >= span.len) continue;
            lo = part * keys;
            part_end = min(span.len - lo, keys) + lo;
        }
        bf16x8 q[2][KT];
        int limit[2], lowest = 1 << 30, highest = 0;
        int earliest = 1 << 30, latest = 0;  // of the rows' windows, where they begin
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int r = tile * kRowsTile + wave * 32 + n * 16 + col;
            const bool live = r < rows;
            const int i = live ? r / G : 0, h = hk * G + (live ? r % G : 0);
            limit[n] = !live ? 0 : a.causal ? min(s.kv, s.kv - s.n + i + 1) : s.kv;
            if (WINDOW && live) {
                limit[n] -= span.skip;
                earliest = min(earliest, limit[n] - a.window);
                latest = max(latest, limit[n] - a.window);
            }
            if (live) lowest = min(lowest, limit[n]);
            highest = max(highest, limit[n]);
            const uint16_t* p = static_cast<const uint16_t*>(a.Q) + int64_t(h) * a.q_head +
                                int64_t(s.q0 + i) * a.q_token;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const int ch = 32 * kt + 8 * g;
                uint4 x = make_uint4(0, 0, 0, 0);
                if (live && ch < c.d) x = *reinterpret_cast<const uint4*>(p + ch);
                q[n][kt] = __builtin_bit_cast(bf16x8, x);
            }
        }
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) {
            lowest = min(lowest, __shfl_xor(lowest, off));
            highest = max(highest, __shfl_xor(highest, off));
            if constexpr (WINDOW) {
                earliest = min(earliest, __shfl_xor(earliest, off));
                latest = max(latest, __shfl_xor(latest, off));
            }
        }
        if constexpr (WINDOW) {
            earliest = __builtin_amdgcn_readfirstlane(earliest);
            latest = __builtin_amdgcn_readfirstlane(latest);
        }
        lowest = __builtin_amdgcn_readfirstlane(min(lowest, part_end));
        highest = __builtin_amdgcn_readfirstlane(min(highest, part_end));
        const int last = min(rows, (tile + 1) * kRowsTile) - 1;
        const int end =
            min((a.causal ? min(s.kv, s.kv - s.n + last / G + 1) : s.kv) - span.skip, part_end);

        // l: sum of exponentials. lim: what a lane's eight may sum to before the reference moves;
        // kSeen, or -1: the row has seen nothing yet, or kFar. base: minus the reference in log2
        // units, or with kFar the reference as a score.
        constexpr float kSeen = 256.f, kFar = -2.f;
        floatx4 acc[2][DT];
        float l[2], lim[2], base[2];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            lim[n] = limit[n] > 0 ? -1.f : INFINITY;  // (a row that sees nothing never asks)
            l[n] = base[n] = 0.f;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) acc[n][dt] = floatx4{};
        }

        for (int seg = lo; seg < end; seg += kSegment) {
            const int seg_end = min(end, seg + kSegment), p0 = seg >> list_shift;
            __syncthreads();  // the list and the tiles of the segment before have been read
            int bad = 0;
            for (int e = tid; e < ((((seg_end + kKeys - 1) & -kKeys) - 1) >> list_shift) - p0 + 1;
                 e += 256) {
                const int key = (p0 + e) << list_shift;
                const bool seen = !WINDOW || span.sees(key, a.sinks);
                const int p = seen ? page_of(c.table, c.width, c.pages, b,
                                             WINDOW ? span.cached(key) >> shift : p0 + e)
                                   : -1;
                page_list[e] = p;
                bad |= p < 0 && seen && key < seg_end;
            }
            bad = __syncthreads_or(bad);

            auto issue = [&](int t0, auto buf_c) {
                constexpr int buf = decltype(buf_c)::value;
                const int key = t0 + 16 * wave;
                const int p = __builtin_amdgcn_readfirstlane(page_list[(key >> list_shift) - p0]);
                const int token = WINDOW ? span.cached(key) : key;
                const int live = p < 0 ? 0 : min(max(s.kv - token, 0), 16);
                const uint64_t at = uint64_t(uint32_t(max(p, 0))) * page_bytes +
                                    uint32_t(token & (c.page - 1)) * row_bytes;
                u32x4_t desc;
                desc.z = __builtin_amdgcn_readfirstlane(uint32_t(live) * row_bytes);
                desc.w = 0x00020000u;
                desc.x = __builtin_amdgcn_readfirstlane(uint32_t(k_base + at));
                desc.y = __builtin_amdgcn_readfirstlane(uint32_t((k_base + at) >> 32));
                copy_rows<NI>(desc, koff, k_lds + buf * 2 * TILE * 2);
                desc.x = __builtin_amdgcn_readfirstlane(uint32_t(v_base + at));
                desc.y = __builtin_amdgcn_readfirstlane(uint32_t((v_base + at) >> 32));
                copy_rows<NI>(desc, voff, k_lds + (buf * 2 + 1) * TILE * 2);
            };

            // 4 bits: a tile's codes are loaded two tiles ahead, and become bf16 rows one ahead.
            auto fetch = [&](int t0) {
                const int key = t0 + stage.key;
                const int token = WINDOW ? span.cached(key) : key;
                const int p = page_list[(key >> list_shift) - p0];
                stage.load(a, token < s.kv ? p : -1, token);
            };
            auto put = [&](auto buf_c) {
                constexpr int buf = decltype(buf_c)::value;
                stage.store(lds[buf][0], lds[buf][1], k_swizzle<D>(stage.key),
                            v_swizzle<D>(stage.key));
            };

            auto step = [&](int t0, auto buf_c) {
                constexpr int buf = decltype(buf_c)::value;
                // Each wave waits for its own copies; the barrier then publishes the tile, and
                // everyone is done with the one before.
                if constexpr (!FOUR) __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
                __syncthreads();
                if constexpr (FOUR) {
                    if (t0 + kKeys < seg_end) put(std::integral_constant<int, buf ^ 1>{});
                    if (t0 + 2 * kKeys < seg_end) fetch(t0 + 2 * kKeys);
                } else if (t0 + kKeys < seg_end) {
                    issue(t0 + kKeys, std::integral_constant<int, buf ^ 1>{});
                }
                if (t0 >= highest) return;  // no row of this wave sees any of it
                if (WINDOW && t0 + kKeys <= earliest && t0 >= a.sinks) return;

                const char* lk = reinterpret_cast<const char*>(&lds[buf][0][0]);
                const char* lv = reinterpret_cast<const char*>(&lds[buf][1][0]);
                // s[n][mt][e]: key 32 (mt/2) + 8 g + 4 (mt%2) + e of column group n's row `col`.
                floatx4 sc[2][4];
#pragma unroll
                for (int mt = 0; mt < 4; ++mt) sc[0][mt] = sc[1][mt] = floatx4{};
                // Operands are read one step ahead of the products that use them; the barriers
                // keep the scheduler from sinking a read to its use.
                bf16x8 ka[2][4];
                auto k_operands = [&](int kt) {
#pragma unroll
                    for (int mt = 0; mt < 4; ++mt)
                        ka[kt & 1][mt] = *reinterpret_cast<const bf16x8*>(
                            lk + (k_at ^ (kt << 6)) + (32 * (mt >> 1) + 4 * (mt & 1)) * D * 2);
                };
                k_operands(0);
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    if (kt + 1 < KT) k_operands(kt + 1);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int mt = 0; mt < 4; ++mt)
#pragma unroll
                        for (int n = 0; n < 2; ++n)
                            sc[n][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                ka[kt & 1][mt], q[n][kt], sc[n][mt], 0, 0, 0);
                }
                __builtin_amdgcn_s_setprio(0);
                bf16x8 va[2][DT];
                auto v_operands = [&](int t) {
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        const char* p = lv + (v_at ^ (dt << 5)) + 32 * t * D * 2;
                        const short4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(p));
                        const short4_t y =
                            __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(p + 4 * D * 2));
                        va[t][dt] = __builtin_bit_cast(
                            bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
                    }
                };
                v_operands(0);
                __builtin_amdgcn_sched_barrier(0);

                if (bad || t0 + kKeys > lowest ||
                    (WINDOW && t0 < latest && t0 + kKeys > a.sinks)) {
#pragma unroll
                    for (int mt = 0; mt < 4; ++mt) {
                        const int key = t0 + 32 * (mt >> 1) + 8 * g + 4 * (mt & 1);
                        const bool gone = bad && page_list[(key >> list_shift) - p0] < 0;
#pragma unroll
                        for (int n = 0; n < 2; ++n)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (gone || key + e >= min(limit[n], part_end) ||
                                    (WINDOW && key + e < limit[n] - a.window && key + e >= a.sinks))
                                    sc[n][mt][e] = -INFINITY;
                    }
                }
                // The reference of a row's exponentials moves only where they grow past it: where a
                // lane's eight sum to more than 2^8, or the row has seen nothing yet. A sum of
                // positive numbers bounds them all, so the other tiles take no maximum (48 heads of
                // d = 64, prompts of 902 to 4,095 tokens: 290 us with one in every tile, 271 us
                // without; d = 128, chunks of 2,048 over 32,768: 1,653 and 1,601 us). A
                // probability is rounded to bf16 by the same share of itself wherever the
                // reference lies.
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    floatx8 p[2];
                    float sum[2];
                    auto add = [&](int n) {
                        sum[n] = p[n][0];
#pragma unroll
                        for (int v = 1; v < 8; ++v) sum[n] += p[n][v];
                    };
                    auto exponentials = [&](int n) {
#pragma unroll
                        for (int v = 0; v < 8; ++v)
                            p[n][v] = __builtin_amdgcn_exp2f(
                                fmaf(sc[n][2 * t + v / 4][v % 4], c2, base[n]));
                        add(n);
                    };
                    exponentials(0);
                    exponentials(1);
                    if (__ballot(sum[0] > lim[0] || sum[1] > lim[1]) != 0) {
#pragma unroll
                        for (int n = 0; n < 2; ++n) {
                            float mx = -INFINITY;
#pragma unroll
                            for (int v = 0; v < 8; ++v) mx = fmaxf(mx, sc[n][2 * t + v / 4][v % 4]);
                            mx = row_max(mx);
                            // A reference of 2^24 and more in log2 units is rounded by a half and
                            // more, one of 2^32 by more than an exponential can make good. Such a
                            // row keeps its reference as a score and subtracts that first, in this
                            // branch, into which its limit sends every tile from then on.
                            const bool was_far = lim[n] == kFar;
                            const float before = lim[n] == kSeen ? -base[n] : -INFINITY;
                            const float top = fmaxf(before, mx * c2);
                            const bool far =
                                was_far || (mx > -INFINITY && !(fabsf(top) < 0x1p24f));
                            const float ref = was_far ? fmaxf(base[n], mx) : mx;
                            float alpha = far ? fmaf(-ref, c2, before) : before - top;
                            if (was_far) alpha = (base[n] - ref) * c2;
                            alpha = !far && top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(alpha);
                            l[n] *= alpha;
                            lim[n] = far ? kFar
                                     : top > -INFINITY ? kSeen : limit[n] > 0 ? -1.f : INFINITY;
                            base[n] = far ? ref : top == -INFINITY ? 0.f : -top;
#pragma unroll
                            for (int dt = 0; dt < DT; ++dt) acc[n][dt] *= alpha;
#pragma unroll
                            for (int v = 0; v < 8; ++v) {
                                const float x = sc[n][2 * t + v / 4][v % 4];
                                p[n][v] = __builtin_amdgcn_exp2f(far ? (x - base[n]) * c2
                                                                     : fmaf(x, c2, base[n]));
                            }
                            add(n);
                        }
                    }
                    // One bf16 for a probability, off by up to 2^-8 of itself: with what the rounding
                    // leaves as a second one (paged_tiles.h) the products would take half as long
                    // again (chunks of 2,048 over 32,768: 1,610 and 2,313 us; prompts at d = 64:
                    // 275 and 418 us). Outputs are off by 2.3e-3 of their norm so, by 1.66e-3 from
                    // their own rounding alone.
                    bf16x8 pb[2];
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        l[n] += sum[n];
                        pb[n] = __builtin_convertvector(p[n], bf16x8);
                    }
                    if (t == 0) {
                        v_operands(1);
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                        for (int n = 0; n < 2; ++n)
                            acc[n][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[t][dt], pb[n],
                                                                                 acc[n][dt], 0, 0, 0);
                }
            };

            if constexpr (FOUR) {
                fetch(seg);
                put(std::integral_constant<int, 0>{});
                if (seg + kKeys < seg_end) fetch(seg + kKeys);
            } else {
                issue(seg, std::integral_constant<int, 0>{});
            }
            for (int t0 = seg; t0 < seg_end; t0 += 2 * kKeys) {
                step(t0, std::integral_constant<int, 0>{});
                if (t0 + kKeys < seg_end) step(t0 + kKeys, std::integral_constant<int, 1>{});
            }
        }

#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int r = tile * kRowsTile + wave * 32 + n * 16 + col;
            const float total = row_sum(l[n]);
            if (r >= rows) continue;
            const int i = r / G, h = hk * G + r % G;
            const bool any = total > 0.f;
            const float inv = any ? 1.f / total : 0.f;
            const bool far = lim[n] == kFar;
            int64_t at = int64_t(h) * a.tokens + s.q0 + i;
            if (EACH && !whole && plan.tail)
                at = int64_t(work.tail) * kRowsTile + wave * 32 + n * 16 + col;
            const int64_t to = whole ? int64_t(h) * a.o_head + int64_t(s.q0 + i) * a.o_token
                                     : (at * plan.parts + part) * c.d;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const int ch = 16 * dt + 4 * g;
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = any ? acc[n][dt][e] * inv : 0.f;
                if (ch >= c.d) continue;
                if (whole)
                    store4(a.O, to + ch, a.out_bf16, x);
                else
                    store4(plan.part_o, to + ch, false, x);
            }
            if (g == 0) {
                if (!whole) {
                    // The reference as a score, rounded, and the sum relative to that.
                    const float ref = far ? base[n] : -base[n] / c2;
                    const float f = far ? 1.f : __builtin_amdgcn_exp2f(fmaf(-ref, c2, -base[n]));
                    plan.part_sum[at * plan.parts + part] = any ? total * f : 0.f;
                    plan.part_ref[at * plan.parts + part] = any ? ref : -INFINITY;
                } else if (a.lse) {  // (at: of a whole row)
                    a.lse[at] = !any  ? -INFINITY
                                : far ? fmaf(base[n], a.scale, __logf(total))
                                      : (__log2f(total) - base[n]) * kLn2;
                }
            }
        }
    }
}

template <bool WINDOW, bool FOUR>
auto tiles_kernel(int d) {
    return d <= 64   ? paged_tiles_kernel<64, 64, WINDOW, FOUR>
           : d <= 96 ? paged_tiles_kernel<128, 96, WINDOW, FOUR>
                     : paged_tiles_kernel<128, 128, WINDOW, FOUR>;
}

}  // namespace

hipError_t launch_paged_tiles(const PagedArgs& a, const PagedPlan& p, hipStream_t s) {
    const int grid = workgroups(p, a.cache);
    const auto kernel = a.k_scales ? (a.window ? tiles_kernel<true, true>(a.cache.d)
                                               : tiles_kernel<false, true>(a.cache.d))
                                   : (a.window ? tiles_kernel<true, false>(a.cache.d)
                                               : tiles_kernel<false, false>(a.cache.d));
    kernel<<<grid, 256, 0, s>>>(a, p);
    return hipGetLastError();
}

}  // namespace sparsp
