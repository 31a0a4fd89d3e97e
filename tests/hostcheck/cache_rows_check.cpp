// Strides of the row tensors that a call writes, against a search over all pairs of rows: refused
// exactly where two of them share a channel. Exits with the number of failures.
#include <cstdio>
#include <cstdlib>

#include "../../include/sparsp_cache.h"

extern int g_launches;

static bool shares(int heads, int tokens, int64_t hs, int64_t ts, int d) {
    for (int64_t h = 0; h < heads; ++h)
        for (int64_t t = 0; t < tokens; ++t)
            for (int64_t k = 0; k < heads; ++k)
                for (int64_t u = 0; u < tokens; ++u) {
                    const int64_t apart = llabs(h * hs + t * ts - k * hs - u * ts);
                    if ((h != k || t != u) && apart < d) return true;
                }
    return false;
}

int main() {
    int bad = 0, checks = 0, refused = 0;
    const int d = 8;
    static char spot[3][16] __attribute__((aligned(16)));
    const sparsp_rotary r = {d, SPARSP_ROPE_HALF, 1, {d / 2, 0, 0}, 1.0f, 0};
    auto expect = [&](const char* what, int got, int want, int heads, int tokens, int64_t hs,
                      int64_t ts) {
        ++checks;
        if (got != want || g_launches != (want == SPARSP_OK)) {
            ++bad;
            printf("FAIL %s: %d for %d, heads %d (%lld) tokens %d (%lld): %s\n", what, got, want,
                   heads, (long long)hs, tokens, (long long)ts, sparsp_last_error());
        }
        g_launches = 0;
    };
    sparsp_cache c = {};
    c.K = c.V = spot[0];
    c.V = spot[1];
    int32_t array[4] = {};
    c.table = c.new_off = c.kv_len = array;
    c.pages = c.H = c.width = c.B = 1;
    c.page = 16;
    c.d = d;
    c.dtype = SPARSP_BF16;
    float f = 1.f;
    for (int heads = 1; heads <= 5; ++heads)
        for (int tokens = 1; tokens <= 5; ++tokens)
            for (int64_t hs = 8; hs <= 64; hs += 8)
                for (int64_t ts = 8; ts <= 64; ts += 8) {
                    const bool share = shares(heads, tokens, hs, ts, d);
                    const int want = share ? SPARSP_E_INVALID : SPARSP_OK;
                    refused += share;
                    const sparsp_rows x = {spot[2], int64_t(tokens) * d, d, heads, 0};
                    const sparsp_rows y = {array, hs, ts, heads, 0};
                    sparsp_rows o = y;
                    o.data = spot[0];
                    expect("rope", sparsp_rope(&r, tokens, d, SPARSP_BF16, &x, &o, 1, array, 32, &f,
                                               nullptr), want, heads, tokens, hs, ts);
                    expect("rope in place", sparsp_rope(&r, tokens, d, SPARSP_BF16, &o, &o, 1, array,
                                                        32, &f, nullptr), want, heads, tokens, hs, ts);
                    expect("attention", sparsp_paged_attn(&c, tokens, &x, &o, SPARSP_BF16, nullptr, 1,
                                                          1.f, 0, 0, nullptr, 0, nullptr),
                           want, heads, tokens, hs, ts);
                    const sparsp_rows kv = {spot[2], int64_t(tokens) * d, d, 1, 0};
                    expect("append", sparsp_paged_append(&c, tokens, &kv, &kv, &r, array, 32, &f, &x,
                                                         &o, nullptr), want, heads, tokens, hs, ts);
                    // Rows that are only read may share channels.
                    expect("weights' Q", sparsp_paged_attn(&c, tokens, &o, &x, SPARSP_BF16, nullptr, 1,
                                                           1.f, 0, 0, nullptr, 0, nullptr),
                           SPARSP_OK, heads, tokens, hs, ts);
                }
    // The largest sizes: products of strides and counts pass 64 bits.
    const int most = 1 << 26;
    const int64_t wide = int64_t(1) << 40;
    for (int k = 0; k < 4; ++k) {
        const int64_t hs = k & 1 ? wide : 8, ts = k & 2 ? wide : 8;
        const sparsp_rows x = {spot[2], 8, int64_t(1024) * 8, 1024, 0}, o = {spot[0], hs, ts, 1024, 0};
        // (8 and 8 share; 2^40 and 8 hold 2^26 rows of a head; 8 and 2^40 hold 1,024 of a token; and
        // with both 2^40 rows (h, t) and (h - 1, t + 1) share)
        expect("large", sparsp_rope(&r, most, 8, SPARSP_BF16, &x, &o, 1, array, 32, &f, nullptr),
               k == 0 || k == 3 ? SPARSP_E_INVALID : SPARSP_OK, 1024, most, hs, ts);
    }
    printf("%d checks, %d refused, %d failures\n", checks, refused, bad);
    return bad != 0;
}
