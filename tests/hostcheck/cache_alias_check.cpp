// Tensors given twice to a call that writes them: refused where two writes, or a write and a read, would
// meet, and taken where the call allows it. Exits with the number of failures.
#include <cstdio>

#include "../../include/sparsp_cache.h"

extern int g_launches;
static int g_bad = 0, g_checks = 0;

static void expect(const char* what, int got, int want) {
    ++g_checks;
    if (got != want || g_launches != (want == SPARSP_OK)) {
        ++g_bad;
        printf("FAIL %s: %d for %d, %d launches: %s\n", what, got, want, g_launches,
               sparsp_last_error());
    }
    g_launches = 0;
}

int main() {
    static char spot[6][16] __attribute__((aligned(16)));
    int32_t array[4] = {}, len[4] = {}, kept[4] = {};
    float f[4] = {1.f, 1.f, 1.f, 1.f};
    const int d = 8, n = 3, OK = SPARSP_OK, I = SPARSP_E_INVALID;
    const sparsp_rotary r = {d, SPARSP_ROPE_HALF, 1, {d / 2, 0, 0}, 1.0f, 0};
    auto rows = [&](int k) { return sparsp_rows{spot[k], int64_t(n) * d, d, 1, 0}; };
    const sparsp_rows A = rows(0), B = rows(1), C = rows(2), D = rows(3);
    auto rope = [&](sparsp_rows x0, sparsp_rows x1, sparsp_rows y0, sparsp_rows y1) {
        const sparsp_rows x[2] = {x0, x1}, y[2] = {y0, y1};
        return sparsp_rope(&r, n, d, SPARSP_BF16, x, y, 2, array, 32, f, nullptr);
    };
    expect("rope apart", rope(A, B, C, D), OK);
    expect("rope in place", rope(A, B, A, B), OK);
    expect("rope of one tensor", rope(A, A, C, D), OK);
    expect("rope into one tensor", rope(A, B, C, C), I);
    expect("rope in place twice", rope(A, A, A, A), I);
    expect("rope into the other's input", rope(A, B, B, C), I);
    expect("rope into the other's input", rope(A, B, C, A), I);

    // Empty tensors have no address of their own.
    const sparsp_rows none[2] = {A, A};
    const int rc = sparsp_rope(&r, 0, d, SPARSP_BF16, none, none, 2, array, 32, f, nullptr);
    g_launches += 1;  // (nothing is launched)
    expect("rope of nothing", rc, OK);

    sparsp_cache c = {};
    c.K = spot[4];
    c.V = spot[5];
    c.weights = f;
    c.table = c.new_off = c.kv_len = array;
    c.pages = c.H = c.width = c.B = 1;
    c.page = 16;
    c.d = d;
    c.dtype = SPARSP_BF16;
    auto append = [&](sparsp_rows K, sparsp_rows V, sparsp_rows Q, sparsp_rows out) {
        return sparsp_paged_append(&c, n, &K, &V, &r, array, 32, f, &Q, &out, nullptr);
    };
    expect("append", append(A, B, C, D), OK);
    expect("append of one tensor", append(A, A, A, D), OK);
    expect("append, Q in place", append(A, B, C, C), OK);
    auto evict = [&](int32_t* out, int32_t* list) {
        return sparsp_cache_evict(&c, 3, 0, 0, nullptr, 0, out, list, nullptr, 0, nullptr);
    };
    expect("evict", evict(len, kept), OK);
    expect("evict, one array for both", evict(len, len), I);
    expect("evict, the list over the lengths", evict(len, array), I);
    c.V = c.K;
    expect("attention of K as V", sparsp_paged_attn(&c, n, &A, &B, SPARSP_BF16, nullptr, 1, 1.f, 0, 0,
                                                    nullptr, 0, nullptr), OK);
    expect("weights of K as V", sparsp_paged_weights(&c, n, &A, f, 1, 1.f, 1, 0, 0, nullptr), OK);
    expect("append, K is V", append(A, B, C, D), I);
    expect("evict, K is V", evict(len, kept), I);
    printf("%d checks, %d failures\n", g_checks, g_bad);
    return g_bad != 0;
}
