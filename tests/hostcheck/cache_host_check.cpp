// The C ABI of the paged cache without a GPU: every refusal, the paths into the launchers, and
// the rotary frequencies. Exits with the number of failures.
#include <climits>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <functional>

#include "../../include/sparsp_cache.h"

extern int g_launches;
static int g_bad = 0, g_checks = 0;

static void expect(const char* what, int64_t got, int64_t want, int launches) {
    ++g_checks;
    const bool message = (want < 0) == (sparsp_last_error()[0] != 0);
    if (got != want || g_launches != launches || !message) {
        ++g_bad;
        printf("FAIL %s: %lld for %lld, %d launches, \"%s\"\n", what, (long long)got,
               (long long)want, g_launches, sparsp_last_error());
    }
    g_launches = 0;
}

static void* at(uintptr_t x) { return reinterpret_cast<void*>(x); }
static int32_t* ints(uintptr_t x) { return static_cast<int32_t*>(at(x)); }
static float* floats(uintptr_t x) { return static_cast<float*>(at(x)); }

static sparsp_cache cache() {
    sparsp_cache c = {};
    c.K = at(1 << 20);
    c.V = at(2 << 20);
    c.weights = floats(3 << 20);
    c.table = ints(4 << 20);
    c.new_off = ints(5 << 20);
    c.kv_len = ints(6 << 20);
    c.pages = 10;
    c.H = 2;
    c.page = 32;
    c.d = 64;
    c.dtype = SPARSP_BF16;
    c.width = 4;
    c.B = 3;
    return c;
}
static sparsp_rows rows(int heads, int tokens = 5, int d = 64) {
    return {at(7 << 20), int64_t(tokens) * d, d, heads, 0};
}
static sparsp_rotary rotary() { return {64, SPARSP_ROPE_HALF, 1, {32, 0, 0}, 1.0f, 0}; }

struct Call {
    sparsp_cache c = cache();
    sparsp_rows K = rows(2), V = rows(2), Q = rows(4), O = rows(4);
    sparsp_rotary r = rotary();
    void* pos = at(8 << 20);
    int bits = 32, tokens = 5, out = SPARSP_BF16, max_new = 0, max_kv = 0;
    float* freq = floats(9 << 20);
    float scale = 0.125f;
    float* lse = floats(10 << 20);
    void* ws = at(11 << 20);
    int64_t ws_bytes = 1000;
    int keep = 40, first = 1, recent = 2, dst_width = 2;
    int32_t *dst = nullptr, *len = ints(12 << 20), *kept = ints(13 << 20);
    Call() { O.data = at(14 << 20); }
    int append() {
        return sparsp_paged_append(&c, tokens, &K, &V, &r, pos, bits, freq, &Q, &O, nullptr);
    }
    int attend() {
        return sparsp_paged_attn(&c, tokens, &Q, &O, out, lse, 1, scale, max_new, max_kv, ws,
                                 ws_bytes, nullptr);
    }
    int weigh() {
        return sparsp_paged_weights(&c, tokens, &Q, lse, 1, scale, 1, max_new, max_kv, nullptr);
    }
    int evict() {
        return sparsp_cache_evict(&c, keep, first, recent, dst, dst_width, len, kept, ws, ws_bytes,
                                  nullptr);
    }
    int rope() { return sparsp_rope(&r, tokens, 64, c.dtype, &Q, &O, 1, pos, bits, freq, nullptr); }
};

using Change = std::function<void(Call&)>;

int main() {
    enum { APPEND = 1, ATTEND = 2, WEIGH = 4, EVICT = 8, ROPE = 16 };
    struct Case {
        const char* what;
        int calls, want;
        Change change;
    };
    const int I = SPARSP_E_INVALID, U = SPARSP_E_UNSUPPORTED, T = SPARSP_E_DTYPE, C = SPARSP_E_CAPACITY;
    const int all = APPEND | ATTEND | WEIGH | EVICT;
    const Case cases[] = {
        {"as it is", all | ROPE, SPARSP_OK, [](Call&) {}},
        {"float32", all, SPARSP_OK, [](Call& x) { x.c.dtype = SPARSP_F32; x.out = SPARSP_F32; }},
        {"no weights where none are needed", APPEND | ATTEND, SPARSP_OK, [](Call& x) { x.c.weights = nullptr; }},
        {"no workspace, no lse", ATTEND, SPARSP_OK, [](Call& x) { x.ws = nullptr; x.lse = nullptr; }},
        {"dtype", all, T, [](Call& x) { x.c.dtype = 2; }},
        {"d = 0", all, I, [](Call& x) { x.c.d = 0; }},
        {"d = 136", all, U, [](Call& x) { x.c.d = 136; }},
        {"d = 60 in bf16", all, U, [](Call& x) { x.c.d = 60; }},
        {"no pages", all, I, [](Call& x) { x.c.pages = 0; }},
        {"no width", all, I, [](Call& x) { x.c.width = 0; }},
        {"no sequence", all, I, [](Call& x) { x.c.B = 0; }},
        {"too many sequences", all, U, [](Call& x) { x.c.B = 65537; }},
        {"too many pairs", all, U, [](Call& x) { x.c.B = 65536; x.c.H = 17; }},
        {"no head", all, U, [](Call& x) { x.c.H = 0; }},
        {"page 8", all, U, [](Call& x) { x.c.page = 8; }},
        {"page 48", all, U, [](Call& x) { x.c.page = 48; }},
        {"page 512", all, U, [](Call& x) { x.c.page = 512; }},
        {"negative page", all, U, [](Call& x) { x.c.page = INT_MIN; }},
        {"width * page", all, U, [](Call& x) { x.c.width = 1 << 26; }},
        {"K NULL", all, I, [](Call& x) { x.c.K = nullptr; }},
        {"V NULL", APPEND | ATTEND | EVICT, I, [](Call& x) { x.c.V = nullptr; }},
        {"V not needed", WEIGH, SPARSP_OK, [](Call& x) { x.c.V = nullptr; }},
        {"table NULL", all, I, [](Call& x) { x.c.table = nullptr; }},
        {"kv_len NULL", all, I, [](Call& x) { x.c.kv_len = nullptr; }},
        {"new_off NULL", APPEND | ATTEND | WEIGH, I, [](Call& x) { x.c.new_off = nullptr; }},
        {"new_off not needed", EVICT, SPARSP_OK, [](Call& x) { x.c.new_off = nullptr; }},
        {"weights NULL", WEIGH | EVICT, I, [](Call& x) { x.c.weights = nullptr; }},
        {"K misaligned", all, I, [](Call& x) { x.c.K = at((1 << 20) + 8); }},
        {"tokens < 0", APPEND | ATTEND | WEIGH | ROPE, I, [](Call& x) { x.tokens = -1; }},
        {"too many tokens", APPEND | ATTEND | WEIGH | ROPE, I, [](Call& x) { x.tokens = INT_MAX; }},
        {"rows NULL", APPEND | ATTEND | WEIGH | ROPE, I, [](Call& x) { x.Q.data = nullptr; }},
        {"rows misaligned", APPEND | ATTEND | WEIGH | ROPE, I, [](Call& x) { x.Q.data = at((7 << 20) + 2); }},
        {"stride no multiple of 16 bytes", APPEND | ATTEND | WEIGH | ROPE, I, [](Call& x) { x.Q.token_stride = 68; }},
        {"stride below d", APPEND | ATTEND | WEIGH | ROPE, I, [](Call& x) { x.Q.token_stride = 0; }},
        {"negative stride", APPEND | ATTEND | WEIGH | ROPE, I, [](Call& x) { x.Q.head_stride = -64; }},
        {"too many heads", APPEND | ATTEND | WEIGH | ROPE, U, [](Call& x) { x.Q.heads = 1025; }},
        {"heads no multiple", ATTEND | WEIGH, I, [](Call& x) { x.Q.heads = 3; }},
        {"K heads", APPEND, I, [](Call& x) { x.K = rows(1); }},
        {"O heads", ATTEND | APPEND | ROPE, I, [](Call& x) { x.O.heads = 2; }},
        {"O is Q", ATTEND, I, [](Call& x) { x.O = x.Q; }},
        {"in place", APPEND | ROPE, SPARSP_OK, [](Call& x) { x.O = x.Q; }},
        {"in place, other strides", APPEND | ROPE, I, [](Call& x) { x.O = x.Q; x.O.head_stride += 64; }},
        {"out_dtype", ATTEND, T, [](Call& x) { x.out = 5; }},
        {"bf16 from f32", ATTEND, T, [](Call& x) { x.c.dtype = SPARSP_F32; }},
        {"too many rows", ATTEND | WEIGH, U, [](Call& x) { x.tokens = 1 << 26; x.c.H = 1; x.Q = rows(32); x.O = rows(32); x.O.data = at(14 << 20); }},
        {"scale 0", ATTEND | WEIGH, I, [](Call& x) { x.scale = 0; }},
        {"scale NaN", ATTEND | WEIGH, I, [](Call& x) { x.scale = NAN; }},
        {"scale inf", ATTEND | WEIGH, I, [](Call& x) { x.scale = INFINITY; }},
        {"max_new < 0", ATTEND | WEIGH, I, [](Call& x) { x.max_new = -1; }},
        {"max_kv < 0", ATTEND | WEIGH, I, [](Call& x) { x.max_kv = -1; }},
        {"workspace misaligned", ATTEND | EVICT, I, [](Call& x) { x.ws = at((11 << 20) + 4); }},
        {"workspace_bytes < 0", ATTEND | EVICT, I, [](Call& x) { x.ws_bytes = -1; }},
        {"lse NULL", WEIGH, I, [](Call& x) { x.lse = nullptr; }},
        {"rot_dim odd", APPEND | ROPE, I, [](Call& x) { x.r.rot_dim = 33; }},
        {"rot_dim 0", APPEND | ROPE, I, [](Call& x) { x.r.rot_dim = 0; }},
        {"rot_dim > d", APPEND | ROPE, I, [](Call& x) { x.r.rot_dim = 66; }},
        {"layout", APPEND | ROPE, I, [](Call& x) { x.r.layout = 2; }},
        {"axes 0", APPEND | ROPE, I, [](Call& x) { x.r.axes = 0; }},
        {"axes 4", APPEND | ROPE, I, [](Call& x) { x.r.axes = 4; }},
        {"pairs", APPEND | ROPE, I, [](Call& x) { x.r.axis_pairs[0] = 31; }},
        {"negative pairs", APPEND | ROPE, I, [](Call& x) { x.r.axes = 2; x.r.axis_pairs[0] = 40; x.r.axis_pairs[1] = -8; }},
        {"factor", APPEND | ROPE, I, [](Call& x) { x.r.factor = INFINITY; }},
        {"positions NULL", APPEND | ROPE, I, [](Call& x) { x.pos = nullptr; }},
        {"frequencies NULL", APPEND | ROPE, I, [](Call& x) { x.freq = nullptr; }},
        {"position bits", APPEND | ROPE, T, [](Call& x) { x.bits = 16; }},
        {"keep 0", EVICT, I, [](Call& x) { x.keep = 0; }},
        {"first < 0", EVICT, I, [](Call& x) { x.first = -1; }},
        {"recent < 0", EVICT, I, [](Call& x) { x.recent = -1; }},
        {"first + recent", EVICT, I, [](Call& x) { x.first = 20; x.recent = 21; }},
        {"first + recent past 32 bits", EVICT, I, [](Call& x) { x.first = x.recent = INT_MAX; }},
        {"kv_len_out is kv_len", EVICT, I, [](Call& x) { x.len = const_cast<int32_t*>(x.c.kv_len); }},
        {"kept NULL", EVICT, I, [](Call& x) { x.kept = nullptr; }},
        {"other pages", EVICT, SPARSP_OK, [](Call& x) { x.dst = ints(15 << 20); }},
        {"too few other pages", EVICT, C, [](Call& x) { x.dst = ints(15 << 20); x.dst_width = 1; }},
        {"dst_table is table", EVICT, I, [](Call& x) { x.dst = const_cast<int32_t*>(x.c.table); }},
    };
    for (const Case& k : cases) {
        const int launches = k.want == SPARSP_OK;
        auto one = [&](int which, int (Call::*call)()) {
            if (!(k.calls & which)) return;
            Call x;
            k.change(x);
            expect(k.what, (x.*call)(), k.want, launches);
        };
        one(APPEND, &Call::append);
        one(ATTEND, &Call::attend);
        one(WEIGH, &Call::weigh);
        one(EVICT, &Call::evict);
        one(ROPE, &Call::rope);
    }
    Call x;
    expect("cache NULL", sparsp_paged_attn(nullptr, 5, &x.Q, &x.O, 1, nullptr, 1, 1.f, 0, 0, nullptr, 0, nullptr), I, 0);
    expect("cache NULL", sparsp_cache_evict(nullptr, 1, 0, 0, nullptr, 0, x.len, x.kept, nullptr, 0, nullptr), I, 0);
    expect("K alone", sparsp_paged_append(&x.c, 5, &x.K, &x.V, nullptr, nullptr, 0, nullptr, nullptr, nullptr, nullptr), SPARSP_OK, 1);
    expect("Q, no rotation", sparsp_paged_append(&x.c, 5, &x.K, &x.V, nullptr, nullptr, 0, nullptr, &x.Q, &x.O, nullptr), I, 0);
    expect("Q, no Q_out", sparsp_paged_append(&x.c, 5, &x.K, &x.V, &x.r, x.pos, 32, x.freq, &x.Q, nullptr, nullptr), I, 0);
    expect("rope of three", sparsp_rope(&x.r, 5, 64, 1, &x.Q, &x.O, 3, x.pos, 32, x.freq, nullptr), I, 0);
    expect("rope of none", sparsp_rope(&x.r, 5, 64, 1, nullptr, &x.O, 1, x.pos, 32, x.freq, nullptr), I, 0);
    expect("rope, no rotation", sparsp_rope(nullptr, 5, 64, 1, &x.Q, &x.O, 1, x.pos, 32, x.freq, nullptr), I, 0);
    x.tokens = 0;
    expect("no tokens", x.append(), SPARSP_OK, 0);
    expect("no tokens", x.attend(), SPARSP_OK, 0);
    expect("no tokens", x.weigh(), SPARSP_OK, 0);
    expect("no tokens", x.rope(), SPARSP_OK, 0);
    expect("workspace", sparsp_paged_attn_workspace_bytes(&x.c, 5, 4, 0, 0), 4096, 0);
    expect("workspace of none", sparsp_paged_attn_workspace_bytes(&x.c, 0, 4, 0, 0), 0, 0);
    expect("workspace heads", sparsp_paged_attn_workspace_bytes(&x.c, 5, 3, 0, 0), I, 0);
    expect("workspace NULL", sparsp_paged_attn_workspace_bytes(nullptr, 5, 4, 0, 0), I, 0);

    expect("evict workspace", sparsp_cache_evict_workspace_bytes(&x.c), 8192, 0);
    expect("evict workspace NULL", sparsp_cache_evict_workspace_bytes(nullptr), I, 0);

    float f[128], s;
    expect("frequencies", sparsp_rope_frequencies(256, 1e4, 0, 0, 0, 0, 0, f, &s), SPARSP_OK, 0);
    expect("frequencies odd", sparsp_rope_frequencies(7, 1e4, 0, 1, 0, 0, 0, f, &s), I, 0);
    expect("frequencies 258", sparsp_rope_frequencies(258, 1e4, 0, 1, 0, 0, 0, f, &s), I, 0);
    expect("theta", sparsp_rope_frequencies(8, 0.0, 0, 1, 0, 0, 0, f, &s), I, 0);
    expect("theta NaN", sparsp_rope_frequencies(8, NAN, 0, 1, 0, 0, 0, f, &s), I, 0);
    expect("scaling", sparsp_rope_frequencies(8, 1e4, 4, 1, 0, 0, 0, f, &s), I, 0);
    expect("scale", sparsp_rope_frequencies(8, 1e4, 1, 0.5, 0, 0, 0, f, &s), I, 0);
    expect("base of one pair", sparsp_rope_frequencies(2, 1e4, 2, 2, 0, 0, 0, f, &s), I, 0);
    expect("parts untrained", sparsp_rope_frequencies(8, 1e4, 3, 2, 0, 1, 32, f, &s), I, 0);
    expect("parts ramp", sparsp_rope_frequencies(8, 1e4, 3, 2, 100, 3, 3, f, &s), I, 0);
    expect("no output", sparsp_rope_frequencies(8, 1e4, 0, 1, 0, 0, 0, nullptr, &s), I, 0);
    printf("%d checks, %d failures\n", g_checks, g_bad);
    return g_bad != 0;
}
