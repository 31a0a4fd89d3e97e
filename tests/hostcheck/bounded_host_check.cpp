// The C ABI of the bounded cache without a GPU: the page calls' workspaces, which the stand-in
// launchers fill, and the paths into the launchers. Exits with the number of failures.
#include <cstdio>
#include <vector>

#include "../../include/sparsp_bounded.h"

extern int g_launches;
static int g_bad = 0, g_checks = 0;

static void expect(const char* what, int64_t got, int64_t want, int launches) {
    ++g_checks;
    const bool message = (want < 0) == (sparsp_last_error()[0] != 0);
    if (got != want || g_launches != launches || !message) {
        ++g_bad;
        printf("FAIL %s: %lld for %lld, %d launches, \"%s\"\n", what, (long long)got, (long long)want,
               g_launches, sparsp_last_error());
    }
    g_launches = 0;
}

struct alignas(16) Sixteen {
    int32_t x[4];
};

static void* at(uintptr_t x) { return reinterpret_cast<void*>(x << 20); }
static int32_t* ints(uintptr_t x) { return static_cast<int32_t*>(at(x)); }
static uint8_t* bytes(uintptr_t x) { return static_cast<uint8_t*>(at(x)); }

static void page_calls(int pages, int B, int rows) {
    sparsp_pages p = {ints(1), ints(2), ints(3), pages, 16, 7, B};
    const int64_t need = sparsp_pages_workspace_bytes(&p, rows);
    // (its own allocation, so that the sanitizer sees the first byte behind it)
    std::vector<Sixteen> exact(need / 16 + (need % 16 != 0));
    void* ws = exact.data();
    sparsp_page_buffer b[2] = {{at(8), 64}, {at(9), 1 << 20}};
    expect("reserve", sparsp_pages_reserve(&p, ints(4), ints(5), ws, need, nullptr), 0, 1);
    expect("fork", sparsp_pages_fork(&p, ints(4), rows, b, 2, ints(5), ints(6), ints(7), ints(10), ws,
                                     need, nullptr), 0, 1);
    expect("compact", sparsp_pages_compact(&p, b, 2, ints(5), ints(6), ints(7), ws, need, nullptr), 0, 1);
    expect("fork of less", sparsp_pages_fork(&p, ints(4), rows, b, 2, ints(5), ints(6), ints(7), ints(10),
                                             ws, 15, nullptr), SPARSP_E_CAPACITY, 0);
    expect("release", sparsp_pages_release(&p, 5, 2, nullptr), 0, 1);
    expect("copy", sparsp_pages_copy(b, 2, pages, ints(5), ints(6), 3, nullptr), 0, 1);
}

int main() {
    for (int pages : {1, 5, 16384, 16385, 50000})
        for (int B : {1, 1024, 1025, 9000})
            for (int rows : {1, 1024, 3000}) page_calls(pages, B, rows);
    sparsp_cache4 c = {bytes(1), bytes(2), bytes(3), bytes(4), ints(5), ints(6), ints(7),
                       10, 2, 32, 64, 4, 3, {0, 0}};
    const sparsp_rows K = {at(8), 320, 64, 2, 0}, V = {at(9), 320, 64, 2, 0}, Q = {at(10), 320, 64, 4, 0},
                      O = {at(11), 320, 64, 4, 0};
    const sparsp_rotary r = {64, SPARSP_ROPE_HALF, 1, {32, 0, 0}, 1.0f, 0};
    const float* f = static_cast<float*>(at(12));
    expect("append4", sparsp_paged_append4(&c, 5, SPARSP_BF16, &K, &V, &r, at(13), 32, f, &Q, &O, nullptr),
           0, 1);
    expect("append4 as it is", sparsp_paged_append4(&c, 5, SPARSP_F32, &K, &V, nullptr, nullptr, 0, nullptr,
                                                    nullptr, nullptr, nullptr), 0, 1);
    expect("read4", sparsp_paged_read4(&c, 5, SPARSP_BF16, &K, &V, nullptr), 0, 1);
    expect("attn4", sparsp_paged_attn4(&c, 5, SPARSP_BF16, &Q, &O, SPARSP_F32, nullptr, 1, 0, 0, 0.1f, 0, 0,
                                       nullptr, 0, nullptr), 0, 1);
    expect("attn4 window", sparsp_paged_attn4(&c, 5, SPARSP_F32, &Q, &O, SPARSP_F32, nullptr, 1, 1 << 30,
                                              2147483647, 0.1f, 0, 0, nullptr, 0, nullptr), 0, 1);
    expect("attn4 workspace", sparsp_paged_attn4_workspace_bytes(&c, 5, SPARSP_BF16, 4, 0, 0, 0, 0), 4096, 0);
    sparsp_cache w = {at(1), at(2), nullptr, ints(3), ints(4), ints(5), 10, 2, 32, 64, SPARSP_BF16, 4, 3, 0};
    expect("window", sparsp_paged_attn_window(&w, 5, &Q, &O, SPARSP_BF16, nullptr, 7, 2, 0.1f, 0, 0, nullptr,
                                              0, nullptr), 0, 1);
    expect("window 0", sparsp_paged_attn_window(&w, 5, &Q, &O, SPARSP_BF16, nullptr, 0, 2, 0.1f, 0, 0,
                                                nullptr, 0, nullptr), SPARSP_E_INVALID, 0);
    printf("%d checks, %d failures\n", g_checks, g_bad);
    return g_bad;
}
