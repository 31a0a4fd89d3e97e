// Stand-ins for the device side of the bounded cache, beside those of cache_stub_launchers.cpp. The
// page calls touch what their checks say that they have.
#include <cstring>

#include "../../paper_2609_32197_amd/csrc/cache_launch.h"

extern int g_launches;

namespace sparsp {

static hipError_t launched() {
    ++g_launches;
    return hipSuccess;
}

// Every list of the workspace, to its last number.
static hipError_t listed(const PageArgs& a, int rows) {
    if (a.moves) *a.moves = 1;
    for (int i = 0; i < (a.pages + 16383) / 16384 + (rows + 1023) / 1024; ++i) a.counts[i] = 2;
    for (int i = 0; i < a.pages; ++i) a.src[i] = a.dst[i] = a.to[i] = 3;
    if (a.from)
        for (int i = 0; i < rows; ++i) a.from[i] = 4;
    return launched();
}

hipError_t launch_four_append(const FourArgs&, hipStream_t) { return launched(); }
hipError_t launch_four_read(const FourArgs&, hipStream_t) { return launched(); }
hipError_t launch_pages_reserve(const PageArgs& a, hipStream_t) { return listed(a, a.rows); }
hipError_t launch_pages_release(const PageArgs&, hipStream_t) { return launched(); }
hipError_t launch_pages_fork(const PageArgs& a, const PageBuffers&, hipStream_t) {
    return listed(a, a.rows);
}
hipError_t launch_pages_copy(const PageBuffers&, const int32_t*, const int32_t*, int, int, hipStream_t) {
    return launched();
}
hipError_t launch_pages_compact(const PageArgs& a, const PageBuffers&, hipStream_t) {
    return listed(a, a.rows);
}

}  // namespace sparsp
