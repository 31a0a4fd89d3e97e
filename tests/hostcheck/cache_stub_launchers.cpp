// Stand-ins for the device side of the paged cache, beside those of stub_launchers.cpp.
#include "../../paper_2609_32197_amd/csrc/cache_launch.h"

extern int g_launches;

namespace sparsp {

static hipError_t launched() {
    ++g_launches;
    return hipSuccess;
}

hipError_t launch_rotate_rows(const RotateArgs&, hipStream_t) { return launched(); }
hipError_t launch_paged_attn(const PagedArgs&, hipStream_t) { return launched(); }
int64_t paged_attn_workspace(const PagedArgs&) { return 4096; }
hipError_t launch_paged_weights(const PagedArgs&, hipStream_t) { return launched(); }
hipError_t launch_cache_evict(const sparsp_cache&, int, int, int, const int32_t*, int, int32_t*,
                              int32_t*, void*, int64_t, hipStream_t) { return launched(); }
int64_t evict_workspace(const sparsp_cache&) { return 8192; }

}  // namespace sparsp
