// Stand-ins for the launchers behind the paged cache's front end (csrc/paged_api.hip), so that its host-side validation can run
// inside a sanitizer build on a machine without a GPU.
#include "../../paper_2601_01298_amd/csrc/paged_internal.h"

extern "C" int g_paged_launches = 0;
extern "C" double g_turns[64] = {};
extern "C" unsigned char g_axis[64] = {};

namespace ws {

hipError_t launch_paged_append(const ws_paged_cache &, const ws_rows &, const ws_rows &, int, const int32_t *, const int32_t *,
                               const RotaryTable &rot, const ws_rows *, int, void *, const int32_t *, int32_t *, float *, hipStream_t)
{
    ++g_paged_launches;
    for (int c = 0; c < 64; ++c) g_turns[c] = rot.turns[c], g_axis[c] = rot.axis[c];
    return hipSuccess;
}
hipError_t launch_paged_attend(const ws_paged_cache &, const void *, int, float, float *, float *, float, const float *, float *, void *,
                               hipStream_t)
{
    ++g_paged_launches;
    return hipSuccess;
}
hipError_t launch_paged_evict(const ws_paged_cache &, int, int, int, const int32_t *, const float *, float *, const int32_t *, int32_t *,
                              int32_t *, int32_t *, void *, hipStream_t)
{
    ++g_paged_launches;
    return hipSuccess;
}

}  // namespace ws
