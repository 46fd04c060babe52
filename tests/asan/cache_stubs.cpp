// Host stand-ins for the chunk cache's launchers: reached only by a call that passed
// validation, they report a launch failure.
#include <hip/hip_runtime_api.h>

#include "cache_plan.hpp"

namespace gca {
static int g_cache_launches = 0;
int cache_launches() { return g_cache_launches; }
static hipError_t launched() {
  ++g_cache_launches;
  return hipErrorLaunchFailure;
}
int64_t xattn_items(const gca_cache& c, int64_t nQ, int64_t rows) {
  return (int64_t)c.B * c.Hkv * nQ * ((c.H / c.Hkv * rows + 15) / 16);
}
hipError_t launch_cache_store(const gca_cache&, const void*, const void*, const void*, const int32_t*, const int32_t*,
                              int64_t, hipStream_t) {
  return launched();
}
hipError_t launch_cache_select(const gca_cache&, const void*, int32_t*, float*, float*, void*, hipStream_t) {
  return launched();
}
hipError_t launch_cache_xattn(const gca_cache&, const void*, const int32_t*, const float*, void*, float*, float*,
                              int64_t, int64_t, int, hipStream_t) {
  return launched();
}
hipError_t launch_cache_evict(const gca_cache&, const int32_t*, const float*, int64_t, float, int, int, const int32_t*,
                              int32_t*, int64_t, void*, hipStream_t) {
  return launched();
}
}  // namespace gca
