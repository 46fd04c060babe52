// Host stand-ins for the token window's launchers and plans: the launchers are reached only by a call
// that passed validation, and report a launch failure.
#include <hip/hip_runtime_api.h>

#include "window_plan.hpp"

namespace gca {
static int g_window_launches = 0;
int window_launches() { return g_window_launches; }
static hipError_t launched() {
  ++g_window_launches;
  return hipErrorLaunchFailure;
}
size_t window_workspace(const gca_window& w, int64_t T) { return align256((size_t)w.H * (size_t)T); }
size_t verify_workspace(int64_t B, int64_t T, int64_t V) { return align256((size_t)(B * T + V)); }
hipError_t launch_window_append(const gca_window&, const void*, const void*, const int32_t*, int64_t, hipStream_t) {
  return launched();
}
hipError_t launch_window_attn(const gca_window&, const void*, const int32_t*, const int32_t*, const float*, void*,
                              float*, int64_t, void*, hipStream_t) {
  return launched();
}
hipError_t launch_window_keep(const gca_window&, const int32_t*, int64_t, const int32_t*, int64_t, hipStream_t) {
  return launched();
}
hipError_t launch_verify(int64_t, int64_t, int64_t, const float*, const float*, const int32_t*, const int32_t*,
                         const float*, const int32_t*, int32_t*, int32_t*, int32_t*, void*, hipStream_t) {
  return launched();
}
}  // namespace gca
