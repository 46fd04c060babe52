// Drives the token window's and the verification's entry points through their checks on the host, and
// each once into a (stubbed) launch.  Prints OK and exits 0 when every status is the expected one.
#include <climits>
#include <cstdio>
#include <cstring>

#include "gca.h"

namespace gca {
int window_launches();
}

static int g_fail = 0;
#define EXPECT(cond)                                                                   \
  do {                                                                                 \
    if (!(cond)) {                                                                     \
      std::fprintf(stderr, "line %d: %s (%s)\n", __LINE__, #cond, gca_last_error()); \
      ++g_fail;                                                                        \
    }                                                                                  \
  } while (0)

int main() {
  alignas(256) static unsigned char mem[4096];
  void* A = mem;
  int32_t* I = reinterpret_cast<int32_t*>(mem);
  float* F = reinterpret_cast<float*>(mem);
  const size_t big = size_t(1) << 40;
  gca_window w;
  std::memset(&w, 0, sizeof w);
  w.B = 2; w.H = 8; w.Hkv = 4; w.d = 64; w.capacity = 20032; w.window = 500;
  w.attn_scale = -1.f; w.dtype = GCA_FP32; w.format = GCA_INT8;
  auto all = [&](const gca_window* p, int64_t T, gca_status want) {
    EXPECT(gca_window_append(p, A, A, I, T, nullptr) == want);
    EXPECT(gca_window_attn(p, A, nullptr, I, F, A, F, T, A, big, nullptr) == want);
    EXPECT(gca_window_keep(p, I, 3, I, T, nullptr) == want);
  };
  all(nullptr, 3, GCA_ERR_INVALID);
  all(&w, 3, GCA_ERR_INVALID);  // no members
  w.k = w.v = A;
  w.k_scale = w.v_scale = F;
  w.length = w.ticket = I;
  const int32_t most[] = {0, -1, INT_MAX, INT_MIN};
  for (int32_t x : most) {
    gca_window e = w;
    e.B = x;
    all(&e, 3, x > 0 ? GCA_ERR_UNSUPPORTED : GCA_ERR_INVALID);
    e = w;
    e.H = e.Hkv = x;
    all(&e, 3, x > 0 ? GCA_ERR_UNSUPPORTED : GCA_ERR_INVALID);
    e = w;
    e.capacity = x > 0 ? INT64_MAX : x;
    all(&e, 3, x > 0 ? GCA_ERR_UNSUPPORTED : GCA_ERR_INVALID);
    if (x != 0) {
      e = w;
      e.window = x;
      all(&e, 3, GCA_ERR_INVALID);
    }
  }
  // counts at the ends of their types
  all(&w, INT64_MAX, GCA_ERR_UNSUPPORTED);
  all(&w, INT64_MIN, GCA_ERR_INVALID);
  EXPECT(gca_window_attn(&w, A, I, I, F, A, F, 65, A, big, nullptr) == GCA_ERR_UNSUPPORTED);
  EXPECT(gca_window_keep(&w, I, INT64_MAX, I, 3, nullptr) == GCA_ERR_UNSUPPORTED);
  EXPECT(gca_window_keep(&w, I, INT64_MIN, I, 3, nullptr) == GCA_ERR_INVALID);
  EXPECT(gca_window_workspace_size(&w, INT64_MAX) == 0 && gca_window_workspace_size(nullptr, 1) == 0);
  EXPECT(gca_window_attn(&w, A, I, I, F, A, F, 3, nullptr, 0, nullptr) == GCA_ERR_WORKSPACE);
  const int64_t ends[] = {INT64_MAX, INT64_MIN, 0};
  for (int64_t x : ends) {
    const gca_status want = x > 0 ? GCA_ERR_UNSUPPORTED : GCA_ERR_INVALID;
    EXPECT(gca_verify(x, 5, 100, F, F, I, I, F, I, I, I, I, A, big, nullptr) == want);
    EXPECT(gca_verify(2, x, 100, F, F, I, I, F, I, I, I, I, A, big, nullptr) == want);
    EXPECT(gca_verify(2, 5, x, F, F, I, I, F, I, I, I, I, A, big, nullptr) == want);
    EXPECT(gca_verify_workspace_size(x, 5, 100) == 0);
  }
  EXPECT(gca_verify(2, 5, 100, F, F, I, I, F, I, I, I, I, A, 0, nullptr) == GCA_ERR_WORKSPACE);
  EXPECT(gca::window_launches() == 0);
  // valid calls reach their launchers, whose failure comes back
  all(&w, 3, GCA_ERR_HIP);
  EXPECT(gca_window_keep(&w, nullptr, 0, nullptr, 3, nullptr) == GCA_ERR_HIP);
  EXPECT(gca_window_attn(&w, A, I, nullptr, nullptr, A, nullptr, 64, A, big, nullptr) == GCA_ERR_HIP);
  EXPECT(gca_verify(2, 64, 1 << 19, F, nullptr, I, nullptr, F, nullptr, I, I, I, A, big, nullptr) == GCA_ERR_HIP);
  EXPECT(gca::window_launches() == 6);
  if (g_fail == 0) std::printf("OK\n");
  return g_fail != 0;
}
