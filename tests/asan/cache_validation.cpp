// Drives the chunk cache's entry points through their checks on the host, and each once into
// a (stubbed) launch.  Prints OK and exits 0 when every status is the expected one.
#include <climits>
#include <cstdio>
#include <cstring>

#include "gca.h"

namespace gca {
int cache_launches();
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
  gca_cache c;
  std::memset(&c, 0, sizeof c);
  c.B = 2; c.H = 8; c.Hkv = 4; c.Hr = 4; c.d = 64; c.S = 64; c.capacity = 20000; c.topk = 8; c.D = 256;
  c.score_scale = 1.f; c.attn_scale = -1.f; c.dtype = GCA_FP32; c.format = GCA_INT8;
  auto all = [&](const gca_cache* p, gca_status want) {
    EXPECT(gca_cache_store(p, A, A, A, I, I, 3, nullptr) == want);
    EXPECT(gca_cache_select(p, A, I, F, F, A, big, nullptr) == want);
    EXPECT(gca_cache_xattn(p, A, I, F, A, F, F, 2, 5, 1, nullptr) == want);
    EXPECT(gca_cache_evict(p, I, F, 2, 0.5f, 1, 2, I, I, 3, A, big, nullptr) == want);
  };
  all(nullptr, GCA_ERR_INVALID);
  all(&c, GCA_ERR_INVALID);  // no members
  c.k = c.v = c.lmk = A;
  c.k_scale = c.v_scale = c.mass = F;
  c.tokens = c.number = c.next = I;
  const int32_t most[] = {0, -1, INT_MAX, INT_MIN};
  for (int32_t x : most) {
    gca_cache e = c;
    e.B = x;
    all(&e, x > 0 ? GCA_ERR_UNSUPPORTED : GCA_ERR_INVALID);
    e = c;
    e.H = e.Hkv = e.Hr = x;
    all(&e, x > 0 ? GCA_ERR_UNSUPPORTED : GCA_ERR_INVALID);
    e = c;
    e.topk = x;
    all(&e, x > 0 ? GCA_ERR_UNSUPPORTED : GCA_ERR_INVALID);
    e = c;
    e.capacity = x > 0 ? INT64_MAX : x;
    all(&e, x > 0 ? GCA_ERR_UNSUPPORTED : GCA_ERR_INVALID);
  }
  // counts at the ends of their types
  EXPECT(gca_cache_store(&c, A, A, A, I, I, INT64_MAX, nullptr) == GCA_ERR_UNSUPPORTED);
  EXPECT(gca_cache_store(&c, A, A, A, I, I, INT64_MIN, nullptr) == GCA_ERR_INVALID);
  EXPECT(gca_cache_xattn(&c, A, I, F, A, F, F, INT64_MAX, INT64_MAX, 0, nullptr) == GCA_ERR_UNSUPPORTED);
  EXPECT(gca_cache_xattn(&c, A, I, F, A, F, F, 1 << 26, 1 << 26, 0, nullptr) == GCA_ERR_UNSUPPORTED);
  EXPECT(gca_cache_evict(&c, I, F, INT64_MAX, 0.5f, 1, 2, I, I, 3, A, big, nullptr) == GCA_ERR_UNSUPPORTED);
  EXPECT(gca_cache_evict(&c, I, F, 1, 0.5f, 1, 2, I, I, INT64_MAX, A, big, nullptr) == GCA_ERR_INVALID);
  EXPECT(gca_cache_workspace_size(&c, GCA_OP_CACHE_EVICT, INT64_MAX) == 0);
  EXPECT(gca_cache_workspace_size(&c, GCA_OP_CACHE_EVICT, INT64_MIN) == 0);
  EXPECT(gca_cache_workspace_size(nullptr, GCA_OP_CACHE_SELECT, 0) == 0);
  EXPECT(gca_cache_evict(&c, I, F, 1, 0.5f, 1, 2, I, I, 3, nullptr, 0, nullptr) == GCA_ERR_WORKSPACE);
  EXPECT(gca_cache_select(&c, A, I, F, F, A, 0, nullptr) == GCA_ERR_WORKSPACE);
  EXPECT(gca::cache_launches() == 0);
  all(&c, GCA_ERR_HIP);
  EXPECT(gca::cache_launches() == 4);
  if (g_fail) {
    std::fprintf(stderr, "%d checks failed\n", g_fail);
    return 1;
  }
  std::printf("OK\n");
  return 0;
}
