// C ABI of the chunk cache: argument validation, workspace sizes and dispatch.  As in
// api.cpp nothing is launched unless every check passes.
#include <cmath>
#include <cstddef>
#include <string>

#include "cache_plan.hpp"
#include "gca_check.hpp"

using gca::check_ptr;
using gca::check_ws;
using gca::fail;
using gca::from_hip;

namespace {

// the layout the Python binding mirrors
static_assert(sizeof(gca_cache) == 136 && offsetof(gca_cache, capacity) == 24 && offsetof(gca_cache, flags) == 60 &&
                  offsetof(gca_cache, k) == 64 && offsetof(gca_cache, next) == 128,
              "gca_cache layout");

// one wave each: a launch holds below 2^32 threads, its workgroups rounded up to a multiple of 8
constexpr int64_t kMaxItems = (int64_t(1) << 26) - 8;

gca_status check_cache(const gca_cache* c) {
  if (!c) return fail(GCA_ERR_INVALID, "cache pointer is NULL");
  if (c->B < 1 || c->H < 1 || c->Hkv < 1) return fail(GCA_ERR_INVALID, "B, H and Hkv must be >= 1");
  if (c->H % c->Hkv != 0) return fail(GCA_ERR_INVALID, "H must be a multiple of Hkv");
  if (c->Hr != 1 && c->Hr != c->Hkv) return fail(GCA_ERR_INVALID, "Hr must be 1 or Hkv");
  if (c->d != 64) return fail(GCA_ERR_UNSUPPORTED, "head dimension d must be 64");
  if (c->S != 64) return fail(GCA_ERR_UNSUPPORTED, "chunk size S must be 64");
  if (c->capacity < 1) return fail(GCA_ERR_INVALID, "capacity must be >= 1");
  if (c->capacity > gca::kMaxCapacity)
    return fail(GCA_ERR_UNSUPPORTED, "capacity must be <= " + std::to_string(gca::kMaxCapacity));
  if (c->topk < 1) return fail(GCA_ERR_INVALID, "topk must be >= 1");
  if (c->topk > 32) return fail(GCA_ERR_UNSUPPORTED, "topk must be <= 32");
  if (c->D < 1) return fail(GCA_ERR_INVALID, "landmark width D must be >= 1");
  if (c->D % 64 != 0 || c->D > 8192) return fail(GCA_ERR_UNSUPPORTED, "D must be a multiple of 64, at most 8192");
  if (c->dtype != GCA_FP32 && c->dtype != GCA_BF16) return fail(GCA_ERR_INVALID, "unknown dtype");
  if (c->format != GCA_E4M3 && c->format != GCA_INT8) return fail(GCA_ERR_INVALID, "unknown format");
  if (c->off_by_one != 0 && c->off_by_one != 1) return fail(GCA_ERR_INVALID, "off_by_one must be 0 or 1");
  if (c->flags != 0) return fail(GCA_ERR_INVALID, "unknown flag bits");
  if (!std::isfinite(c->score_scale) || !std::isfinite(c->attn_scale))
    return fail(GCA_ERR_INVALID, "scales must be finite");
  if ((int64_t)c->B * c->H > kMaxItems / 256) return fail(GCA_ERR_UNSUPPORTED, "cache too large for one launch");
  return GCA_OK;
}

gca_status check_tiles(const gca_cache* c) {
  GCA_TRY(check_ptr(c->k, "cache k", true, 16));
  GCA_TRY(check_ptr(c->v, "cache v", true, 16));
  GCA_TRY(check_ptr(c->k_scale, "cache k_scale", true, 4));
  GCA_TRY(check_ptr(c->v_scale, "cache v_scale", true, 4));
  return check_ptr(c->tokens, "cache tokens", true, 4);
}

void begin() {
  (void)hipGetLastError();
  (void)gca::take_launch_error();
}

}  // namespace

extern "C" {

size_t gca_cache_workspace_size(const gca_cache* c, int op, int64_t n) {
  const std::string saved = gca_last_error();
  if (check_cache(c) != GCA_OK) {
    (void)fail(GCA_OK, saved);
    return 0;
  }
  if (op == GCA_OP_CACHE_SELECT) return gca::decode_workspace(gca::select_shape(*c));
  if (op == GCA_OP_CACHE_EVICT) return n < 1 || n > c->capacity ? 0 : gca::evict_workspace(*c, n);
  return 0;
}

gca_status gca_cache_store(const gca_cache* c, const void* k, const void* v, const void* lmk, const int32_t* slots,
                           const int32_t* lengths, int64_t n, hipStream_t stream) {
  GCA_TRY(check_cache(c));
  if (n < 1) return fail(GCA_ERR_INVALID, "n must be >= 1");
  if (n > kMaxItems / (2 * c->Hkv + c->Hr) / c->B)
    return fail(GCA_ERR_UNSUPPORTED, "too many chunks for one launch");
  GCA_TRY(check_tiles(c));
  GCA_TRY(check_ptr(k, "k", true, 16));
  GCA_TRY(check_ptr(v, "v", true, 16));
  GCA_TRY(check_ptr(lmk, "lmk", false, 16));
  GCA_TRY(check_ptr(c->lmk, "cache lmk", lmk != nullptr, 16));
  GCA_TRY(check_ptr(slots, "slots", true, 4));
  GCA_TRY(check_ptr(lengths, "lengths", false, 4));
  begin();
  return from_hip(gca::launch_cache_store(*c, k, v, lmk, slots, lengths, n, stream), "gca_cache_store");
}

gca_status gca_cache_select(const gca_cache* c, const void* lmk_q, int32_t* idx, float* sel, float* w,
                            void* workspace, size_t ws_bytes, hipStream_t stream) {
  GCA_TRY(check_cache(c));
  GCA_TRY(check_ptr(c->lmk, "cache lmk", true, 16));
  GCA_TRY(check_ptr(c->tokens, "cache tokens", true, 4));
  GCA_TRY(check_ptr(lmk_q, "lmk_q", true, 16));
  GCA_TRY(check_ptr(idx, "idx", true, 4));
  GCA_TRY(check_ptr(sel, "sel", true, 4));
  GCA_TRY(check_ptr(w, "w", false, 4));
  GCA_TRY(check_ws(workspace, ws_bytes, gca::decode_workspace(gca::select_shape(*c))));
  begin();
  return from_hip(gca::launch_cache_select(*c, lmk_q, idx, sel, w, workspace, stream), "gca_cache_select");
}

gca_status gca_cache_xattn(const gca_cache* c, const void* q, const int32_t* idx, const float* sel, void* out,
                           float* lse, float* w, int64_t nQ, int64_t rows, int32_t lag, hipStream_t stream) {
  GCA_TRY(check_cache(c));
  if (nQ < 1 || rows < 1) return fail(GCA_ERR_INVALID, "nQ and rows must be >= 1");
  if (lag != 0 && lag != 1) return fail(GCA_ERR_INVALID, "lag must be 0 or 1");
  // (bounds before products: B * H is at most 2^18)
  if (nQ > kMaxItems || rows > kMaxItems || (int64_t)c->H / c->Hkv * rows > kMaxItems ||
      gca::xattn_items(*c, 1, rows) > kMaxItems / nQ)
    return fail(GCA_ERR_UNSUPPORTED, "too many query rows for one launch");
  GCA_TRY(check_tiles(c));
  GCA_TRY(check_ptr(q, "q", true, 16));
  GCA_TRY(check_ptr(idx, "idx", true, 4));
  GCA_TRY(check_ptr(sel, "sel", true, 4));
  GCA_TRY(check_ptr(out, "out", true, 16));
  GCA_TRY(check_ptr(lse, "lse", false, 4));
  GCA_TRY(check_ptr(w, "w", false, 4));
  begin();
  return from_hip(gca::launch_cache_xattn(*c, q, idx, sel, out, lse, w, nQ, rows, lag, stream), "gca_cache_xattn");
}

gca_status gca_cache_evict(const gca_cache* c, const int32_t* idx, const float* w, int64_t nQ, float decay,
                           int32_t keep_first, int32_t keep_last, const int32_t* want, int32_t* slots, int64_t n,
                           void* workspace, size_t ws_bytes, hipStream_t stream) {
  GCA_TRY(check_cache(c));
  if (n < 0 || n > c->capacity) return fail(GCA_ERR_INVALID, "n must be 0 .. capacity");
  if (!(decay >= 0.f && decay <= 1.f)) return fail(GCA_ERR_INVALID, "decay must be 0 .. 1");
  if (keep_first < 0 || keep_last < 0) return fail(GCA_ERR_INVALID, "keep_first and keep_last must be >= 0");
  if ((idx == nullptr) != (w == nullptr)) return fail(GCA_ERR_INVALID, "idx and w are given together");
  if (idx && nQ < 1) return fail(GCA_ERR_INVALID, "nQ must be >= 1");
  if (idx && nQ > 0x7fffffff / ((int64_t)c->Hr * c->topk))
    return fail(GCA_ERR_UNSUPPORTED, "too many lists for one call");
  GCA_TRY(check_ptr(c->tokens, "cache tokens", true, 4));
  GCA_TRY(check_ptr(c->mass, "cache mass", true, 4));
  GCA_TRY(check_ptr(c->number, "cache number", true, 4));
  GCA_TRY(check_ptr(c->next, "cache next", true, 4));
  GCA_TRY(check_ptr(idx, "idx", false, 4));
  GCA_TRY(check_ptr(w, "w", false, 4));
  GCA_TRY(check_ptr(want, "want", false, 4));
  GCA_TRY(check_ptr(slots, "slots", n > 0, 4));
  GCA_TRY(check_ws(workspace, ws_bytes, n > 0 ? gca::evict_workspace(*c, n) : 0));
  begin();
  return from_hip(gca::launch_cache_evict(*c, idx, w, nQ, decay, keep_first, keep_last, want, slots, n, workspace,
                                          stream),
                  "gca_cache_evict");
}

}  // extern "C"
