// C ABI of the token window and of the verification of drafts: argument validation, workspace sizes and
// dispatch.  As in api.cpp nothing is launched unless every check passes.
#include <cmath>
#include <cstddef>
#include <string>

#include "gca_check.hpp"
#include "window_plan.hpp"

using gca::check_ptr;
using gca::check_ws;
using gca::fail;
using gca::from_hip;

namespace {

// the layout the Python binding mirrors
static_assert(sizeof(gca_window) == 96 && offsetof(gca_window, capacity) == 16 && offsetof(gca_window, flags) == 44 &&
                  offsetof(gca_window, k) == 48 && offsetof(gca_window, ticket) == 88,
              "gca_window layout");

// a launch holds below 2^32 threads, its workgroups (up to 512 threads) rounded up to a multiple of 8
constexpr int64_t kMaxItems = (int64_t(1) << 23) - 8;

gca_status check_window(const gca_window* w) {
  if (!w) return fail(GCA_ERR_INVALID, "window pointer is NULL");
  if (w->B < 1 || w->H < 1 || w->Hkv < 1) return fail(GCA_ERR_INVALID, "B, H and Hkv must be >= 1");
  if (w->H % w->Hkv != 0) return fail(GCA_ERR_INVALID, "H must be a multiple of Hkv");
  if (w->d != 64) return fail(GCA_ERR_UNSUPPORTED, "head dimension d must be 64");
  if (w->capacity < 1) return fail(GCA_ERR_INVALID, "capacity must be >= 1");
  if (w->capacity % 64 != 0 || w->capacity > gca::kMaxWindowRows)
    return fail(GCA_ERR_UNSUPPORTED, "capacity must be a multiple of 64, at most " + std::to_string(gca::kMaxWindowRows));
  if (w->window < 0 || w->window > w->capacity) return fail(GCA_ERR_INVALID, "window must be 0 .. capacity");
  if (w->dtype != GCA_FP32 && w->dtype != GCA_BF16) return fail(GCA_ERR_INVALID, "unknown dtype");
  if (w->format != GCA_E4M3 && w->format != GCA_INT8) return fail(GCA_ERR_INVALID, "unknown format");
  if (w->off_by_one != 0 && w->off_by_one != 1) return fail(GCA_ERR_INVALID, "off_by_one must be 0 or 1");
  if (w->flags != 0) return fail(GCA_ERR_INVALID, "unknown flag bits");
  if (!std::isfinite(w->attn_scale)) return fail(GCA_ERR_INVALID, "scales must be finite");
  // (biases are taken in units of a score before its scale)
  if (w->attn_scale != 0.f && std::fabs(w->attn_scale) < 0x1p-64f)
    return fail(GCA_ERR_UNSUPPORTED, "attn_scale must be 0 or at least 2^-64");
  if ((int64_t)w->B * w->H > kMaxItems / 16) return fail(GCA_ERR_UNSUPPORTED, "window too large for one launch");
  return GCA_OK;
}

gca_status check_rows(const gca_window* w) {
  GCA_TRY(check_ptr(w->k, "window k", true, 16));
  GCA_TRY(check_ptr(w->v, "window v", true, 16));
  GCA_TRY(check_ptr(w->k_scale, "window k_scale", true, 4));
  GCA_TRY(check_ptr(w->v_scale, "window v_scale", true, 4));
  GCA_TRY(check_ptr(w->length, "window length", true, 4));
  return check_ptr(w->ticket, "window ticket", true, 4);
}

// T new tokens of every sequence (bounds before products: B * H is below 2^19).
gca_status check_tokens(const gca_window* w, int64_t T) {
  if (T < 1) return fail(GCA_ERR_INVALID, "T must be >= 1");
  if (T > 0x40000000 || T > kMaxItems / ((int64_t)w->B * w->H) * 16)
    return fail(GCA_ERR_UNSUPPORTED, "too many tokens for one launch");
  return GCA_OK;
}

gca_status check_draft_sizes(int64_t B, int64_t T, int64_t V) {
  if (B < 1 || T < 1 || V < 1) return fail(GCA_ERR_INVALID, "B, T and V must be >= 1");
  if (T > gca::kTreeNodes) return fail(GCA_ERR_UNSUPPORTED, "T must be <= 64");
  if (V > gca::kMaxVocab) return fail(GCA_ERR_UNSUPPORTED, "V must be <= " + std::to_string(gca::kMaxVocab));
  if (B > kMaxItems / 256) return fail(GCA_ERR_UNSUPPORTED, "too many sequences for one launch");
  return GCA_OK;
}

void begin() {
  (void)hipGetLastError();
  (void)gca::take_launch_error();
}

}  // namespace

extern "C" {

size_t gca_window_workspace_size(const gca_window* w, int64_t T) {
  const std::string saved = gca_last_error();
  const bool ok = check_window(w) == GCA_OK && check_tokens(w, T) == GCA_OK;
  if (ok) return gca::window_workspace(*w, T);
  (void)fail(GCA_OK, saved);
  return 0;
}

size_t gca_verify_workspace_size(int64_t B, int64_t T, int64_t V) {
  const std::string saved = gca_last_error();
  if (check_draft_sizes(B, T, V) == GCA_OK) return gca::verify_workspace(B, T, V);
  (void)fail(GCA_OK, saved);
  return 0;
}

gca_status gca_window_append(const gca_window* w, const void* k, const void* v, const int32_t* lengths, int64_t T,
                             hipStream_t stream) {
  GCA_TRY(check_window(w));
  GCA_TRY(check_tokens(w, T));
  GCA_TRY(check_rows(w));
  GCA_TRY(check_ptr(k, "k", true, 16));
  GCA_TRY(check_ptr(v, "v", true, 16));
  GCA_TRY(check_ptr(lengths, "lengths", false, 4));
  begin();
  return from_hip(gca::launch_window_append(*w, k, v, lengths, T, stream), "gca_window_append");
}

gca_status gca_window_attn(const gca_window* w, const void* q, const int32_t* parents, const int32_t* lengths,
                           const float* slopes, void* out, float* lse, int64_t T, void* workspace, size_t ws_bytes,
                           hipStream_t stream) {
  GCA_TRY(check_window(w));
  GCA_TRY(check_tokens(w, T));
  if (parents && T > gca::kTreeNodes) return fail(GCA_ERR_UNSUPPORTED, "a tree has at most 64 nodes");
  if (w->window > 0 && w->window + T - 1 > w->capacity)
    return fail(GCA_ERR_INVALID, "window + T - 1 must be <= capacity");
  GCA_TRY(check_rows(w));
  GCA_TRY(check_ptr(q, "q", true, 16));
  GCA_TRY(check_ptr(parents, "parents", false, 4));
  GCA_TRY(check_ptr(lengths, "lengths", false, 4));
  GCA_TRY(check_ptr(slopes, "slopes", false, 4));
  GCA_TRY(check_ptr(out, "out", true, 16));
  GCA_TRY(check_ptr(lse, "lse", false, 4));
  GCA_TRY(check_ws(workspace, ws_bytes, gca::window_workspace(*w, T)));
  begin();
  return from_hip(gca::launch_window_attn(*w, q, parents, lengths, slopes, out, lse, T, workspace, stream),
                  "gca_window_attn");
}

gca_status gca_window_keep(const gca_window* w, const int32_t* path, int64_t n, const int32_t* lengths, int64_t T,
                           hipStream_t stream) {
  GCA_TRY(check_window(w));
  GCA_TRY(check_tokens(w, T));
  if (n < 0) return fail(GCA_ERR_INVALID, "n must be >= 0");
  if (n > gca::kTreeNodes) return fail(GCA_ERR_UNSUPPORTED, "a path has at most 64 entries");
  // (a dropped token's row was another's, which a row behind what is kept may see)
  if (w->window > 0 && w->window + T - 1 > w->capacity)
    return fail(GCA_ERR_INVALID, "window + T - 1 must be <= capacity");
  GCA_TRY(check_rows(w));
  GCA_TRY(check_ptr(path, "path", n > 0, 4));
  GCA_TRY(check_ptr(lengths, "lengths", false, 4));
  begin();
  return from_hip(gca::launch_window_keep(*w, path, n, lengths, T, stream), "gca_window_keep");
}

gca_status gca_verify(int64_t B, int64_t T, int64_t V, const float* p, const float* q, const int32_t* tokens,
                      const int32_t* parents, const float* u, const int32_t* lengths, int32_t* path, int32_t* count,
                      int32_t* next, void* workspace, size_t ws_bytes, hipStream_t stream) {
  GCA_TRY(check_draft_sizes(B, T, V));
  GCA_TRY(check_ptr(p, "p", true, 4));
  GCA_TRY(check_ptr(q, "q", false, 4));
  GCA_TRY(check_ptr(tokens, "tokens", true, 4));
  GCA_TRY(check_ptr(parents, "parents", false, 4));
  GCA_TRY(check_ptr(u, "u", true, 4));
  GCA_TRY(check_ptr(lengths, "lengths", false, 4));
  GCA_TRY(check_ptr(path, "path", true, 4));
  GCA_TRY(check_ptr(count, "count", true, 4));
  GCA_TRY(check_ptr(next, "next", true, 4));
  GCA_TRY(check_ws(workspace, ws_bytes, gca::verify_workspace(B, T, V)));
  begin();
  return from_hip(gca::launch_verify(B, T, V, p, q, tokens, parents, u, lengths, path, count, next, workspace, stream),
                  "gca_verify");
}

}  // extern "C"
