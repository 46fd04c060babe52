// Host-side contract between the token window's part of the C ABI (window_api.cpp) and its
// kernel files.  Host C++ only.
#pragma once

#include "gca.h"
#include "gca_plan.hpp"

namespace gca {

constexpr int64_t kMaxWindowRows = int64_t(1) << 24;
constexpr int kTreeNodes = 64;  // nodes of a tree: one per lane, ancestors as 64 bits
constexpr int64_t kMaxVocab = int64_t(1) << 19;

// Tiles of 64 rows that T consecutive positions touch at most.
inline int64_t tiles_of(int64_t T) { return (T + 62) / 64 + 1; }

// Work split of the attention.
struct WindowAttnPlan {
  int rows;         // query rows per item: 16, 32 or 64
  int64_t per_head; // items per head, or 0: the rows of a group's heads are cut as one list
  int64_t blocks;   // row blocks per (sequence, cached head)
  int waves;        // per workgroup
  int splits;       // workgroups per row block
  int64_t groups;   // row blocks in all
};
WindowAttnPlan window_attn_plan(const gca_window& w, int64_t T);
size_t window_workspace(const gca_window& w, int64_t T);

struct VerifyPlan {
  int64_t slices;  // of the vocabulary, per sequence
  int64_t per;     // entries of one wave of a slice
};
VerifyPlan verify_plan(int64_t B, int64_t V);
size_t verify_workspace(int64_t B, int64_t T, int64_t V);

hipError_t launch_window_append(const gca_window& w, const void* k, const void* v, const int32_t* lengths, int64_t T,
                                hipStream_t stream);
hipError_t launch_window_attn(const gca_window& w, const void* q, const int32_t* parents, const int32_t* lengths,
                              const float* slopes, void* out, float* lse, int64_t T, void* ws, hipStream_t stream);
hipError_t launch_window_keep(const gca_window& w, const int32_t* path, int64_t n, const int32_t* lengths, int64_t T,
                              hipStream_t stream);
hipError_t launch_verify(int64_t B, int64_t T, int64_t V, const float* p, const float* q, const int32_t* tokens,
                         const int32_t* parents, const float* u, const int32_t* lengths, int32_t* path, int32_t* count,
                         int32_t* next, void* ws, hipStream_t stream);

}  // namespace gca
