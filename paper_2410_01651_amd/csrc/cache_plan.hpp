// Host-side contract between the chunk cache's part of the C ABI (cache_api.cpp) and its
// kernel files.  Host C++ only.
#pragma once

#include "gca.h"
#include "gca_plan.hpp"

namespace gca {

constexpr int64_t kMaxCapacity = 262144;

// Eviction: one workgroup per sequence for up to kEvictWhole slots; a cache of more is cut into
// tiles, and a second launch chooses among every tile's candidates.
constexpr int kEvictWhole = 8192;
constexpr int kEvictTile = 2048;
inline int64_t evict_tiles(const gca_cache& c) {
  return c.capacity <= kEvictWhole ? 1 : (c.capacity + kEvictTile - 1) / kEvictTile;
}
// Candidates per tile: enough for the tile to give all n.
inline int64_t evict_per_tile(int64_t n) { return n < kEvictTile ? n : kEvictTile; }
inline size_t evict_workspace(const gca_cache& c, int64_t n) {
  const int64_t tiles = evict_tiles(c);
  return tiles > 1 ? align256((size_t)c.B * tiles * evict_per_tile(n) * 8) : 0;
}

// The selection's problem as the decode scan takes it.
inline Shape select_shape(const gca_cache& c) {
  Shape s{};
  s.B = c.B;
  s.H = c.Hkv;
  s.Hr = c.Hr;
  s.D = c.D;
  s.topk = c.topk;
  s.nQ = 1;
  s.nKV = c.capacity;
  s.Sq = kChunk;
  s.bf16 = c.dtype == GCA_BF16;
  s.off_by_one = c.off_by_one;
  s.score_scale = c.score_scale;
  s.attn_scale = c.attn_scale;
  return s;
}

// Work items of the attention: blocks of 16, 32 or 64 query rows of a group and cached head.
int64_t xattn_items(const gca_cache& c, int64_t nQ, int64_t rows);

hipError_t launch_cache_store(const gca_cache& c, const void* k, const void* v, const void* lmk, const int32_t* slots,
                              const int32_t* lengths, int64_t n, hipStream_t stream);
hipError_t launch_cache_select(const gca_cache& c, const void* lmk_q, int32_t* idx, float* sel, float* w, void* ws,
                               hipStream_t stream);
hipError_t launch_cache_xattn(const gca_cache& c, const void* q, const int32_t* idx, const float* sel, void* out,
                              float* lse, float* w, int64_t nQ, int64_t rows, int lag, hipStream_t stream);
hipError_t launch_cache_evict(const gca_cache& c, const int32_t* idx, const float* w, int64_t nQ, float decay,
                              int keep_first, int keep_last, const int32_t* want, int32_t* slots, int64_t n, void* ws,
                              hipStream_t stream);

}  // namespace gca
