// Host-side contract between the chunk cache's part of the C ABI (cache_api.cpp) and its
// kernel files.  Host C++ only.
#pragma once

#include "gca.h"
#include "gca_plan.hpp"

namespace gca {

constexpr int64_t kMaxCapacity = 262144;

// Eviction: one workgroup per sequence for up to kEvictWhole slots (106 KB of LDS; 16,384 would not fit);
// a cache of more is cut into tiles, and a second launch chooses among every tile's candidates.
// Whole / in tiles, us: one sequence of 4,096 slots, one to go 6.5 / 9.1, of 8,192 7.7 / 10.3, 1,024 to go
// 13.5 / 20.8; 64 of 8,192, 8 to go 12.9 / 14.7; 256 of 4,096 8.9 / 11.7, of 8,192 11.9 / 14.1.
constexpr int kEvictWhole = 8192;
// Of 1,024 / 2,048 / 4,096 slots, both launches: 16,384 slots, one to go 9.7 / 10.5 / 12.4; 4 sequences of
// 50,000, 40 to go 16.7 / 16.4 / 20.4, 1,024 to go 155 / 74 / 42; 262,144 slots, 64 to go 43 / 21.4 / 21.7.
// Caches of up to a tile take the smaller workgroup: 64 of 2,048 slots, 8 to go 10.8 / 9.9 / 11.3.
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
