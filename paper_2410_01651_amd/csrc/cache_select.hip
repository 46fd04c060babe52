// Retrieval among the chunks in use of a cache (gca_cache_select): the decode scan over the
// landmark keys with the free slots left out (decode_scan.hpp, MASK), then one workgroup per
// retrieval row merges the scan's lists into the row's best k and writes them ascending by
// slot with their fusion weights.  The scan is bound by reading the landmarks once, the merge
// by its chain of dependent steps.  Small caches take one launch (cache_select_few_kernel).
// 262,144 slots of width 512 bf16 43.6 us (6.1 TB/s) + 6.2, 32 sequences of 1,000 slots of width
// 1,024 14.7 + 3.9, one sequence of 128 slots 5.8.
//
// The merge's waves each take a share of the lists and keep their best 64 candidates as one
// sorted 64-bit key per lane.  Candidates that beat the k-th are gathered in LDS until there are
// 64, sorted and merged in (27 compare-exchange steps).  First come the lists' heads; an entry of
// the row's k best can only sit in a list whose head is among its share's k best, and as a list is
// sorted, its next entries are read only while one before them was kept.
#include <algorithm>

#include "cache_plan.hpp"
#include "decode_scan.hpp"

namespace gca {
namespace {

constexpr int kMergeThreads = 512;
constexpr int kMergeWaves = kMergeThreads / 64;
constexpr int kFewSlots = 256;
constexpr int64_t kFewBytes = 768 << 10;  // of a row's landmarks

// One step of a bitonic merge, largest first: lane l against l ^ J.
template <int J>
__device__ __forceinline__ uint64_t merge_step(uint64_t k) {
  uint32_t a0, a1, b0, b1;
  const uint32_t lo = (uint32_t)k, hi = (uint32_t)(k >> 32);
  if constexpr (J == 32) {
    pair32(lo, a0, b0);
    pair32(hi, a1, b1);
  } else if constexpr (J == 16) {
    pair16(lo, a0, b0);
    pair16(hi, a1, b1);
  } else {
    a0 = lo;
    a1 = hi;
    b0 = J == 8 ? dpp<kDppRor8>(lo) : J == 4 ? swz_xor4(lo) : J == 2 ? dpp<kDppXor2>(lo) : dpp<kDppXor1>(lo);
    b1 = J == 8 ? dpp<kDppRor8>(hi) : J == 4 ? swz_xor4(hi) : J == 2 ? dpp<kDppXor2>(hi) : dpp<kDppXor1>(hi);
  }
  const uint64_t a = (uint64_t)a0 | ((uint64_t)a1 << 32), b = (uint64_t)b0 | ((uint64_t)b1 << 32);
  return ((a > b) == ((threadIdx.x & J) == 0)) ? a : b;
}

// A wave's best 64 candidates so far (lane r: the r-th; 0: none) and those waiting to join.
struct Best {
  uint64_t key = 0;
  uint64_t bar = 0;   // the k-th best: only better ones join
  uint32_t held = 0;
  uint64_t* buf;      // 128 of this wave's own
  int K;

  __device__ __forceinline__ Best(uint64_t* b, int k) : buf(b), K(k) {}
  // the candidates are the lanes' (0: none)
  __device__ __forceinline__ void start(uint64_t x) {
    key = wave_sort_desc(x);
    bar = __shfl(key, K - 1);
  }
  // up to 64 waiting candidates join
  __device__ __forceinline__ void flush() {
    const int lane = threadIdx.x & 63;
    wave_lds_order();
    const uint64_t x = lane < (int)held ? buf[lane] : 0;
    const uint64_t rest = buf[64 + lane];
    wave_lds_order();
    buf[lane] = rest;
    held = held > 64 ? held - 64 : 0;
    // descending against ascending: the larger of each pair are the 64 best, in bitonic order
    const uint64_t up = ~wave_sort_desc(~x);
    key = key > up ? key : up;
    key = merge_step<1>(merge_step<2>(merge_step<4>(merge_step<8>(merge_step<16>(merge_step<32>(key))))));
    bar = __shfl(key, K - 1);
  }
  // every lane offers a candidate (0: none)
  __device__ __forceinline__ void offer(uint64_t x) {
    const bool in = x > bar;
    const uint64_t mask = __ballot(in);
    if (in) buf[held + lanes_below(mask)] = x;
    held += __popcll(mask);
    if (held >= 64) flush();
  }
  __device__ __forceinline__ void settle() {
    while (held) flush();
  }
};

// A row's best candidates (lane r: the r-th, 0: none) ascending by slot, with their fusion weights.
__device__ __forceinline__ void write_list(uint64_t best, int K, int64_t row, int32_t* __restrict__ idx,
                                           float* __restrict__ sel, float* __restrict__ w) {
  const int lane = threadIdx.x & 63;
  const uint64_t key = lane < K ? best : 0;
  const bool valid = key != 0;
  const int cnt = __popcll(__ballot(valid));
  const int mj = valid ? key_chunk(key) : kNoChunk;
  const float ms = valid ? key_score(key) : -INFINITY;
  const int rank = rank_by_chunk(mj, cnt);
  // best first: lane 0 holds the maximum; the valid lanes sit in the lower half
  const float mx = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(ms)));
  const float e = valid ? expf(ms - mx) : 0.f;
  const float sum = sum32(e);
  if (lane < K) {
    const int64_t at = row * K + (valid ? rank : lane);
    idx[at] = valid ? mj : -1;
    sel[at] = ms;
    if (w) w[at] = valid ? e / sum : 0.f;
  }
}

__global__ __launch_bounds__(kMergeThreads) void cache_merge_kernel(const float* __restrict__ ls,
                                                                    const int* __restrict__ lj, int64_t lists,
                                                                    int64_t pw, int K, int32_t* __restrict__ idx,
                                                                    float* __restrict__ sel, float* __restrict__ w) {
  __shared__ uint64_t buf[kMergeWaves][128];
  __shared__ uint64_t result[kMergeWaves][32];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = blockIdx.x;
  const int* score_bits = reinterpret_cast<const int*>(ls) + row * lists * K;
  const int* rj = lj + row * lists * K;
  const int64_t share = (lists + kMergeWaves - 1) / kMergeWaves;
  const int64_t l_lo = wave * share, l_hi = l_lo + share < lists ? l_lo + share : lists;
  // entry `at` of the row, 0 if not wanted.  The loads are made on every path and all before the
  // first use (the empty asm): one that a branch guards is waited for before the next.
  auto ask = [&](bool wanted, int64_t at, int& v, int& j) {
    at = wanted ? at : 0;
    v = score_bits[at];
    j = rj[at];
  };
  auto got = [&](bool wanted, int v, int j) { return wanted && j >= 0 ? pack_key(__int_as_float(v), j) : 0; };
  auto entry = [&](bool wanted, int64_t at) -> uint64_t {
    int v, j;
    ask(wanted, at, v, j);
    asm volatile("" : "+v"(v), "+v"(j));
    return got(wanted, v, j);
  };
  Best best(buf[wave], K);
  if (share * K <= 64) {
    // an entry per lane
    const int l = lane / K;
    best.start(entry(l_lo + l < l_hi && l < share, l_lo * K + lane));
  } else {
    if (share <= 64) {
      best.start(entry(l_lo + lane < l_hi, (l_lo + lane) * K));
    } else {
      for (int64_t l0 = l_lo; l0 < l_hi; l0 += 64) best.offer(entry(l0 + lane < l_hi, (l0 + lane) * K));
      best.settle();
    }
    // lane s < K: the list that the s-th best head heads
    const uint64_t head = lane < K ? best.key : 0;
    const int list = head != 0 ? (int)scan_list_of(key_chunk(head), pw) : -1;
    if (K * K <= 64) {
      const int l = __shfl(list, lane / K);
      best.start(entry(lane < K * K && l >= 0, (int64_t)l * K + lane % K));
    } else {
      bool more = list >= 0;
      for (int r = 1; r < K; r += 4) {
        int v[4], j[4];
        uint64_t x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) ask(more && r + u < K, (int64_t)list * K + r + u, v[u], j[u]);
        asm volatile(""
                     : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]), "+v"(j[0]), "+v"(j[1]), "+v"(j[2]), "+v"(j[3]));
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          x[u] = got(more && r + u < K, v[u], j[u]);
          best.offer(x[u]);
        }
        more = more && x[3] > best.bar;  // (else nothing behind it can join)
        if (__ballot(more) == 0) break;
      }
      best.settle();
    }
  }
  if (lane < K) result[wave][lane] = best.key;
  __syncthreads();
  if (wave != 0) return;
  if (kMergeWaves * K <= 64) {
    best.start(lane < kMergeWaves * K ? result[lane / K][lane % K] : 0);
  } else {
    for (int y = 1; y < kMergeWaves; ++y) best.offer(lane < K ? result[y][lane] : 0);
    best.settle();
  }

  write_list(best.key, K, row, idx, sel, w);
}

// Small caches (few_slots): one workgroup per retrieval row, a wave for 8 slots at a time, their landmarks'
// rows all in flight, and the row's list from the scores in LDS: one launch.
template <typename T>
__global__ __launch_bounds__(1024) void cache_select_few_kernel(const T* __restrict__ lmk_q, const T* __restrict__ lmk,
                                                                const int32_t* __restrict__ tokens, int Hr, int C,
                                                                int D, int K, float scale, int32_t* __restrict__ idx,
                                                                float* __restrict__ sel, float* __restrict__ w) {
  constexpr int E = 16 / sizeof(T);
  __shared__ uint64_t keys[kFewSlots];
  __shared__ uint64_t buf[128];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = blockIdx.x;
  const T* q = lmk_q + row * D;
  const T* k = lmk + row * C * D;
  for (int first = wave * 8; first < C; first += (int)(blockDim.x >> 6) * 8) {
    const int slot = first + (lane & 7);
    const int used = tokens[row / Hr * C + min(slot, C - 1)];
    float acc[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) acc[u] = 0.f;
    for (int d0 = 0; d0 < D; d0 += 64 * E) {
      // (lanes behind the row's end take its start, times zero: what is not finite there is not finite either way)
      const bool in = d0 + lane * E < D;
      const int d = in ? d0 + lane * E : 0;
      u32x4 x = *reinterpret_cast<const u32x4*>(q + d), y[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        y[u] = *reinterpret_cast<const u32x4*>(k + (int64_t)min(first + u, C - 1) * D + d);
      if (!in) x = u32x4{0, 0, 0, 0};
      auto at = [](const u32x4& v, int e) {
        if constexpr (E == 4) return __uint_as_float(v[e]);
        else return __uint_as_float((e & 1) ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16);
      };
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[u] = fmaf(at(x, e), at(y[u], e), acc[u]);
    }
    float score = 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float f = sum64(acc[u]);
      score = (lane & 7) == u ? f : score;
    }
    score *= scale;
    if (lane < 8 && slot < C) keys[slot] = used > 0 && __builtin_isfinite(score) ? pack_key(score, slot) : 0;
  }
  __syncthreads();
  if (wave != 0) return;
  Best best(buf, K);
  best.start(lane < C ? keys[lane] : 0);
  for (int s0 = 64; s0 < C; s0 += 64) best.offer(s0 + lane < C ? keys[s0 + lane] : 0);
  best.settle();
  write_list(best.key, K, row, idx, sel, w);
}

// A workgroup reads a row's landmarks alone, which pays while that takes less than the scan's and the merge's
// start: one launch / scan and merge, us, bf16: 1 row, 128 slots of width 1,024 5.8 / 10.2, 256 8.8 / 10.5,
// 384 11.6 / 10.6, 256 of 2,048 12.7 / 12.9; 256 rows, 128 of 1,024 13.6 / 18.6, 256 22.2 / 28.0, 512 43.4 /
// 47.8, of 2,048 91.9 / 84.6; 2,048 rows, 64 of 1,024 40.6 / 52.8.
bool few_slots(const gca_cache& c) {
  return c.capacity <= kFewSlots && c.capacity * c.D * (c.dtype == GCA_BF16 ? 2 : 4) <= kFewBytes;
}

}  // namespace

hipError_t launch_cache_select(const gca_cache& c, const void* lmk_q, int32_t* idx, float* sel, float* w, void* ws,
                               hipStream_t stream) {
  const Shape s = select_shape(c);
  if (few_slots(c)) {
    const dim3 grid((unsigned)((int64_t)s.B * s.Hr)), block((unsigned)std::min<int64_t>(1024, (c.capacity + 7) / 8 * 64));
    auto run = [&](auto tag) {
      using T = decltype(tag);
      launch_kernel("cache_select_few_kernel", cache_select_few_kernel<T>, grid, block, 0, stream,
                    static_cast<const T*>(lmk_q), static_cast<const T*>(c.lmk), c.tokens, s.Hr, (int)c.capacity, s.D,
                    s.topk, s.score_scale, idx, sel, w);
    };
    if (s.bf16) run(__bf16{});
    else run(float{});
    return take_launch_error();
  }
  const hipError_t e = s.bf16 ? launch_scan<__bf16, false, true>(s, lmk_q, c.lmk, c.tokens, ws, stream)
                              : launch_scan<float, false, true>(s, lmk_q, c.lmk, c.tokens, ws, stream);
  if (e != hipSuccess) return e;
  const DecodePlan plan = decode_plan(s);
  launch_kernel("cache_merge_kernel", cache_merge_kernel, dim3((unsigned)((int64_t)s.B * s.Hr)), dim3(kMergeThreads), 0,
                stream, decode_list_scores(s, ws), decode_list_chunks(s, ws), plan.lists, plan.pw, s.topk, idx, sel, w);
  return take_launch_error();
}

}  // namespace gca
