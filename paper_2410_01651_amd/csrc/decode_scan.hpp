// The decode scan (Eq. 1 for one landmark query per retrieval row), included by the files
// that launch it: over a past of equal length for every sequence (scores.hip) and over the
// chunks in use of a cache (cache_select.hip).
#pragma once

#include "gca_device.hpp"
#include "gca_launch.hpp"

namespace gca {
namespace {

constexpr int kScanThreads = 256;
constexpr int kScanWaves = kScanThreads / 64;
static_assert(kScanWaves == kScanListWaves, "the merge's list mapping assumes four scan waves");
constexpr int kScanBatch = 8;  // column blocks per lane in one batch of loads

constexpr int kLoadNonTemporal = 2;  // cache policy: streamed once

// Partial dot product of one lane's 8 elements of a key column block with the
// query's (both 16 bytes of bf16, or 32 bytes of fp32 as two records).
__device__ __forceinline__ float dot_block(const u32x4* v, const bf16x8 b, float acc) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  const bf16x8 a = __builtin_bit_cast(bf16x8, v[0]);
  acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(a, a, 0, 1), __builtin_shufflevector(b, b, 0, 1),
                                        acc, false);
  acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(a, a, 2, 3), __builtin_shufflevector(b, b, 2, 3),
                                        acc, false);
  acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(a, a, 4, 5), __builtin_shufflevector(b, b, 4, 5),
                                        acc, false);
  acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(a, a, 6, 7), __builtin_shufflevector(b, b, 6, 7),
                                        acc, false);
  return acc;
}
__device__ __forceinline__ float dot_block(const u32x4* v, const f32x8 b, float acc) {
  const f32x4 a0 = __builtin_bit_cast(f32x4, v[0]), a1 = __builtin_bit_cast(f32x4, v[1]);
#pragma unroll
  for (int m = 0; m < 4; ++m) acc = fmaf(a0[m], b.lo[m], acc);
#pragma unroll
  for (int m = 0; m < 4; ++m) acc = fmaf(a1[m], b.hi[m], acc);
  return acc;
}

// Every workgroup scans one contiguous range of 4 pw landmark keys of its row:
// its four waves take the range's groups of 8 keys in turn (wave w: groups w,
// w + 4, ...), so the workgroup reads one stream (one stream per wave, 1,024 in
// all, measured 6-7 % slower), and each wave leaves the best k of its groups
// (sorted best first, padded with chunk -1) as list number (workgroup * 4 +
// wave) of the row.  8 lanes share a key: lane
// 8m + s reads bytes 16 s .. 16 s + 15 (bf16) of every 128-byte column block of
// key m of the current group of 8 keys, so one load instruction covers 8 keys x
// 128 contiguous bytes.  Loads are streamed (non-temporal) through a buffer
// descriptor per key group, whose range check zeroes the lanes past the end of
// the wave's range with no memory access, and run one batch of 8 column blocks
// ahead of the arithmetic.  The plan spreads any number of keys over about one
// workgroup per CU, down to one key group per wave where that pays (scan_floor): bound
// by the key stream for long pasts, by a few round trips for short ones.  16,384 keys of
// width 768: 18.4 -> 7.8 us against ranges of at least 64 keys per wave (64 workgroups);
// 32 rows of 1,000 keys of width 1,024: 22.6 -> 14.4 us.  The lists this adds (up to
// 1,024 per row) cost the merge 0.5 us at k = 8.
// GUMBEL: the lists rank (and hold) score + Gumbel noise; the decode attention
// recomputes the chosen chunks' raw scores.  Q8 (D = 512, eight column blocks
// per key): every lane keeps its eight query fragments in registers, so there
// is no staging of the query through LDS and no barrier before the first loads,
// and a batch of loads is exactly one key group.
// MASK: only chunks with tokens[b, chunk] > 0 are candidates (b: the row's sequence).  The
// workgroup first turns its range's lengths into a bit mask in LDS and ends its range behind
// the last chunk in use, so the free end of a cache that is not full is not read.
template <typename T, int KM, bool KEEP_ALL, bool GUMBEL, bool Q8, bool MASK>
__global__ __launch_bounds__(kScanThreads) void decode_scan_kernel(const T* __restrict__ lq,
                                                                   const T* __restrict__ lk, float* __restrict__ cs,
                                                                   int* __restrict__ cj, int64_t nC, int D,
                                                                   float scale, int K, int64_t pw, int64_t lists,
                                                                   int64_t wgs, uint64_t seed,
                                                                   const int32_t* __restrict__ tokens, int Hr) {
  constexpr int LPS = (int)sizeof(T) / 2;  // 16-byte records per lane per column block
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  T* sq = reinterpret_cast<T*>(smem);

  const int64_t row = blockIdx.x / wgs, g = blockIdx.x % wgs;
  const int tid = threadIdx.x, lane = tid & 63, sub = lane & 7, kl = lane >> 3;
  const T* q = lq + row * D;  // the one landmark query of this row
  Frag<T> qreg[Q8 ? kScanBatch : 1];
  if constexpr (Q8) {
#pragma unroll
    for (int k = 0; k < kScanBatch; ++k) qreg[k] = load_frag(q + 64 * k + sub * 8);
  }
  // (otherwise the query is read here and staged in LDS after the first keys have
  // been asked for, so that its round trip is not ahead of theirs)
  constexpr int kQVec = 16 / (int)sizeof(T);
  u32x4 qv = u32x4{0, 0, 0, 0};
  if (!Q8 && tid * kQVec < D) qv = *reinterpret_cast<const u32x4*>(q + tid * kQVec);

  const int wv = tid >> 6;
  const int64_t list = uniform64(g * kScanWaves + wv);  // < lists = wgs * kScanWaves
  // the workgroup's contiguous range of keys; this wave takes its key groups
  // wv, wv + 4, wv + 8, ... (group = 8 consecutive keys)
  const int64_t lo = g * kScanWaves * pw;
  int64_t n = kScanWaves * pw < nC - lo ? kScanWaves * pw : nC - lo;  // keys in the range (>= 1)
  const uint64_t* used = nullptr;  // bit x: key x of the range may be retrieved
  if constexpr (MASK) {
    uint64_t* bits = reinterpret_cast<uint64_t*>(smem + (Q8 ? 0 : D * sizeof(T)));
    __shared__ int end;
    if (tid == 0) end = 0;
    __syncthreads();
    const int32_t* tk = tokens + (row / Hr) * nC + lo;
    int last = 0;
    for (int64_t x = tid; x - tid < n; x += kScanThreads) {
      const uint64_t m = __ballot(x < n && tk[x < n ? x : 0] > 0);
      if (lane == 0) bits[x >> 6] = m;
      if (m != 0) last = (int)((x >> 6) << 6) + 64 - __builtin_clzll(m);
    }
    if (lane == 0) atomicMax(&end, last);
    __syncthreads();
    n = __builtin_amdgcn_readfirstlane(end);
    used = bits;
  }
  auto in_use = [&](int64_t key) { return !MASK || ((used[key >> 6] >> (key & 63)) & 1) != 0; };
  const int NB = D / 64;                          // column blocks per key
  const int64_t KB = (int64_t)D * sizeof(T);      // bytes per key
  const int64_t ngroups_wg = (n + 7) / 8;
  const int64_t ngroups = ngroups_wg > wv ? (ngroups_wg - wv + kScanWaves - 1) / kScanWaves : 0;
  auto key_of = [&](int64_t gi, int kk) { return 8 * (wv + kScanWaves * gi) + kk; };  // key of the range
  const int64_t nsteps = ngroups * NB;
  const int64_t nbatch = (nsteps + kScanBatch - 1) / kScanBatch;
  const char* const wbase = reinterpret_cast<const char*>(lk + (row * nC + lo) * D);
  const uint32_t lane_off = (uint32_t)(kl * KB) + (uint32_t)(sub * 16 * LPS);

  // issue cursor: key group ig, column block icb, and the group's descriptor
  int64_t ig = 0;
  int icb = 0;
  auto rsrc_of = [&](int64_t gi) {  // this wave's gi-th group
    const int64_t gg = wv + kScanWaves * gi;
    const int64_t left = (n - 8 * gg) * KB;
    const uint32_t bytes = left <= 0 ? 0u : (uint32_t)(left < 8 * KB ? left : 8 * KB);
    return range_rsrc(wbase + (left <= 0 ? 0 : gg * 8 * KB), bytes);
  };
  __amdgpu_buffer_rsrc_t rs = rsrc_of(0);
  auto issue = [&](u32x4* v) {
#pragma unroll
    for (int k = 0; k < kScanBatch; ++k) {
#pragma unroll
      for (int e = 0; e < LPS; ++e)
        v[k * LPS + e] = __builtin_amdgcn_raw_buffer_load_b128(rs, lane_off + 16 * e,
                                                               icb * 64 * (int)sizeof(T), kLoadNonTemporal);
      if (++icb == NB) {
        icb = 0;
        ++ig;
        rs = rsrc_of(ig);
      }
    }
  };

  // compute cursor
  int64_t cg = 0;
  int ccb = 0;
  float acc = 0.f;
  TopList<KM> L;
  L.init();
  // KEEP_ALL (a lane sees at most KM keys): lane (kl, sub) keeps the raw score
  // of key kl of the wave's group 8 m + sub in sc[m], ranked only at the end
  float sc[KEEP_ALL ? KM : 1];
  float mine = -INFINITY;
  if constexpr (KEEP_ALL) {
#pragma unroll
    for (int m = 0; m < KM; ++m) sc[m] = -INFINITY;
  }
  // the dot products of key group cg are complete in acc
  auto finish_group = [&]() {
    // sum over the key's 8 lanes (quad swaps, then the other quad)
    acc += dpp<kDppXor1>(acc);
    acc += dpp<kDppXor2>(acc);
    acc += dpp<kDppHalfMirror>(acc);
    if constexpr (KEEP_ALL) {
      if (sub == (int)(cg & 7)) mine = acc;
      if ((cg & 7) == 7 || cg + 1 == ngroups) {
#pragma unroll
        for (int m = 0; m < KM; ++m)
          if (m == (int)(cg >> 3)) sc[m] = mine;
        mine = -INFINITY;
      }
    } else {
      const int64_t key = key_of(cg, kl);
      // one of the key's 8 lanes inserts it, rotating with the group
      if (key < n && sub == (int)(cg & 7) && in_use(key)) {
        float sv = acc * scale;
        if constexpr (GUMBEL) sv += gumbel_noise(seed, (uint32_t)row, 0u, (uint32_t)(lo + key));
        if (__builtin_isfinite(sv)) L.insert(sv, (int)(lo + key));
      }
    }
    acc = 0.f;
    ++cg;
  };
  auto consume = [&](const u32x4* v, int64_t step0) {
    if constexpr (Q8) {
      if (step0 < nsteps) {  // one whole group
#pragma unroll
        for (int k = 0; k < kScanBatch; ++k) acc = dot_block(v + k * LPS, qreg[k], acc);
        finish_group();
      }
    } else {
#pragma unroll
      for (int k = 0; k < kScanBatch; ++k) {
        if (step0 + k < nsteps) {
          acc = dot_block(v + k * LPS, load_frag(sq + ccb * 64 + sub * 8), acc);
          if (++ccb == NB) {
            ccb = 0;
            finish_group();
          }
        }
      }
    }
  };

  // two register batches alternate: batch b + 1 is in flight while batch b is
  // consumed; the loop body issues unconditionally so the waits stay exact
  u32x4 va[kScanBatch * LPS], vb[kScanBatch * LPS];
  issue(va);
  if constexpr (!Q8) {
    if (tid * kQVec < D) *reinterpret_cast<u32x4*>(sq + tid * kQVec) = qv;
    for (int x = (tid + kScanThreads) * kQVec; x < D; x += kScanThreads * kQVec)
      *reinterpret_cast<u32x4*>(sq + x) = *reinterpret_cast<const u32x4*>(q + x);
    __syncthreads();
  }
  int64_t bt = 0;
  for (; bt + 2 < nbatch; bt += 2) {
    issue(vb);
    consume(va, bt * kScanBatch);
    issue(va);
    consume(vb, (bt + 1) * kScanBatch);
  }
  if (bt + 1 < nbatch) {
    issue(vb);
    consume(va, bt * kScanBatch);
    consume(vb, (bt + 1) * kScanBatch);
  } else {
    consume(va, bt * kScanBatch);
  }

  if constexpr (KEEP_ALL) {
#pragma unroll
    for (int m = 0; m < KM; ++m) {
      const int64_t key = key_of(8 * m + sub, kl);
      float sv = sc[m] * scale;
      if constexpr (GUMBEL) {
        if (key < n) sv += gumbel_noise(seed, (uint32_t)row, 0u, (uint32_t)(lo + key));
      }
      if (key < n && __builtin_isfinite(sv) && in_use(key)) L.insert(sv, (int)(lo + key));
    }
  }
  float ms;
  int mj, cnt;
  wave_merge(L, K, ms, mj, cnt);
  if (lane < K) {
    const int64_t o = (row * lists + list) * K + lane;
    cs[o] = lane < cnt ? ms : -INFINITY;
    cj[o] = lane < cnt ? mj : -1;
  }
}

template <typename T, int KM, bool KEEP_ALL, bool GUMBEL, bool Q8, bool MASK>
hipError_t launch_scan_q(const Shape& s, const void* lq, const void* lk, const int32_t* tokens, void* ws,
                         hipStream_t st) {
  const DecodePlan plan = decode_plan(s);
  const int64_t rows = (int64_t)s.B * s.Hr;
  float* cs = decode_list_scores(s, ws);
  int* cj = decode_list_chunks(s, ws);
  // the query, and with MASK one bit per key of a workgroup's range (whole words of its threads)
  const size_t range = (size_t)((kScanWaves * plan.pw + kScanThreads - 1) / kScanThreads) * kScanThreads;
  const size_t smem = (Q8 ? 0 : (size_t)s.D * sizeof(T)) + (MASK ? range / 8 : 0);
  launch_kernel(MASK ? "cache_scan_kernel" : "decode_scan_kernel",
                decode_scan_kernel<T, KM, KEEP_ALL, GUMBEL, Q8, MASK>, dim3((unsigned)(rows * plan.wgs)),
                dim3(kScanThreads), smem, st, (const T*)lq, (const T*)lk, cs, cj, s.nKV, s.D, s.score_scale, s.topk,
                plan.pw, plan.lists, plan.wgs, s.gumbel_seed, tokens, s.Hr);
  return take_launch_error();
}

template <typename T, int KM, bool KEEP_ALL, bool GUMBEL, bool MASK>
hipError_t launch_scan_k(const Shape& s, const void* lq, const void* lk, const int32_t* tokens, void* ws,
                         hipStream_t st) {
  if (s.D == 64 * kScanBatch) return launch_scan_q<T, KM, KEEP_ALL, GUMBEL, true, MASK>(s, lq, lk, tokens, ws, st);
  return launch_scan_q<T, KM, KEEP_ALL, GUMBEL, false, MASK>(s, lq, lk, tokens, ws, st);
}

// The scan of one problem (tokens: with MASK, the lengths of the cached chunks).
template <typename T, bool G, bool MASK>
hipError_t launch_scan(const Shape& s, const void* lmk_q, const void* lmk_k, const int32_t* tokens, void* ws,
                       hipStream_t stream) {
  // A lane sees at most ceil(pw / 64) keys of its wave's range (one key of every
  // eighth group of 8).  Up to k of them it keeps every raw score and ranks them
  // at the end; beyond, it keeps a running best-k list.
  const int64_t per_lane = (decode_plan(s).pw + 63) / 64;
  if (per_lane <= s.topk) {
    if (per_lane <= 1) return launch_scan_k<T, 1, true, G, MASK>(s, lmk_q, lmk_k, tokens, ws, stream);
    if (per_lane <= 2) return launch_scan_k<T, 2, true, G, MASK>(s, lmk_q, lmk_k, tokens, ws, stream);
    if (per_lane <= 4) return launch_scan_k<T, 4, true, G, MASK>(s, lmk_q, lmk_k, tokens, ws, stream);
    if (per_lane <= 8) return launch_scan_k<T, 8, true, G, MASK>(s, lmk_q, lmk_k, tokens, ws, stream);
    if (per_lane <= 16) return launch_scan_k<T, 16, true, G, MASK>(s, lmk_q, lmk_k, tokens, ws, stream);
    return launch_scan_k<T, 32, true, G, MASK>(s, lmk_q, lmk_k, tokens, ws, stream);
  }
  if (s.topk <= 8) return launch_scan_k<T, 8, false, G, MASK>(s, lmk_q, lmk_k, tokens, ws, stream);
  if (s.topk <= 16) return launch_scan_k<T, 16, false, G, MASK>(s, lmk_q, lmk_k, tokens, ws, stream);
  return launch_scan_k<T, 32, false, G, MASK>(s, lmk_q, lmk_k, tokens, ws, stream);
}

}  // namespace
}  // namespace gca
