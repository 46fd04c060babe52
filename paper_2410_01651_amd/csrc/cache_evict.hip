// Eviction from the chunk cache (gca_cache_evict): the chunks' masses take in the attention
// weights of the lists used since, and the slots of the next chunks are chosen, free ones
// first, then the least attended.
//
// Mathematics.  mass'[j] = decay mass[j] + sum of the weights of the entries naming j.  The
// sum is formed in LDS in units of 2^-48 as 64-bit integers, so that it does not depend on the
// order of the atomic additions; the product and the sum with it are one fp64 fma, rounded
// once to fp32.  The choice is the m smallest keys of a slot order: key 0 for a free slot, 1 +
// the bits of the mass (non-negative floats order as their bits) for one that may go, the
// largest key for one that must stay.  The m-th smallest key is found by splitting the range
// of the keys into at most 256 equal parts (a histogram in LDS), and again the part that holds
// it, at most four times; keys below it are taken, and of its equals the lowest slots.
//
// Work.  One workgroup per sequence and tile of kEvictTile slots: masses read and written
// once, keys in LDS.  A cache of more tiles leaves each tile's n smallest in the workspace and
// a second launch, one workgroup per sequence, chooses among them.  Bound by its chain of
// dependent steps (a few barriers each): there are 16 bytes per slot to read.
#include "cache_plan.hpp"
#include "gca_device.hpp"
#include "gca_launch.hpp"

namespace gca {
namespace {

constexpr uint32_t kStays = 0xffffffffu;
constexpr int kBins = 256;

struct EvictParams {
  const int32_t* idx;
  const float* w;
  const int32_t* want;
  int32_t* slots;
  int32_t* tokens;
  float* mass;
  int32_t* number;
  int32_t* next;
  uint32_t* cand_key;  // [B, tiles, per] (more than one tile)
  int32_t* cand_slot;
  int64_t C;
  uint32_t entries;  // of a sequence's lists
  uint32_t tiles, per;
  int n, keep_first, keep_last;
  float decay;
};

// Scratch of one workgroup (up to 16 waves).
struct Scratch {
  uint32_t hist[kBins];
  uint32_t a[16], b[16], c[16];
  uint32_t lo, hi, below, done;
};

__device__ __forceinline__ uint32_t wave_min(uint32_t x) {
  x = min(x, dpp<kDppXor1>(x));
  x = min(x, dpp<kDppXor2>(x));
  x = min(x, dpp<kDppRor4>(x));
  x = min(x, dpp<kDppRor8>(x));
  uint32_t a, b;
  pair16(x, a, b);
  x = min(a, b);
  pair32(x, a, b);
  return min(a, b);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) { return ~wave_min(~x); }
__device__ __forceinline__ uint32_t wave_sum(uint32_t x) {
  x += dpp<kDppXor1>(x);
  x += dpp<kDppXor2>(x);
  x += dpp<kDppRor4>(x);
  x += dpp<kDppRor8>(x);
  uint32_t a, b;
  pair16(x, a, b);
  x = a + b;
  pair32(x, a, b);
  return a + b;
}
// Sum over the lanes up to and including this one.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

// The m smallest of keys[0 .. N) that are not kStays, of equal keys the first ones: calls
// take(rank, index) for each, ranks 0, 1, .. in order of index.  Returns how many there are (at
// most m).  keys: LDS or global memory, written before a barrier; every thread of the
// workgroup takes part.
template <typename Keys, typename Take>
__device__ uint32_t take_smallest(Scratch& s, Keys keys, uint32_t N, uint32_t m, Take take) {
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nw = blockDim.x >> 6;
  const uint32_t seg = (N + blockDim.x - 1) / blockDim.x;  // a thread's consecutive keys
  const uint32_t x0 = min(tid * seg, N), x1 = min(x0 + seg, N);
  // how many there are, the least and the largest
  uint32_t cnt = 0, lo = kStays, hi = 0;
  for (uint32_t x = x0; x < x1; ++x) {
    const uint32_t k = keys(x);
    if (k == kStays) continue;
    ++cnt;
    lo = min(lo, k);
    hi = max(hi, k);
  }
  cnt = wave_sum(cnt);
  lo = wave_min(lo);
  hi = wave_max(hi);
  __syncthreads();  // the scratch's last readers are done
  if (lane == 0) {
    s.a[wave] = cnt;
    s.b[wave] = lo;
    s.c[wave] = hi;
  }
  __syncthreads();
  cnt = 0;
  for (uint32_t y = 0; y < nw; ++y) {
    cnt += s.a[y];
    lo = min(lo, s.b[y]);
    hi = max(hi, s.c[y]);
  }
  m = min(m, cnt);
  if (m == 0) return 0;
  // [lo, hi] holds the m-th smallest key; `below` keys are less than lo
  uint32_t below = 0;
  if (m == 1) hi = lo;  // the least
  bool whole = m == cnt;  // every key up to hi is taken
  while (!whole && lo < hi) {
    const int range_bits = 32 - __builtin_clz(hi - lo);
    const int shift = range_bits > 8 ? range_bits - 8 : 0;
    for (uint32_t y = tid; y < kBins; y += blockDim.x) s.hist[y] = 0;
    __syncthreads();
    for (uint32_t x = x0; x < x1; ++x) {
      const uint32_t k = keys(x);
      if (k >= lo && k <= hi) atomicAdd(&s.hist[(k - lo) >> shift], 1u);
    }
    __syncthreads();
    if (wave == 0) {
      // lane l: bins 4 l .. 4 l + 3
      uint32_t h[4], sum = 0;
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        h[y] = s.hist[4 * lane + y];
        sum += h[y];
      }
      uint32_t before = below + wave_scan(sum) - sum;
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        if (before < m && m <= before + h[y]) {  // one lane's one bin
          const uint32_t first = lo + ((4 * lane + y) << shift);
          s.lo = first;
          s.hi = min(hi, first + ((1u << shift) - 1u));
          s.below = before;
          s.done = m == before + h[y];
        }
        before += h[y];
      }
    }
    __syncthreads();
    lo = s.lo;
    hi = s.hi;
    below = s.below;
    whole = s.done != 0;
    __syncthreads();
  }
  // taken: keys up to hi (whole), or keys below lo and the first m - below equal to lo
  const uint32_t need = whole ? 0 : m - below;
  auto less = [&](uint32_t k) { return whole ? k <= hi : k < lo; };
  uint32_t nl = 0, ne = 0;
  for (uint32_t x = x0; x < x1; ++x) {
    const uint32_t k = keys(x);
    if (k == kStays) continue;
    nl += less(k);
    ne += !whole && k == lo;
  }
  const uint32_t sl = wave_scan(nl), se = wave_scan(ne);
  __syncthreads();
  if (lane == 63) {
    s.a[wave] = sl;
    s.b[wave] = se;
  }
  __syncthreads();
  uint32_t rl = sl - nl, re = se - ne;  // taken outright / equal, before this thread's keys
  for (uint32_t y = 0; y < wave; ++y) {
    rl += s.a[y];
    re += s.b[y];
  }
  for (uint32_t x = x0; x < x1; ++x) {
    const uint32_t k = keys(x);
    if (k == kStays) continue;
    if (less(k)) {
      take(rl + min(re, need), x);
      ++rl;
    } else if (!whole && k == lo) {
      if (re < need) take(rl + re, x);
      ++re;
    }
  }
  return m;
}

// The slots that a sequence gives to its next chunks (the caller's keys name them).
template <typename Keys, typename Slot>
__device__ void give_slots(const EvictParams& p, Scratch& s, uint32_t b, Keys keys, uint32_t N, Slot slot_of) {
  const int want = p.want ? min(max(p.want[b], 0), p.n) : p.n;
  const int first = p.next[b];
  int32_t* out = p.slots + (int64_t)b * p.n;
  const int64_t base = (int64_t)b * p.C;
  const uint32_t got = take_smallest(s, keys, N, (uint32_t)want, [&](uint32_t rank, uint32_t x) {
    const int slot = slot_of(x);
    out[rank] = slot;
    p.tokens[base + slot] = 0;
    p.mass[base + slot] = 0.f;
    p.number[base + slot] = (int32_t)((uint32_t)first + rank);
  });
  for (uint32_t x = got + threadIdx.x; x < (uint32_t)p.n; x += blockDim.x) out[x] = -1;
  __syncthreads();  // every thread has read next[b]
  if (threadIdx.x == 0) p.next[b] = (int32_t)((uint32_t)first + (uint32_t)want);
}

__global__ __launch_bounds__(1024) void cache_evict_kernel(EvictParams p) {
  __shared__ unsigned long long acc[kEvictTile];  // units of 2^-48
  __shared__ uint32_t key[kEvictTile];
  __shared__ Scratch s;
  const uint32_t b = blockIdx.x / p.tiles, tile = blockIdx.x % p.tiles, tid = threadIdx.x;
  const uint32_t c0 = tile * kEvictTile;
  const uint32_t N = (uint32_t)min((int64_t)kEvictTile, p.C - c0);
  if (p.entries) {
    for (uint32_t x = tid; x < N; x += blockDim.x) acc[x] = 0;
    __syncthreads();
    const int32_t* idx = p.idx + (int64_t)b * p.entries;
    const float* w = p.w + (int64_t)b * p.entries;
    for (uint32_t e = tid; e < p.entries; e += blockDim.x) {
      const uint32_t x = (uint32_t)idx[e] - c0;  // entries of other tiles and pads fall outside
      if (idx[e] < 0 || x >= N) continue;
      const float f = w[e];
      const double u = f > 0.f ? (double)fminf(f, 32768.f) * 0x1p48 : 0.0;
      atomicAdd(&acc[x], (unsigned long long)(u + 0.5));
    }
    __syncthreads();
  }
  const int64_t base = (int64_t)b * p.C + c0;
  const int64_t next = p.next[b];
  for (uint32_t x = tid; x < N; x += blockDim.x) {
    const bool used = p.tokens[base + x] > 0;
    float m = 0.f;
    if (used) {
      m = p.mass[base + x];
      const double add = p.entries ? (double)acc[x] * 0x1p-48 : 0.0;
      m = (float)fma((double)p.decay, (double)m, add);
    }
    p.mass[base + x] = m;
    const int64_t num = p.number[base + x];
    const bool stays = used && (num < p.keep_first || num >= next - p.keep_last);
    key[x] = !used ? 0u : stays ? kStays : m > 0.f ? __float_as_uint(m) + 1u : 1u;
  }
  if (p.n == 0) return;
  __syncthreads();
  auto keys = [&](uint32_t x) { return key[x]; };
  if (p.tiles == 1) {
    give_slots(p, s, b, keys, N, [](uint32_t x) { return (int)x; });
  } else {
    const int64_t at = (int64_t)blockIdx.x * p.per;
    const uint32_t got = take_smallest(s, keys, N, p.per, [&](uint32_t rank, uint32_t x) {
      p.cand_key[at + rank] = key[x];
      p.cand_slot[at + rank] = (int32_t)(c0 + x);
    });
    for (uint32_t x = got + tid; x < p.per; x += blockDim.x) p.cand_key[at + x] = kStays;
  }
}

__global__ __launch_bounds__(1024) void cache_evict_merge_kernel(EvictParams p) {
  __shared__ Scratch s;
  const uint32_t b = blockIdx.x, N = p.tiles * p.per;
  const uint32_t* key = p.cand_key + (int64_t)b * N;
  const int32_t* slot = p.cand_slot + (int64_t)b * N;
  give_slots(p, s, b, [&](uint32_t x) { return key[x]; }, N, [&](uint32_t x) { return slot[x]; });
}

}  // namespace

hipError_t launch_cache_evict(const gca_cache& c, const int32_t* idx, const float* w, int64_t nQ, float decay,
                              int keep_first, int keep_last, const int32_t* want, int32_t* slots, int64_t n, void* ws,
                              hipStream_t stream) {
  EvictParams p;
  p.idx = idx;
  p.w = w;
  p.want = want;
  p.slots = slots;
  p.tokens = c.tokens;
  p.mass = c.mass;
  p.number = c.number;
  p.next = c.next;
  p.C = c.capacity;
  p.entries = idx ? (uint32_t)((int64_t)c.Hr * nQ * c.topk) : 0u;
  p.tiles = (uint32_t)evict_tiles(c);
  p.per = n > 0 ? (uint32_t)evict_per_tile(n) : 0u;
  p.cand_key = static_cast<uint32_t*>(ws);
  p.cand_slot = reinterpret_cast<int32_t*>(p.cand_key + (size_t)c.B * p.tiles * p.per);
  p.n = (int)n;
  p.keep_first = keep_first;
  p.keep_last = keep_last;
  p.decay = decay;
  const unsigned threads = c.capacity <= 2048 ? 256 : 1024;
  launch_kernel("cache_evict_kernel", cache_evict_kernel, dim3((unsigned)(c.B * (int64_t)p.tiles)), dim3(threads), 0,
                stream, p);
  if (p.tiles > 1 && n > 0) {
    const unsigned mt = p.tiles * p.per <= 2048 ? 256 : 1024;
    launch_kernel("cache_evict_merge_kernel", cache_evict_merge_kernel, dim3((unsigned)c.B), dim3(mt), 0, stream, p);
  }
  return take_launch_error();
}

}  // namespace gca
