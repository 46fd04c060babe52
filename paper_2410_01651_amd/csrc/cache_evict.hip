// Eviction from the chunk cache (gca_cache_evict): the chunks' masses take in the attention
// weights of the lists used since, and the slots of the next chunks are chosen, free ones
// first, then the least attended.
//
// Mathematics.  mass'[j] = decay mass[j] + sum of the weights of the entries naming j.  The
// sum is formed in LDS in units of 2^-48 (coarser from 2^16 entries on, so that no sum of weights up
// to 1 passes 64 bits) as 64-bit integers, so that it does not depend on the order of the atomic
// additions; the product and the sum with it are one fp64 fma, rounded
// once to fp32.  The choice is the m smallest keys of a slot order: key 0 for a free slot, 1 +
// the bits of the mass (non-negative floats order as their bits) for one that may go, the
// largest key for one that must stay.  The m-th smallest key is found by splitting the range
// of the keys into at most 2,048 equal parts (a histogram in LDS), and again the part that holds
// it, at most three times, or until the part has no more than 64 keys, which one wave sorts; keys
// below it are taken, and of its equals the lowest slots.
//
// Work.  One workgroup per sequence for up to kEvictWhole slots: masses read and written once,
// keys in LDS.  A larger cache is cut into tiles of kEvictTile slots (more workgroups, so that a
// few long caches spread over the chip); each leaves its n smallest in the workspace and a second
// launch, one workgroup per sequence, chooses among them.  Bound by its chain of
// dependent steps (a few barriers each): there are 12 bytes per slot to read and 4 to write.
// 32 sequences of 256 slots, one to go: 4.1 us; 64 of 8,192, 8 to go: 12.9; 4 of 50,000, 40 to go:
// 9.2 + 5.7, 1,024 to go (more candidates than the registers hold, read again in every pass): 10.6 + 63.
#include "cache_plan.hpp"
#include "gca_device.hpp"
#include "gca_launch.hpp"

namespace gca {
namespace {

constexpr uint32_t kStays = 0xffffffffu;
constexpr int kBins = 2048;  // of a histogram; eight per thread of the smaller workgroup

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
  uint64_t list[64];
  uint32_t a[16], b[16], c[16], d[16];
  uint32_t lo, hi, below, count;
  uint64_t bound;
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
// Sum over the lanes up to and including this one (DPP row shifts, then the rows' last lanes
// broadcast to the rows after them).
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, true);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, true);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, true);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, true);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);
  return x;
}

// The sum of x over the threads before this one.
__device__ __forceinline__ uint32_t before_me(uint32_t x, uint32_t* sums) {
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t in = wave_scan(x);
  if (lane == 63) sums[wave] = in;
  block_barrier();
  uint32_t r = in - x;
  for (uint32_t y = 0; y < wave; ++y) r += sums[y];
  return r;
}

// The m smallest of keys(0 .. N) that are not kStays, of equal keys the first ones: calls
// take(rank, index) for each, ranks 0, 1, .. in order of index.  Returns how many there are (at
// most m).  keys reads LDS or global memory written before a barrier; every thread of the
// workgroup takes part.  PER: a thread's keys at most, then held in registers; 0: any number.
// (The barriers order LDS alone.)
template <int PER, typename Keys, typename Take>
__device__ uint32_t take_smallest(Scratch& s, Keys keys, uint32_t N, uint32_t m, Take take) {
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nw = blockDim.x >> 6;
  const uint32_t seg = (N + blockDim.x - 1) / blockDim.x;  // a thread's consecutive keys
  const uint32_t x0 = min(tid * seg, N), x1 = min(x0 + seg, N);
  uint32_t own[PER ? PER : 1];
  if constexpr (PER > 0) {
#pragma unroll
    for (int u = 0; u < PER; ++u) own[u] = x0 + u < x1 ? keys(x0 + u) : kStays;
  }
  auto each = [&](auto f) {  // f(key, index) of a thread's keys in order, kStays among them
    if constexpr (PER > 0) {
#pragma unroll
      for (int u = 0; u < PER; ++u) f(own[u], x0 + u);
    } else {
      for (uint32_t x = x0; x < x1; ++x) f(keys(x), x);
    }
  };
  // how many there are, the least (and the first of those) and the largest
  uint32_t cnt = 0, lo = kStays, hi = 0, at = kStays;
  each([&](uint32_t k, uint32_t x) {
    const bool is = k != kStays;
    cnt += is;
    at = k < lo ? x : at;
    lo = min(lo, k);
    hi = max(hi, is ? k : 0u);
  });
  cnt = wave_sum(cnt);
  const uint32_t least = wave_min(lo);
  at = wave_min(lo == least ? at : kStays);
  hi = wave_max(hi);
  if (lane == 0) {
    s.a[wave] = cnt;
    s.b[wave] = least;
    s.c[wave] = hi;
    s.d[wave] = at;
  }
  block_barrier();
  cnt = 0;
  lo = kStays;
  hi = 0;
  for (uint32_t y = 0; y < nw; ++y) {
    cnt += s.a[y];
    if (s.b[y] < lo) {
      lo = s.b[y];
      at = s.d[y];
    }
    hi = max(hi, s.c[y]);
  }
  block_barrier();  // (the scratch is written again)
  m = min(m, cnt);
  if (m == 0) return 0;
  if (m == 1) {
    if (tid == 0) take(0, at);
    return 1;
  }
  // Taken are the keys with (key, index) up to a bound.  [lo, hi] holds the m-th smallest key,
  // `below` keys are less than lo.
  uint64_t bound = ((uint64_t)hi << 32) | 0xffffffffu;
  uint32_t below = 0, count = cnt;
  while (m != below + count) {  // (else all of the range's keys are taken)
    if (count <= 64) {
      // few enough to be sorted by one wave
      if (tid == 0) s.count = 0;
      block_barrier();
      each([&](uint32_t k, uint32_t x) {
        if (k >= lo && k <= hi) s.list[atomicAdd(&s.count, 1u)] = ((uint64_t)k << 32) | x;
      });
      block_barrier();
      if (wave == 0) {
        const uint64_t sorted = wave_sort_desc(lane < count ? ~s.list[lane] : uint64_t(0));  // least first
        if (lane == m - below - 1) s.bound = ~sorted;
      }
      block_barrier();
      bound = s.bound;
      break;
    }
    if (lo == hi) {
      // the first m - below of equal keys
      uint32_t ne = 0;
      each([&](uint32_t k, uint32_t) { ne += k == lo; });
      uint32_t r = before_me(ne, s.a);
      each([&](uint32_t k, uint32_t x) {
        if (k == lo && ++r == m - below) s.bound = ((uint64_t)k << 32) | x;
      });
      block_barrier();
      bound = s.bound;
      break;
    }
    // the part, of at most kBins equal ones, that holds the m-th smallest
    const int range_bits = 32 - __builtin_clz(hi - lo);
    const int shift = range_bits > 11 ? range_bits - 11 : 0;
    for (uint32_t y = tid; y < kBins; y += blockDim.x) s.hist[y] = 0;
    block_barrier();
    // (masses repeat, zeros above all: a thread adds runs of one bin at once, and a wave whose last
    // runs share a bin their sum, so that equal keys do not queue for one counter)
    uint32_t bin = kBins, run = 0;
    each([&](uint32_t k, uint32_t) {
      if (k < lo || k > hi) return;
      const uint32_t to = (k - lo) >> shift;
      if (to != bin && run) {
        atomicAdd(&s.hist[bin], run);
        run = 0;
      }
      bin = to;
      ++run;
    });
    const uint64_t have = __ballot(run != 0);
    if (have) {
      const uint32_t shared = __builtin_amdgcn_readlane(bin, __builtin_ctzll(have));
      if (__ballot(run != 0 && bin != shared) == 0) {
        const uint32_t sum = wave_sum(run);
        if (lane == 0) atomicAdd(&s.hist[shared], sum);
      } else if (run) {
        atomicAdd(&s.hist[bin], run);
      }
    }
    block_barrier();
    const uint32_t bins = kBins / blockDim.x;  // 8 or 2 per thread, consecutive
    uint32_t sum = 0;
    for (uint32_t y = 0; y < bins; ++y) sum += s.hist[tid * bins + y];
    uint32_t before = below + before_me(sum, s.a);
    if (before < m && m <= before + sum) {  // one thread
      for (uint32_t y = 0; y < bins; ++y) {
        const uint32_t n = s.hist[tid * bins + y];
        if (m <= before + n) {
          const uint32_t first = lo + ((tid * bins + y) << shift);
          s.lo = first;
          s.hi = min(hi, first + ((1u << shift) - 1u));
          s.below = before;
          s.count = n;
          break;
        }
        before += n;
      }
    }
    block_barrier();
    lo = s.lo;
    hi = s.hi;
    below = s.below;
    count = s.count;
    bound = ((uint64_t)hi << 32) | 0xffffffffu;
    block_barrier();  // (the scratch is written again)
  }
  auto taken = [&](uint32_t k, uint32_t x) { return k != kStays && (((uint64_t)k << 32) | x) <= bound; };
  uint32_t n = 0;
  each([&](uint32_t k, uint32_t x) { n += taken(k, x); });
  uint32_t rank = before_me(n, s.b);
  each([&](uint32_t k, uint32_t x) {
    if (taken(k, x)) take(rank++, x);
  });
  return m;
}

// The slots that a sequence gives to its next chunks (the caller's keys name them).
template <int PER, typename Keys, typename Slot>
__device__ void give_slots(const EvictParams& p, Scratch& s, uint32_t b, Keys keys, uint32_t N, Slot slot_of) {
  const int want = p.want ? min(max(p.want[b], 0), p.n) : p.n;
  const int first = p.next[b];
  int32_t* out = p.slots + (int64_t)b * p.n;
  const int64_t base = (int64_t)b * p.C;
  const uint32_t got = take_smallest<PER>(s, keys, N, (uint32_t)want, [&](uint32_t rank, uint32_t x) {
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

// TILE: slots per workgroup; a thread has at most kPer of them.
template <int TILE, int THREADS>
__global__ __launch_bounds__(THREADS) void cache_evict_kernel(EvictParams p) {
  constexpr int kPer = TILE / THREADS;
  __shared__ unsigned long long acc[TILE];  // in units
  // key x at x + x / 32: the threads' consecutive keys then lie in different banks
  __shared__ uint32_t key[TILE + TILE / 32];
  __shared__ Scratch s;
  const uint32_t b = blockIdx.x / p.tiles, tile = blockIdx.x % p.tiles, tid = threadIdx.x;
  const uint32_t c0 = tile * TILE;
  const uint32_t N = (uint32_t)min((int64_t)TILE, p.C - c0);
  const int64_t base = (int64_t)b * p.C + c0;
  const int64_t next = p.next[b];
  // entries < 2^bits, each at most 2^(64 - bits) units
  const int bits = max(16, 32 - __builtin_clz(p.entries | 1));
  const double units = __longlong_as_double((int64_t)(1023 + 64 - bits) << 52);
  const double unit = __longlong_as_double((int64_t)(1023 - 64 + bits) << 52);
  // everything of a thread's slots is asked for before the lists, and at once: a load that a branch
  // guards would be waited for before the next (threads without a slot take the last one's)
  int32_t tokens[kPer], number[kPer];
  float mass[kPer];
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const uint32_t x = min(tid + u * THREADS, N - 1);
    tokens[u] = p.tokens[base + x];
    mass[u] = p.mass[base + x];
    number[u] = p.number[base + x];
  }
  if (p.entries) {
    for (uint32_t x = tid; x < N; x += THREADS) acc[x] = 0;
    __syncthreads();
    const int32_t* idx = p.idx + (int64_t)b * p.entries;
    const float* w = p.w + (int64_t)b * p.entries;
    auto add = [&](int32_t j, float f) {
      const uint32_t x = (uint32_t)j - c0;  // entries of other tiles and pads fall outside
      if (j < 0 || x >= N) return;
      const double u = f > 0.f ? (double)fminf(f, 1.f) * units : 0.0;
      atomicAdd(&acc[x], (unsigned long long)(u + 0.5));
    };
    uint32_t e = tid;
    for (; (uint64_t)e + 7 * THREADS < p.entries; e += 8 * THREADS) {  // eight in flight
      int32_t j[8];
      float f[8];
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        j[y] = idx[e + y * THREADS];
        f[y] = w[e + y * THREADS];
      }
#pragma unroll
      for (int y = 0; y < 8; ++y) add(j[y], f[y]);
    }
    for (; e < p.entries; e += THREADS) add(idx[e], w[e]);
    __syncthreads();
  }
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const uint32_t x = tid + u * THREADS;
    if (x < N) {
      const bool used = tokens[u] > 0;
      const double add = p.entries ? (double)acc[x] * unit : 0.0;
      const float m = used ? (float)fma((double)p.decay, (double)mass[u], add) : 0.f;
      p.mass[base + x] = m;
      const int64_t num = number[u];
      const bool stays = used && (num < p.keep_first || num >= next - p.keep_last);
      key[x + x / 32] = !used ? 0u : stays ? kStays : m > 0.f ? __float_as_uint(m) + 1u : 1u;
    }
  }
  if (p.n == 0) return;
  __syncthreads();
  auto keys = [&](uint32_t x) { return key[x + x / 32]; };
  if (p.tiles == 1) {
    give_slots<kPer>(p, s, b, keys, N, [](uint32_t x) { return (int)x; });
  } else {
    const int64_t at = (int64_t)blockIdx.x * p.per;
    const uint32_t got = take_smallest<kPer>(s, keys, N, p.per, [&](uint32_t rank, uint32_t x) {
      p.cand_key[at + rank] = keys(x);
      p.cand_slot[at + rank] = (int32_t)(c0 + x);
    });
    for (uint32_t x = got + tid; x < p.per; x += THREADS) p.cand_key[at + x] = kStays;
  }
}

template <int PER>
__global__ __launch_bounds__(1024) void cache_evict_merge_kernel(EvictParams p) {
  __shared__ Scratch s;
  const uint32_t b = blockIdx.x, N = p.tiles * p.per;
  const uint32_t* key = p.cand_key + (int64_t)b * N;
  const int32_t* slot = p.cand_slot + (int64_t)b * N;
  give_slots<PER>(p, s, b, [&](uint32_t x) { return key[x]; }, N, [&](uint32_t x) { return slot[x]; });
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
  const dim3 grid((unsigned)(c.B * (int64_t)p.tiles));
  if (p.tiles == 1 && c.capacity > kEvictTile)
    launch_kernel("cache_evict_kernel", cache_evict_kernel<kEvictWhole, 1024>, grid, dim3(1024), 0, stream, p);
  else
    launch_kernel("cache_evict_kernel", cache_evict_kernel<kEvictTile, 256>, grid, dim3(256), 0, stream, p);
  if (p.tiles > 1 && n > 0) {
    const uint32_t N = p.tiles * p.per;
    launch_kernel("cache_evict_merge_kernel", N <= 8192 ? cache_evict_merge_kernel<8> : cache_evict_merge_kernel<0>,
                  dim3((unsigned)c.B), dim3(N <= 2048 ? 256 : 1024), 0, stream, p);
  }
  return take_launch_error();
}

}  // namespace gca
