// Verification of drafted tokens (gca_verify): a walk down each sequence's tree by rejection sampling, and
// the draw of the token that follows.
//
// Mathematics.  At node a, with r = p[a] and z = 1, child x is accepted with probability
// min(1, r[x] / (z q[x])); a rejection leaves r <- max(r - z q, 0), z <- sum r.  (r / z is then the
// distribution that the next child, drawn from q too, has to make up for; with the draw from r at
// the end each token comes out with probability p[a].)  Children that were chosen rather than drawn are q = 1
// at x.  Everything is fp64 without contraction, and sums are of whole multiples of 2^-44 in 64-bit unsigned
// integers (2^19 entries of at most 1 are at most 2^63), so that results do not depend on how the work is cut.
//
// Work.  One lane per node holds the node's token and its entries of p and q, so that the walk is
// comparisons and ballots after two dependent loads.  The vocabulary is cut into slices, one
// workgroup each, and each workgroup repeats the walk rather than wait for another's; only a rejected child
// that was drawn from q and has a sibling left needs the sum over the whole vocabulary on the way, which every
// workgroup then forms by itself, from p again for each: of 120,001 tokens, drafts drawn from q, one sequence takes 4.5 us
// for its walk where a single child is rejected, 46 with two siblings, 95 with three, 284 with six and 2,840 with 24 (32
// sequences with one to three and six 8, 98, 201 and 579; 250,000 tokens and 63 siblings 36 ms).  A second launch picks the slice and the token by the slices' sums.
// Bound by HBM, the last node's p (and q, where it was rejected from), or, for few sequences, by
// the trips to memory.  64 chains of 8, 100,000 tokens: 12 us of walk and sums (51 MB, 4.3 TB/s) and 4 of the draw;
// one chain of 5, 32,000 tokens: 4.8 and 3.9.  In one launch, a workgroup of 1,024 threads per sequence: 12.8 us for
// that chain (8.2 for 2,000 tokens), as one CU reads its rows, and for 1,024 of them 53.6 for 30 and 11.  All first
// children's tests at once: 32 trees of up to 25 nodes 8.4 us for 9.9.
#include "gca_device.hpp"
#include "gca_launch.hpp"
#include "window_plan.hpp"

namespace gca {
namespace {

constexpr int kVerifyThreads = 256;
constexpr int kVerifyWaves = kVerifyThreads / 64;
constexpr int kPerThread = 8;  // consecutive entries of a thread where order counts
constexpr double kFix = 17592186044416.0;       // 2^44
constexpr double kUnfix = 1.0 / 17592186044416.0;

// What a walk ends with, per sequence.
struct Walk {
  int32_t node;      // the last node, -1: no nodes
  int32_t rejected;  // children rejected there
  uint64_t on;       // the walk's nodes
  double z[kTreeNodes];      // drawn children: z before each rejection
  int32_t token[kTreeNodes]; // chosen ones: the rejected tokens
};

struct VerifyParams {
  const float* p;
  const float* q;
  const int32_t* tokens;
  const int32_t* parents;
  const float* u;
  const int32_t* lengths;
  int32_t* path;
  int32_t* count;
  int32_t* next;
  Walk* walk;      // [B]
  uint64_t* sums;   // [B][slices][waves]
  uint32_t T, slices;
  uint32_t V, per;  // entries in all, and per wave of a slice (a multiple of 4)
};

// A probability as it counts.
__device__ __forceinline__ double prob(float x) {
  return x > 0.f ? (double)fminf(x, 1.f) : 0.0;  // (NaN and below: 0)
}
// r - z q, at least 0: a product and a difference, each rounded.
__device__ __forceinline__ double less(double r, double z, double q) {
#pragma clang fp contract(off)
  const double s = z * q;
  const double d = r - s;
  return d > 0.0 ? d : 0.0;
}
// Whether u z q < r: two products, each rounded.
__device__ __forceinline__ bool test(double u, double z, double q, double r) {
#pragma clang fp contract(off)
  const double s = z * q;
  const double us = u * s;
  return us < r;
}
// r in whole multiples of 2^-44, to the nearest (ties to even): 0 .. 2^44, so the sum with 2^52 holds it
// in its mantissa.
__device__ __forceinline__ uint64_t whole(double r) {
  const double x = r * kFix + 4503599627370496.0;
  return (uint64_t)__double_as_longlong(x) & 0xfffffffffffffull;
}

// Lane c's value, c the same in every lane.
__device__ __forceinline__ int lane_of(int x, int c) { return __builtin_amdgcn_readlane(x, c); }
__device__ __forceinline__ double lane_of(double x, int c) {
  const uint64_t u = (uint64_t)__double_as_longlong(x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, c);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), c);
  return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}

__device__ __forceinline__ uint64_t wave_sum(uint64_t x) {
#pragma unroll
  for (int s = 1; s < 64; s *= 2) x += __shfl_xor(x, s);
  return x;
}

typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4u;

// What the rejections at the walk's last node leave of N consecutive entries from x on, as whole numbers;
// `chosen`: of the rejected tokens too.
template <int N>
__device__ __forceinline__ void left(const Walk& w, bool drawn, bool chosen, const float* p, const float* q, uint32_t x,
                                     uint64_t* out) {
  double r[N];
#pragma unroll
  for (int e = 0; e < N; ++e) r[e] = prob(p[e]);
  if (drawn)
    for (int j = 0; j < w.rejected; ++j) {
      const double z = w.z[j];
#pragma unroll
      for (int e = 0; e < N; ++e) r[e] = less(r[e], z, prob(q[e]));
    }
  else if (chosen)
    for (int j = 0; j < w.rejected; ++j) {
      const uint32_t t = (uint32_t)w.token[j];
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (t == x + e) r[e] = 0.0;
    }
#pragma unroll
  for (int e = 0; e < N; ++e) out[e] = whole(r[e]);
}

// Part `part` of `parts` (lanes or threads) of the sum of r over entries [lo, hi) of the last node's row, four
// consecutive entries at a time; `plain`: of p[a] itself.
__device__ __forceinline__ uint64_t part_sum(const VerifyParams& p, const Walk& w, uint32_t b, uint32_t lo, uint32_t hi,
                                            bool plain, uint32_t part, uint32_t parts) {
  const int64_t row = ((int64_t)b * p.T + w.node) * p.V;
  const float* pr = p.p + row;
  const bool drawn = p.q != nullptr && w.rejected > 0 && !plain;
  uint64_t sum = 0;
  uint32_t x = lo + 4 * part;
  if (drawn) {
    const float* qr = p.q + row;
#pragma unroll 4
    for (; x + 4 <= hi; x += 4 * parts) {
      const f32x4u a = *reinterpret_cast<const f32x4u*>(pr + x), c = *reinterpret_cast<const f32x4u*>(qr + x);
      const float pe[4] = {a[0], a[1], a[2], a[3]}, qe[4] = {c[0], c[1], c[2], c[3]};
      uint64_t r[4];
      left<4>(w, true, false, pe, qe, x, r);
      sum += r[0] + r[1] + r[2] + r[3];
    }
    for (; x < hi; ++x) {
      uint64_t r;
      left<1>(w, true, false, pr + x, qr + x, x, &r);
      sum += r;
    }
    return sum;
  }
#pragma unroll 8
  for (; x + 4 <= hi; x += 4 * parts) {
    const f32x4u a = *reinterpret_cast<const f32x4u*>(pr + x);
    sum += whole(prob(a[0])) + whole(prob(a[1])) + whole(prob(a[2])) + whole(prob(a[3]));
  }
  for (; x < hi; ++x) sum += whole(prob(pr[x]));
  // (chosen tokens that were rejected: taken off again, each once)
  if (!plain && p.q == nullptr && part < (uint32_t)w.rejected) {
    const uint32_t t = (uint32_t)w.token[part];
    bool once = t >= lo && t < hi;
    for (uint32_t j = 0; j < part; ++j) once = once && (uint32_t)w.token[j] != t;
    if (once) sum -= whole(prob(pr[t]));
  }
  return sum;
}

// Sum over the workgroup, to every thread.
__device__ __forceinline__ uint64_t block_sum(uint64_t x, uint64_t* lds) {
  x = wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  uint64_t s = 0;
#pragma unroll
  for (int w = 0; w < kVerifyWaves; ++w) s += lds[w];
  return s;
}
// Sum of the threads up to this one, and of all.
__device__ __forceinline__ uint64_t block_scan(uint64_t x, uint64_t* lds, uint64_t& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    const uint64_t y = __shfl_up(x, s);
    if (lane >= s) x += y;
  }
  __syncthreads();
  if (lane == 63) lds[wave] = x;
  __syncthreads();
  all = 0;
#pragma unroll
  for (int w = 0; w < kVerifyWaves; ++w) {
    if (w < wave) x += lds[w];
    all += lds[w];
  }
  return x;
}

// The walk of sequence b into w, by the whole workgroup.
__device__ __forceinline__ void walk_tree(const VerifyParams& p, uint32_t b, Walk& w, int& again, uint64_t* lds) {
  const int lane = threadIdx.x & 63;
  const bool first_wave = threadIdx.x < 64, drawn = p.q != nullptr;

  // lane i: node i
  int par = -1, tok = -1;
  float u = 0.f;
  double r = 0.0, q = 0.0;
  bool real = false;  // a token of the vocabulary
  if (first_wave && lane < (int)p.T) {  // (of every node: not to wait for their number)
    const int64_t at = (int64_t)b * p.T + lane;
    par = p.parents ? p.parents[at] : lane - 1;
    if (par >= lane) par = -1;
    tok = p.tokens[at];
    u = p.u[at];
    u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
    real = par >= 0 && tok >= 0 && (uint32_t)tok < p.V;
    if (real) {
      const int64_t e = ((int64_t)b * p.T + par) * p.V + tok;
      r = prob(p.p[e]);
      q = drawn ? prob(p.q[e]) : 1.0;
    }
  }
  int n = p.lengths ? p.lengths[b] : (int)p.T;
  n = max(min(n, (int)p.T), 0);
  real = real && lane < n;
  int cur = n > 0 ? 0 : -1, rejected = 0;
  uint64_t on = n > 0 ? 1 : 0, done = 0;  // accepted nodes; tested ones
  double z = 1.0;
  // Every node's test at once, as it comes out if the siblings before it are rejected.  Where drafts are drawn
  // that holds for first children; where they are chosen a node's z is what they leave.
  const uint64_t valid = __ballot(real);
  uint64_t accept = 0;
  if (first_wave) {
    double mine = 1.0;
    if (!drawn)
      for (uint64_t c = valid; c != 0; c &= c - 1) {
        const int i = __builtin_ctzll(c);
        const bool later = real && lane > i && par == lane_of(par, i);
        if (__ballot(later) == 0) continue;
        const double d = mine - lane_of(r, i);
        if (later) {
          mine = d > 0.0 ? d : 0.0;
          if (tok == lane_of(tok, i)) r = 0.0;
        }
      }
    accept = __ballot(real && test((double)u, mine, q, r));
  }
  for (;;) {
    if (first_wave) {
      again = 0;
      for (;;) {
        const uint64_t open = cur < 0 ? 0 : __ballot(par == cur) & valid & ~done;
        if (open == 0) break;
        if (!drawn) {
          const uint64_t taken = open & accept;
          if (taken == 0) {
            rejected = __builtin_popcountll(open);
            if (open >> lane & 1) w.token[lanes_below(open)] = tok;
            break;
          }
          cur = __builtin_ctzll(taken);
          on |= 1ull << cur;
          continue;
        }
        const int c = __builtin_ctzll(open);
        done |= 1ull << c;
        const bool take = rejected == 0 ? accept >> c & 1
                                        : test(lane_of((double)u, c), z, lane_of(q, c), lane_of(r, c));
        if (take) {
          cur = c;
          on |= 1ull << c;
          rejected = 0;
          z = 1.0;
          continue;
        }
        if (lane == 0) w.z[rejected] = z;
        ++rejected;
        if (par == cur) r = less(r, z, q);
        if ((open & (open - 1)) != 0) {  // a sibling is left: its test needs the sum
          again = 1;
          break;
        }
      }
      if (lane == 0) {
        w.node = cur;
        w.rejected = rejected;
        w.on = on;
      }
    }
    __syncthreads();
    if (!again) break;
    const uint64_t s = block_sum(part_sum(p, w, b, 0, p.V, false, threadIdx.x, kVerifyThreads), lds);
    z = (double)s * kUnfix;
    __syncthreads();  // (`again` and the walk are read before they are written again)
  }
}

// The walk's outputs.
__device__ __forceinline__ void write_path(const VerifyParams& p, uint32_t b, const Walk& w) {
  const int lane = threadIdx.x;
  if (lane >= (int)p.T) return;  // entry i of the path is the i-th node of the walk
  const int64_t at = (int64_t)b * p.T;
  const int count = __builtin_popcountll(w.on);
  if (w.on >> lane & 1) p.path[at + __builtin_popcountll(w.on & ((1ull << lane) - 1))] = lane;
  if (lane >= count) p.path[at + lane] = -1;
  if (lane == 0) p.count[b] = count;
}

__global__ __launch_bounds__(kVerifyThreads) void verify_walk_kernel(VerifyParams p) {
  __shared__ Walk w;
  __shared__ uint64_t lds[kVerifyWaves];
  __shared__ int again;
  const uint32_t b = blockIdx.x / p.slices, slice = blockIdx.x - b * p.slices;
  const int lane = threadIdx.x & 63;
  walk_tree(p, b, w, again, lds);
  if (slice == 0) {
    write_path(p, b, w);
    const int words = sizeof(Walk) / 4;
    for (int x = threadIdx.x; x < words; x += kVerifyThreads)
      reinterpret_cast<uint32_t*>(p.walk + b)[x] = reinterpret_cast<const uint32_t*>(&w)[x];
  }
  if (w.node < 0) return;
  // one sum per wave, each of a quarter of the slice
  const uint32_t quarter = slice * kVerifyWaves + (threadIdx.x >> 6);
  const uint32_t lo = min(quarter * p.per, p.V), hi = min(lo + p.per, p.V);
  const uint64_t s = wave_sum(part_sum(p, w, b, lo, hi, false, lane, 64));
  if (lane == 0) p.sums[(int64_t)b * p.slices * kVerifyWaves + quarter] = s;
}

// The first entry of [lo, hi) of the last node's row whose partial sum from lo on exceeds `place`; `plain`: of
// p[a] itself.  kPerThread consecutive entries per thread.
__device__ __forceinline__ void draw(const VerifyParams& p, const Walk& w, uint32_t b, uint32_t lo, uint32_t hi,
                                     uint64_t place, bool plain, uint64_t* lds) {
  const int64_t row = ((int64_t)b * p.T + w.node) * p.V;
  const bool drawn = p.q != nullptr && w.rejected > 0;
  const float* pr = p.p + row;
  const float* qr = drawn ? p.q + row : pr;
  uint64_t before = 0;
  for (uint32_t x0 = lo; x0 < hi; x0 += kVerifyThreads * kPerThread) {
    const uint32_t x = x0 + threadIdx.x * kPerThread;
    float pe[kPerThread], qe[kPerThread];
    if (x + kPerThread <= p.V) {
#pragma unroll
      for (int e = 0; e < kPerThread; e += 4) {
        const f32x4u a = *reinterpret_cast<const f32x4u*>(pr + x + e), c = *reinterpret_cast<const f32x4u*>(qr + x + e);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          pe[e + i] = a[i];
          qe[e + i] = c[i];
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < kPerThread; ++e) {
        pe[e] = x + e < p.V ? pr[x + e] : 0.f;
        qe[e] = x + e < p.V ? qr[x + e] : 0.f;
      }
    }
    uint64_t r[kPerThread], mine = 0;
    left<kPerThread>(w, drawn && !plain, p.q == nullptr && !plain, pe, qe, x, r);
#pragma unroll
    for (int e = 0; e < kPerThread; ++e) {
      r[e] = x + e < hi ? r[e] : 0;
      mine += r[e];
    }
    uint64_t step;
    const uint64_t upto = before + block_scan(mine, lds, step);
    if (upto > place && upto - mine <= place) {  // one thread
      uint64_t at = upto - mine;
      uint32_t found = x;
#pragma unroll
      for (int e = 0; e < kPerThread; ++e) {
        at += r[e];
        if (at <= place) found = x + e + 1;
      }
      p.next[b] = (int32_t)found;
    }
    before += step;
    if (before > place) break;  // (uniform)
  }
}

// One workgroup per sequence, from what the walk's launch left: the part that the drawn place is in, four sums
// per thread, and the token in it.
__global__ __launch_bounds__(kVerifyThreads) void verify_draw_kernel(VerifyParams p) {
  __shared__ Walk w;
  __shared__ uint64_t lds[kVerifyWaves];
  __shared__ uint64_t place;
  __shared__ uint32_t chosen;
  const uint32_t b = blockIdx.x, tid = threadIdx.x;
  float u = p.u[(int64_t)b * p.T];
  u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
  uint64_t part[kVerifyWaves];
#pragma unroll
  for (int e = 0; e < kVerifyWaves; ++e)
    part[e] = tid < p.slices ? p.sums[((int64_t)b * p.slices + tid) * kVerifyWaves + e] : 0;
  if (tid < sizeof(Walk) / 4) reinterpret_cast<uint32_t*>(&w)[tid] = reinterpret_cast<const uint32_t*>(p.walk + b)[tid];
  static_assert(sizeof(Walk) / 4 <= kVerifyThreads, "one word per thread");
  __syncthreads();
  if (w.node < 0) {
    if (tid == 0) p.next[b] = -1;
    return;
  }
  uint64_t mine = 0, total;
#pragma unroll
  for (int e = 0; e < kVerifyWaves; ++e) mine += part[e];
  const uint64_t upto = block_scan(mine, lds, total);
  uint32_t lo = 0, hi = p.V;
  bool plain = false;
  uint64_t at;
  if (total == 0) {  // nothing is left: of p itself, the whole vocabulary as one part
    plain = true;
    total = block_sum(part_sum(p, w, b, 0, p.V, true, tid, kVerifyThreads), lds);
    if (total == 0) {
      if (tid == 0) p.next[b] = -1;
      return;
    }
    at = (uint64_t)((double)u * (double)total);
  } else {
    at = (uint64_t)((double)u * (double)total);
    if (upto > at && upto - mine <= at) {  // one thread
      at -= upto - mine;
      uint32_t e = 0;
#pragma unroll
      for (int y = 0; y < kVerifyWaves - 1; ++y)
        if (e == (uint32_t)y && at >= part[y]) {
          at -= part[y];
          ++e;
        }
      chosen = tid * kVerifyWaves + e;
      place = at;
    }
    __syncthreads();
    lo = chosen * p.per;
    hi = min(lo + p.per, p.V);
    at = place;
  }
  draw(p, w, b, lo, hi, at, plain, lds);
}

}  // namespace

VerifyPlan verify_plan(int64_t B, int64_t V) {
  // slices of a few thousand entries (four loads in flight per lane), as many as fill the chip four workgroups per CU
  int64_t slices = (V + 4095) / 4096;
  const int64_t fill = 4 * (int64_t)device_cus();
  if (slices * B > fill) slices = fill / B;
  if (slices > kVerifyThreads) slices = kVerifyThreads;
  if (slices < 1) slices = 1;
  VerifyPlan a;
  a.per = ((V + slices * kVerifyWaves - 1) / (slices * kVerifyWaves) + 3) / 4 * 4;
  a.slices = (V + a.per * kVerifyWaves - 1) / (a.per * kVerifyWaves);
  return a;
}

size_t verify_workspace(int64_t B, int64_t T, int64_t V) {
  (void)T;
  const VerifyPlan a = verify_plan(B, V);
  return align256((size_t)B * sizeof(Walk)) + align256((size_t)B * a.slices * kVerifyWaves * sizeof(uint64_t));
}

hipError_t launch_verify(int64_t B, int64_t T, int64_t V, const float* p, const float* q, const int32_t* tokens,
                         const int32_t* parents, const float* u, const int32_t* lengths, int32_t* path, int32_t* count,
                         int32_t* next, void* ws, hipStream_t stream) {
  const VerifyPlan a = verify_plan(B, V);
  VerifyParams k;
  k.p = p;
  k.q = q;
  k.tokens = tokens;
  k.parents = parents;
  k.u = u;
  k.lengths = lengths;
  k.path = path;
  k.count = count;
  k.next = next;
  k.walk = static_cast<Walk*>(ws);
  k.sums = reinterpret_cast<uint64_t*>(static_cast<char*>(ws) + align256((size_t)B * sizeof(Walk)));
  k.T = (uint32_t)T;
  k.slices = (uint32_t)a.slices;
  k.V = (uint32_t)V;
  k.per = (uint32_t)a.per;
  launch_kernel("verify_walk_kernel", verify_walk_kernel, dim3((unsigned)(B * a.slices)), dim3(kVerifyThreads), 0,
                stream, k);
  launch_kernel("verify_draw_kernel", verify_draw_kernel, dim3((unsigned)B), dim3(kVerifyThreads), 0, stream, k);
  return take_launch_error();
}

}  // namespace gca
