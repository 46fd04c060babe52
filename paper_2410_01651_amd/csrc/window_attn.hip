// Attention of the newest tokens over the 8-bit token window (gca_window_attn): single tokens, trees of
// drafted tokens, and prompts.
//
// Mathematics.  K_p = kappa_p N_p and V_p = nu_p M_p with 8-bit numbers N, M and one scale per token.  One
// pass over the tiles of 64 positions that a block of rows sees, with each row's running maximum m and sum
// l:  s = attn_scale kappa_p q N_p^T + slope (p - pos), P = exp(s - m), and out = sum P nu M / l.
// Every e4m3 number and every int8 is exact in bf16 and in fp16.  An e4m3 key takes its scale (a power of
// two) along in the conversion; int8 scores are multiplied by theirs.  So q N^T is a product of exact
// operands with fp32 sums (fp32 queries: three bf16 terms, 24 bits), and P nu / u meets M in fp16,
// 11 bits (fp32 tensors: two fp16 terms, 22 bits), u being a power of two by the largest nu that a row of
// the block has seen so far: P <= 1, so fp16 holds the product, and when a tile brings a larger nu what was
// summed is rescaled with the same factor that a new maximum brings.  (Tokens that none of the block's rows sees, behind
// them, before their windows or on other branches, have no say in u: it may be any number that they bring.)
//
// Layout.  As in the chunk cache's attention: S^T = N Q^T and O^T = M^T P^T on MFMA tiles of W x W, lane
// l = W g + c having query row c as its column, the rows of N in the order that makes a lane's
// accumulators consecutive tokens, so that P is the second product's operand as it stands, and a tile is
// 4 loads of 16 bytes per lane straight into registers.  Scales come one token per lane and are
// handed round through 768 bytes of LDS per wave (keys', values', and which are NaN).
//
// Work.  One item per (sequence, cached head, block of rows); its waves, of one or more workgroups, take the
// tiles in turn and leave (m, l, out) to be joined, by the workgroup through LDS, and for several workgroups by
// the last of them through memory.  No wave waits for another's tile: there is no barrier before the join.
//
// Bound.  Few rows per cached head (single tokens, small trees): HBM, 136 bytes per token and cached head.  One
// token of 64 sequences, 16 heads, a window of 512: 15 us (71.6 MB, 4.8 TB/s); of four sequences of up to 120,000
// tokens, 8 cached heads for 32: 76 us (411 MB, 5.4 TB/s).  Many rows (prompts): instruction issue, of which the
// softmax has most: a tile of 64 x 64 takes 490 vector instructions beside its 32 MFMA (the mean over waves of 220
// tiles).  8,192 tokens of 4 sequences, 16 heads, a window of 512, 9 tiles per wave, two of them masked: 127 us, vector
// pipes busy 69 %, MFMA 24 %.  A tree of 25 nodes over 8 cached heads for 32 heads, 16
// sequences of up to 7,777 tokens: 42 us; four blocks of 32 rows unpack each tile, and vector pipes are busy 33 %.
// One sequence's token of 8 heads over 512: 6 us, the trips to memory (length, tile, parts) one after the other.
#include "gca_device.hpp"
#include "gca_launch.hpp"
#include "numbers8.hpp"
#include "window_plan.hpp"

namespace gca {
namespace {

constexpr int kMaxWaves = 8;
constexpr int kTileBytes = kS * kD;
constexpr float kLowest = -3.402823466e38f;  // of a row that has seen nothing

struct WindowParams {
  uint32_t items;           // workgroups with work
  uint32_t splits, blocks;  // workgroups per row block; row blocks per (sequence, cached head)
  uint32_t nw;              // waves per workgroup
  uint32_t Hkv, G, T, M;    // M = G T: query rows of a group
  uint32_t per_head;        // row blocks per head; 0: the group's rows are one list
  uint32_t H, B;
  uint32_t balance;         // workgroups go by the sequences' lengths
  uint32_t ring_tiles;      // capacity / 64
  int32_t ring, window;
  const int32_t* length;
  const int32_t* parents;
  const int32_t* lengths;
  const float* slopes;
  const uint8_t* k;
  const uint8_t* v;
  const float* ks;
  const float* vs;
  const void* q;
  void* out;
  float* lse;
  float* part;    // partial results of split row blocks: [item][row][64], then [item][row][2]
  float* part_ml;
  int32_t* ticket;  // [row block]: the last workgroup joins the parts; null: window_join_kernel does
  float scale;    // |attn_scale| log2 e (log2 e where attn_scale is 0)
  float unscale;  // 1 / |attn_scale| (1)
  uint32_t negate, keep;  // xor and and masks of one query entry (fp32) or two: the scale's sign, and zero
  int off_by_one;
};

// x of the W lanes of a group joined by f, in every lane of it.
template <int W, typename F>
__device__ __forceinline__ uint32_t fold_rows(uint32_t x, F f) {
  x = f(x, dpp<kDppXor1>(x));
  x = f(x, dpp<kDppXor2>(x));
  x = f(x, dpp<kDppRor4>(x));
  x = f(x, dpp<kDppRor8>(x));
  if constexpr (W == 32) {
    uint32_t a, b;
    pair16(x, a, b);
    x = f(a, b);
  }
  return x;
}

// out = sum_w exp2(m_w - m) o_w / (sum_w exp2(m_w - m) l_w), and the row's log-sum-exp.
struct Joined {
  float m, l;
};
__device__ __forceinline__ Joined finish(float m, float l, int off_by_one) {
  if (off_by_one) {
    const float top = fmaxf(m, 0.f);
    l = l * __builtin_amdgcn_exp2f(m - top) + __builtin_amdgcn_exp2f(-top);
    m = top;
  }
  return Joined{m, l};
}

// Parts of a split row block go through memory that every XCD sees: two floats written and read past the
// caches that each XCD has for itself (agent scope), so that nothing else in those caches is written back or
// dropped: the ticket is drawn once every store of the workgroup has been acknowledged (a wait of each thread,
// then the barrier), and read back after it, by loads that go where the stores went.  With fences of agent
// scope around the ticket instead, four sequences of up to 120,000 tokens take 120 us for 77, 16 sequences' trees of
// 25 nodes 59 for 40.
__device__ __forceinline__ void put2(float* at, float x, float y) {
  const uint64_t u = (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x);
  __hip_atomic_store(reinterpret_cast<uint64_t*>(at), u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 get2(const float* at) {
  const uint64_t u = __hip_atomic_load(reinterpret_cast<const uint64_t*>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return f32x2{__uint_as_float((uint32_t)u), __uint_as_float((uint32_t)(u >> 32))};
}

// Joins parts first .. first + n - 1 of a row block: columns 4 x .. of its row m, row r of the output.
template <typename T, int QB, uint32_t kAhead>  // kAhead: parts asked for at a time
__device__ __forceinline__ void join_rows_by(const WindowParams& p, uint32_t first, uint32_t n, uint32_t m, uint32_t x,
                                             int64_t r) {
  float top = kLowest, l = 0.f;
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
  for (uint32_t s0 = 0; s0 < n; s0 += kAhead) {
    f32x2 ml[kAhead], a[kAhead], c[kAhead];
#pragma unroll
    for (uint32_t s = 0; s < kAhead; ++s) {
      const int64_t at = ((int64_t)first + min(s0 + s, n - 1)) * QB + m;
      ml[s] = get2(p.part_ml + at * 2);
      a[s] = get2(p.part + at * kD + 4 * x);
      c[s] = get2(p.part + at * kD + 4 * x + 2);
    }
    float now = top;
#pragma unroll
    for (uint32_t s = 0; s < kAhead; ++s) now = fmaxf(now, ml[s][0]);  // (the last part's again does no harm)
    const float shrink = __builtin_amdgcn_exp2f(top - now);
    l *= shrink;
    acc *= shrink;
    top = now;
#pragma unroll
    for (uint32_t s = 0; s < kAhead; ++s) {
      if (s0 + s >= n || ml[s][1] == 0.f) continue;
      const float f = __builtin_amdgcn_exp2f(ml[s][0] - top);
      l = fmaf(ml[s][1], f, l);
      acc += f32x4{a[s][0], a[s][1], c[s][0], c[s][1]} * f;
    }
  }
  const Joined j = finish(top, l, p.off_by_one);
  const float f = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(top - j.m) / j.l;
  store4(reinterpret_cast<T*>(p.out) + r * kD + 4 * x, acc[0] * f, acc[1] * f, acc[2] * f, acc[3] * f);
  if (p.lse && x == 0) p.lse[r] = l == 0.f ? -INFINITY : (j.m + __builtin_amdgcn_logf(j.l)) * kLn2;
}

template <typename T, int QB>
__device__ __forceinline__ void join_rows(const WindowParams& p, uint32_t first, uint32_t n, uint32_t m, uint32_t x,
                                          int64_t r) {
  if (n <= 4) join_rows_by<T, QB, 2>(p, first, n, m, x, r);
  else join_rows_by<T, QB, 8>(p, first, n, m, x, r);
}

// T: type of the queries; W: MFMA tile; NC: column blocks of W query rows; TREE: the new tokens are a tree.
template <typename T, bool I8, int W, int NC, bool TREE>
__global__ __launch_bounds__(kMaxWaves * 64, 2) void window_attn_kernel(WindowParams p) {
  constexpr bool kB16 = sizeof(T) == 2;
  constexpr int NG = 64 / W;           // lane groups
  constexpr int NA = 64 / W;           // blocks of W tokens (or columns) per tile
  constexpr int NK = W / 8;            // steps of the contraction over 64 columns (or tokens)
  constexpr int NX = NK / 2;           // 16-byte pieces per lane and block
  constexpr int NR = W * W / 64;       // accumulators per block
  constexpr int NV = NA * NR;          // values per lane and column block
  constexpr int QP = kB16 ? 1 : 3;     // bf16 terms of a query entry
  constexpr int PP = kB16 ? 1 : 2;     // fp16 terms of a probability
  constexpr int QB = W * NC;           // query rows per item
  // Values take their scales along where two column blocks share them; else the probabilities do, which are then
  // fewer.  2^-9 M nu 2^15 / u is below 2^15 and, M having four bits and nu being a power of two, exact in fp16 down
  // to nu = 2^-20 of the largest; below that it is off by 2^-25 at most, a value by 2^-31 u.
  constexpr bool VS = NC == 2;
  static_assert(NC == 1 || (kB16 && !I8), "64 rows: e4m3 numbers, bf16 tensors");
  typedef __attribute__((ext_vector_type(NR))) float Acc;
  extern __shared__ __attribute__((aligned(16))) float smem[];

  const uint32_t tid = __builtin_amdgcn_workitem_id_x(), nw = p.nw;
  const int lane = tid & 63, g = lane / W, col = lane % W;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  auto scalar = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane(x); };
  // item = ((b Hkv + h) blocks + block) splits + split, unless the sequences' lengths have a say
  uint32_t b, h, blk, split, splits = p.splits, it;
  int bare = -1;  // blocks from here on (of each head, cut head by head) have no tokens; -1: not this one's to write
  if (p.balance) {
    // A head's B blocks splits workgroups are dealt out by what its sequences have to do: one to each block that
    // has tokens, the others in proportion to the block's tiles.  Lane i: sequence i.
    it = (uint32_t)xcd_swizzle(__builtin_amdgcn_workgroup_id_x(), (p.items + 7) / 8 * 8);
    if (it >= p.items) return;
    const uint32_t all = p.B * p.blocks * p.splits;
    h = scalar(it / all);
    const uint32_t j = it - h * all, seq = min((uint32_t)lane, p.B - 1);
    const int len = p.length[seq];
    const uint32_t tok = p.lengths ? (uint32_t)max(min(p.lengths[seq], (int)p.T), 0) : p.T;
    const uint32_t mine = (uint32_t)lane < p.B ? 1 : 0;
    const uint32_t tiles = mine * min(((uint32_t)max(len, 1) + kS - 1) / kS, p.ring_tiles);
    // (the first block is there also without tokens: for the rows)
    const uint32_t with = mine * max(p.per_head ? p.G * ((tok + QB - 1) / QB) : (p.G * tok + QB - 1) / QB, 1u);
    auto sum_upto = [&](uint32_t x) {
#pragma unroll
      for (int s = 1; s < 64; s *= 2) {
        const uint32_t y = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (lane - s), (int)x);
        x += lane >= s ? y : 0;
      }
      return x;
    };
    const uint32_t one = scalar((uint32_t)__builtin_amdgcn_readlane((int)sum_upto(with), 63));
    const uint32_t work = scalar((uint32_t)__builtin_amdgcn_readlane((int)sum_upto(with * tiles), 63));
    const uint32_t each = 1 + (all - one) * tiles / work;  // (below 2^11 times 2^18)
    const uint32_t to = sum_upto(with * each), from = to - with * each;
    b = __builtin_popcountll(__ballot(mine && from <= j)) - 1;
    auto of = [&](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, (int)b); };
    if (j >= of(to)) return;
    splits = of(each);
    const uint32_t i = j - of(from);
    blk = scalar(i / splits);
    split = i - blk * splits;
    const uint32_t there = of(with), per = p.per_head ? max(scalar(there / p.G), 1u) : there;
    if (p.per_head) {  // (the blocks with tokens come first in each head)
      const uint32_t gh = scalar(blk / per);
      blk = gh * p.per_head + (blk - gh * per);
    }
    if (i == 0) bare = of(tok) > 0 ? (int)per : 0;
  } else {
    it = (uint32_t)xcd_swizzle(__builtin_amdgcn_workgroup_id_x(), (p.items + 7) / 8 * 8);
    if (it >= p.items) return;
    const uint32_t at = scalar(it / splits);
    split = it - at * splits;
    const uint32_t bhs = scalar(at / p.blocks);
    blk = at - bhs * p.blocks;
    b = scalar(bhs / p.Hkv);
    h = bhs - b * p.Hkv;
  }
  const uint32_t bh = b * p.Hkv + h, bb = bh * p.blocks + blk;

  const int length = max((int)scalar((uint32_t)p.length[b]), 0);
  int n = p.lengths ? (int)scalar((uint32_t)p.lengths[b]) : (int)p.T;
  n = max(min(n, (int)p.T), 0);
  const int base = length - n;  // (negative only if fewer tokens were appended than `lengths` says)

  // ---- the block's rows [m0, m0 + nrows), and the new tokens [tmin, tmax] they belong to.  Rows are cut
  // head by head, or, short of a block per head, a group's rows with tokens as one list and those without behind it.
  const uint32_t live = p.G * (uint32_t)n;
  uint32_t m0, nrows, tmin, tmax;
  if (p.per_head) {
    const uint32_t gh = scalar(blk / p.per_head);
    tmin = (blk - gh * p.per_head) * QB;
    nrows = min((uint32_t)QB, p.T - tmin);
    tmax = tmin + nrows - 1;
    m0 = gh * p.T + tmin;
  } else {
    m0 = blk * QB;
    nrows = min((uint32_t)QB, p.M - m0);
    tmin = (uint32_t)n;
    tmax = p.T - 1;
    if (m0 < live) {
      const uint32_t end = min(m0 + nrows, live) - 1, f = scalar(m0 / (uint32_t)n), l = scalar(end / (uint32_t)n);
      tmin = f == l ? m0 - f * n : 0;
      tmax = f == l ? end - f * n : n - 1;
    }
  }
  // head of the group and token of row m of the block
  auto place = [&](uint32_t m, uint32_t& gh, uint32_t& t) {
    m += m0;
    const bool behind = !p.per_head && m >= live;
    const uint32_t per = p.per_head ? p.T : behind ? p.T - (uint32_t)n : (uint32_t)n;
    m -= behind ? live : 0u;
    gh = m / per;
    t = m - gh * per + (behind ? (uint32_t)n : 0u);
  };

  const int64_t row0 = (int64_t)(b * p.H + h * p.G) * p.T;
  if (bare >= 0) {  // (rows that nobody else gets to)
    const uint32_t heads = p.per_head ? p.G : 1, from = (uint32_t)bare * QB, rows = p.per_head ? p.T : p.M;
    for (uint32_t gh = 0; gh < heads; ++gh)
      for (uint32_t e = tid; from < rows && e < (rows - from) * 16; e += 64 * nw) {
        uint32_t g_, t_, m = from + (e >> 4);
        if (p.per_head) {
          g_ = gh;
          t_ = m;
        } else {
          place(m - m0, g_, t_);
        }
        const int64_t r = row0 + (int64_t)g_ * p.T + t_;
        store4(reinterpret_cast<T*>(p.out) + r * kD + 4 * (e & 15), 0.f, 0.f, 0.f, 0.f);
        if (p.lse && (e & 15) == 0) p.lse[r] = -INFINITY;
      }
  }

  // ---- the tree: lane i holds node i's ancestors and itself as bits
  uint64_t up = 0;
  if constexpr (TREE) {
    const int i = lane;
    int par = p.parents[(int64_t)b * p.T + min((uint32_t)i, p.T - 1)];
    par = par >= 0 && par < i ? par : i;
    uint32_t lo = i < 32 ? 1u << i : 0u, hi = i < 32 ? 0u : 1u << (i - 32);
#pragma unroll
    for (int s = 0; s < 6; ++s) {  // 2^s levels at a time
      lo |= (uint32_t)__builtin_amdgcn_ds_bpermute(4 * par, (int)lo);
      hi |= (uint32_t)__builtin_amdgcn_ds_bpermute(4 * par, (int)hi);
      par = __builtin_amdgcn_ds_bpermute(4 * par, par);
    }
    up = (uint64_t)hi << 32 | lo;
  }

  // ---- this lane's rows
  uint32_t row[NC];    // of the group
  int depth[NC];       // position - base
  float slope[NC];     // in units of a score before its scale
  auto token = [&](int c) {  // (a node's is formed again where it is wanted, to have the registers)
    if constexpr (!TREE) return depth[c];
    uint32_t gh, t;
    place(min((uint32_t)opaque(c * W + col), nrows - 1), gh, t);
    return (int)t;
  };
  // a node's ancestors and itself
  auto above = [&](int i) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * i, (int)(uint32_t)up);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * i, (int)(uint32_t)(up >> 32));
    return (uint64_t)hi << 32 | lo;
  };
  // of a node's ancestors and itself those that it sees: less than `window` levels up
  auto near = [&](uint64_t sees, int deep) {
    if (p.window)
      for (int x = deep - p.window; x >= 0; --x) sees &= sees - 1;
    return sees;
  };
  uint32_t seen_lo = 0, seen_hi = 0, dlow = kTreeNodes;  // of a tree: the nodes that the block's rows see, and their least depth
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    uint32_t gh, t;
    place(min((uint32_t)(c * W + col), nrows - 1), gh, t);
    row[c] = gh * p.T + t;
    depth[c] = (int)t;
    if constexpr (TREE) {
      const uint64_t sees = above((int)t);
      depth[c] = __builtin_popcountll(sees) - 1;
      const uint64_t mine = (int)t < n ? near(sees, depth[c]) : 0ull;
      seen_lo |= (uint32_t)mine;
      seen_hi |= (uint32_t)(mine >> 32);
      dlow = min(dlow, (int)t < n ? (uint32_t)depth[c] : (uint32_t)kTreeNodes);
    }
    slope[c] = p.slopes ? p.slopes[h * p.G + gh] * p.unscale : 0.f;
  }
  uint64_t nodes = 0;
  if constexpr (TREE) {
    seen_lo = fold_rows<W>(seen_lo, [](uint32_t x, uint32_t y) { return x | y; });
    seen_hi = fold_rows<W>(seen_hi, [](uint32_t x, uint32_t y) { return x | y; });
    dlow = fold_rows<W>(dlow, [](uint32_t x, uint32_t y) { return min(x, y); });
    nodes = (uint64_t)scalar(seen_hi) << 32 | scalar(seen_lo);
    dlow = scalar(dlow);
  }

  // ---- tiles of 64 positions that the rows see: [t0, t1)
  const int dmin = TREE ? (int)dlow : (int)tmin, dmax = TREE ? kTreeNodes - 1 : (int)tmax;
  const int first = p.window ? max(base + dmin - p.window + 1, 0) : 0;
  const int last = base + min((int)tmax, n - 1);  // position (a node sees none behind its own)
  const int t0 = first >> 6;
  int t1 = (last >> 6) + 1;
  if (!p.ring) t1 = min(t1, (int)p.ring_tiles);
  if ((int)tmin >= n) t1 = t0;
  // every row sees the whole of a tile within [full0, full1]
  const int full0 = p.window ? base + dmax - p.window + 1 : 0;
  const int full1 = TREE ? base - 1 : base + (int)tmin;
  const uint32_t workers = splits * nw, me = split * nw + wave;

  const uint32_t lane_row = W == 32 ? 16 * ((col >> 2) & 1) + 4 * (col >> 3) + (col & 3)
                                    : 16 * (col >> 2) + (col & 3);
  const uint32_t lane_off = lane_row * kD + 16 * g;
  const int64_t head_tiles = (int64_t)bh * p.ring_tiles;
  // (`there` false: nothing is wanted and the descriptor is empty; the loads are issued either way, so that
  // what is in flight at a wait is known)
  auto slot = [&](int t) { return p.ring ? scalar((uint32_t)t % p.ring_tiles) : (uint32_t)t; };
  auto load_tile = [&](u32x4* x, const uint8_t* from, uint32_t s, bool there) {
    const __amdgpu_buffer_rsrc_t tile =
        range_rsrc(reinterpret_cast<const char*>(from) + (head_tiles + s) * kTileBytes, there ? kTileBytes : 0);
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
      for (int y = 0; y < NX; ++y)
        x[a * NX + y] = __builtin_amdgcn_raw_buffer_load_b128(
            tile, lane_off, (W == 32 ? 32 : 4) * a * kD + 16 * NG * y, 0);
  };
  auto load_scale = [&](const float* from, uint32_t s, bool there) {
    return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(
        range_rsrc(reinterpret_cast<const char*>(from + (head_tiles + s) * kS), there ? kS * 4 : 0), lane * 4, 0, 0));
  };

  int t = t1 - 1 - (int)me;  // (from the newest on: with biases the maximum is there, and stays)
  u32x4 kr[NA * NX], vr[NA * NX];
  float ksc, vsc;
  {
    const bool there = t >= t0;
    const uint32_t s = there ? slot(t) : 0;
    load_tile(kr, p.k, s, there);
    ksc = load_scale(p.ks, s, there);
    vsc = load_scale(p.vs, s, there);
    load_tile(vr, p.v, s, there);
  }

  // ---- the queries: lane (g, c) takes columns 16 (g + NG x) .. of row c, x < NX
  bf16x8 qf[NC][NK][QP];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const auto* qr = scalar_ptr(reinterpret_cast<const T*>(p.q) + row0 * kD) + (int64_t)row[c] * kD;
#pragma unroll
    for (int s = 0; s < NK; ++s) {
      const auto* src = qr + 16 * (g + NG * (s >> 1)) + 8 * (s & 1);
      if constexpr (kB16) {
        u32x4 x = *reinterpret_cast<const __attribute__((address_space(1))) u32x4*>(src);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (x[e] ^ p.negate) & p.keep;
        qf[c][s][0] = __builtin_bit_cast(bf16x8, x);
      } else {
#pragma unroll
        for (int m8 = 0; m8 < 8; ++m8) {
          float x = src[m8];
          x = __uint_as_float((__float_as_uint(x) ^ p.negate) & p.keep);
#pragma unroll
          for (int e = 0; e < QP; ++e) {
            const __bf16 part = (__bf16)x;
            qf[c][s][e][m8] = part;
            x -= (float)part;
          }
        }
      }
    }
  }

  float* const sc_lds = smem + wave * 192;  // this wave's scales: 64 of keys, 64 of values; what is NaN
  Acc o[NC][NA];
  float mx[NC], sum[NC];
  int octave = -1000;  // of u
  float limit = 0.f;   // 2^octave
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    mx[c] = kLowest;
    sum[c] = 0.f;
#pragma unroll
    for (int a = 0; a < NA; ++a) o[c][a] = Acc{};
  }

  for (; t >= t0; t -= (int)workers) {
    const int p0 = t << 6;  // the tile's first position
    const int tn = t - (int)workers;
    const bool more = tn >= t0;
    const uint32_t sn = more ? slot(tn) : 0;

    // scales, those of values over u: tokens that no row of the block sees have none
    const int from = first - p0, to = length - p0;  // what there is of the tile
    bool here = lane >= from && lane <= last - p0;
    if (TREE && p0 + kS > base) {
      const int node = p0 + lane - base;
      here = here && (node < 0 || (nodes >> (node & 63) & 1) != 0);
    }
    const float nu = here ? vsc : 0.f;
    int up_by = 0;  // octaves that u grows by
    if (__ballot(nu > limit) != 0) {
      const int e = __builtin_amdgcn_readfirstlane(__builtin_amdgcn_frexp_expf(max64(nu)));
      up_by = octave == -1000 ? 0 : e - octave;
      octave = e;
      limit = __builtin_ldexpf(1.f, e);
    }
    wave_lds_order();
    sc_lds[lane] = ksc;
    const float nu15 = __builtin_ldexpf(nu, 15 - octave);  // at most 2^15
    // values whose scale is NaN: none here, their tokens' probabilities become NaN in the rows that see them
    const uint64_t bad = __ballot((__float_as_uint(nu) & 0x7fffffffu) > 0x7f800000u);
    const float mine = bad >> lane & 1 ? 0.f : nu15;
    if constexpr (VS) reinterpret_cast<_Float16*>(sc_lds + 64)[lane] = (_Float16)mine;
    else sc_lds[64 + lane] = mine;
    wave_lds_order();

    // S^T = N Q^T
    Acc st[NC][NA];
#pragma unroll
    for (int a = 0; a < NA; ++a) {
#pragma unroll
      for (int c = 0; c < NC; ++c) st[c][a] = Acc{};
      float kappa = 1.f;
      if constexpr (!I8) kappa = sc_lds[lane_row + (W == 32 ? 32 : 4) * a];
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        const u32x4 r = kr[a * NX + (i >> 1)];
        bf16x8 f;
        if constexpr (I8) f = to_bf16<true>(r[2 * (i & 1)], r[2 * (i & 1) + 1]);
        else f = to_bf16_times(r[2 * (i & 1)], r[2 * (i & 1) + 1], kappa);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < QP; ++e) st[c][a] = mma(f, qf[c][i][e], st[c][a]);
      }
    }
    // (the next keys: with two column blocks behind the first one's softmax, which leaves their registers)
    auto next_keys = [&] {
      load_tile(kr, p.k, sn, more);
      ksc = load_scale(p.ks, sn, more);
      vsc = load_scale(p.vs, sn, more);
    };
    if constexpr (NC == 1) next_keys();

    const bool masked = p0 < full0 || p0 + kS - 1 > full1;
    f16x8 pf[NC][NK][PP];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float v[NV];
#pragma unroll
      for (int u = 0; u < NV; ++u) v[u] = st[c][u / NR][u % NR];
      // value u is token tok(u) + 16 g of the tile
      auto tok = [](int u) { return W == 32 ? 32 * (u / 16) + u % 16 : u; };
      if constexpr (I8) {
#pragma unroll
        for (int u = 0; u < NV; u += 4) {
          const f32x4 s4 = *reinterpret_cast<const f32x4*>(sc_lds + 16 * g + tok(u));
#pragma unroll
          for (int e = 0; e < 4; ++e) v[u + e] *= s4[e];
        }
      }
      // tokens of the tile that the row sees: first .. last of them in a chain, in a tree bits
      const int lo = (p.window ? max(base + depth[c] - p.window + 1 - p0, 0) : 0) - 16 * g;
      const int hi = min(base + depth[c] - p0, to - 1) - 16 * g;
      uint64_t bits = ~0ull;
      if (TREE && masked) {
        const int off = base - p0;  // the first new token
        bits = off >= 64 ? ~0ull : off > 0 ? (1ull << off) - 1 : 0ull;
        const uint64_t sees = near(above(token(c)), depth[c]);
        if (p.window) {
          const int l = lo + 16 * g;
          bits = l < 64 ? bits & (~0ull << l) : 0ull;
        }
        if (off < 64) bits |= off >= 0 ? sees << off : off > -64 ? sees >> -off : 0ull;
        if (to < 64) bits &= to > 0 ? (1ull << to) - 1 : 0ull;
        bits >>= 16 * g;
      }
      if (bad != 0) {  // NaN for the rows that see it (the others are masked behind)
        wave_lds_order();
        reinterpret_cast<uint32_t*>(sc_lds + 128)[lane] = bad >> lane & 1 ? 0x7fc00000u : 0u;
        wave_lds_order();
#pragma unroll
        for (int u = 0; u < NV; u += 4) {
          const f32x4 s4 = *reinterpret_cast<const f32x4*>(sc_lds + 128 + 16 * g + tok(u));
#pragma unroll
          for (int e = 0; e < 4; ++e) v[u + e] += s4[e];
        }
      }
      if (p.slopes) {
        // relative to the tile's first token; its own place joins the maximum below
#pragma unroll
        for (int u = 0; u < NV; ++u) v[u] = fmaf(slope[c], (float)tok(u), v[u]);
        if (TREE && p0 + kS > base) {  // a node's position is its depth's, not its place's
          const uint64_t ups = above(token(c));
#pragma unroll
          for (int u = 0; u < NV; ++u) {
            const int a = p0 + 16 * g + tok(u) - base;
            if (a > 0 && a < 64) {
              const int d = __builtin_popcountll(ups & ((1ull << a) - 1));
              v[u] = fmaf(slope[c], (float)(d - a), v[u]);
            }
          }
        }
      }
      if constexpr (TREE) {
        if (masked) {
#pragma unroll
          for (int u = 0; u < NV; ++u)
            if (!(bits >> tok(u) & 1)) v[u] = -INFINITY;
        }
      } else {
        if (p0 < full0) {
          const int x = opaque(lo);
#pragma unroll
          for (int u = 0; u < NV; ++u)
            if (tok(u) < x) v[u] = -INFINITY;
        }
        if (p0 + kS - 1 > full1) {
          const int x = opaque(hi);
#pragma unroll
          for (int u = 0; u < NV; ++u)
            if (tok(u) > x) v[u] = -INFINITY;
        }
      }
      float top = fmaxf(fmaxf(v[0], v[1]), v[2]), top2 = fmaxf(fmaxf(v[3], v[4]), v[5]);
#pragma unroll
      for (int u = 6; u + 3 < NV; u += 4) {
        top = fmaxf(fmaxf(top, v[u]), v[u + 1]);
        top2 = fmaxf(fmaxf(top2, v[u + 2]), v[u + 3]);
      }
      top = fmaxf(fmaxf(top, v[NV - 2]), fmaxf(top2, v[NV - 1]));
      // where this lane's tokens begin, from the row
      const float at = slope[c] * (float)(p0 + 16 * g - base - depth[c]);
      top += at;
      if constexpr (W == 16) {
        uint32_t x, y;
        pair16(__float_as_uint(top), x, y);
        top = fmaxf(__uint_as_float(x), __uint_as_float(y));
      }
      top = fmaxf(max_xor32(top) * p.scale, mx[c]);
      const float shrink = __builtin_amdgcn_exp2f(mx[c] - top);
      mx[c] = top;
      const float sub = at * p.scale - top + (VS ? 15.f : 0.f);  // (VS: P up to 2^15)
#pragma unroll
      for (int u = 0; u < NV; ++u) v[u] = __builtin_amdgcn_exp2f(fmaf(v[u], p.scale, sub));
      float add = v[0], add2 = v[1];
#pragma unroll
      for (int u = 2; u < NV; u += 2) {
        add += v[u];
        add2 += v[u + 1];
      }
      sum[c] = fmaf(sum[c], shrink, add + add2);
      const float both = up_by == 0 ? shrink : __builtin_ldexpf(shrink, -up_by);
      if (__ballot(both != 1.f) != 0) {
#pragma unroll
        for (int a = 0; a < NA; ++a)
#pragma unroll
          for (int r = 0; r < NR; ++r) o[c][a][r] *= both;
      }
      if constexpr (VS) {
#pragma unroll
        for (int u = 0; u < NV; ++u) pf[c][u / 8][0][u % 8] = (_Float16)v[u];
      } else {
#pragma unroll
        for (int u = 0; u < NV; u += 4) {
          const f32x4 s4 = *reinterpret_cast<const f32x4*>(sc_lds + 64 + 16 * g + tok(u));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = v[u + e] * s4[e];
            if constexpr (PP == 2) asm("" : "+v"(x));  // (one rounding of x for both terms)
            const int i = (u + e) / 8, m = (u + e) % 8;
            const _Float16 hi = (_Float16)x;
            pf[c][i][0][m] = hi;
            if constexpr (PP == 2) pf[c][i][PP - 1][m] = (_Float16)(x - (float)hi);
          }
        }
      }
      if (NC > 1 && c == 0) next_keys();
    }

    // O^T += M^T P^T (numbers behind the newest token are cleared: they may be anything)
    if (to < kS) {
      const int left0 = opaque(to - 16 * g);
#pragma unroll
      for (int y = 0; y < NX; ++y)
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const int left = left0 - (16 * NG * y + 4 * d);
          const uint32_t only = left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
#pragma unroll
          for (int a = 0; a < NA; ++a) vr[a * NX + y][d] &= only;
        }
    }
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        const u32x4 r = vr[a * NX + (i >> 1)];
        f16x8 f;
        if constexpr (VS)
          f = to_f16_small(r[2 * (i & 1)], r[2 * (i & 1) + 1]) *
              *reinterpret_cast<const f16x8*>(reinterpret_cast<const _Float16*>(sc_lds + 64) + 16 * g +
                                              32 * (i >> 1) + 8 * (i & 1));
        else
          f = to_f16<I8>(r[2 * (i & 1)], r[2 * (i & 1) + 1]);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < PP; ++e) o[c][a] = mma(f, pf[c][i][e], o[c][a]);
      }
    load_tile(vr, p.v, sn, more);
  }

  // ---- output: value u of a lane is column 32 (u / 16) + 16 g + u % 16 (W = 32) or 16 g + u
  const int back = octave == -1000 ? 0 : octave - 15 + (VS ? 9 - 15 : 0);
#pragma unroll
  for (int c = 0; c < NC; ++c) {  // the groups' shares of the sums
    if constexpr (W == 16) {
      uint32_t x, y;
      pair16(__float_as_uint(sum[c]), x, y);
      sum[c] = __uint_as_float(x) + __uint_as_float(y);
    }
    sum[c] = sum_xor32(sum[c]) * (VS ? 0x1p-15f : 1.f);
  }
  T* const out0 = (T*)scalar_ptr(reinterpret_cast<T*>(p.out) + row0 * kD);
  auto row_of = [&](uint32_t m) {  // row m of the block, among the group's
    uint32_t gh, t;
    place(m, gh, t);
    return (int64_t)(gh * p.T + t);
  };
  if (NC == 2 || workers == 1) {  // (64 rows: always a wave each)
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const uint32_t m = c * W + col;
      if (m >= nrows) continue;
      const Joined j = finish(mx[c], sum[c], p.off_by_one);
      const bool none = token(c) >= n || sum[c] == 0.f;
      // (off by one: the row's own scale between its maximum and the denominator's)
      const float f = none ? 0.f : __builtin_amdgcn_exp2f(mx[c] - j.m) / j.l;
      const int64_t r = row_of(m);
      T* dst = out0 + r * kD + 16 * g;
#pragma unroll
      for (int u = 0; u < NV; u += 8) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
          x[e] = none ? 0.f : __builtin_ldexpf(o[c][(u + e) / NR][(u + e) % NR] * f, back);
        store8(dst + (u / 16) * 32 + u % 16, x);
      }
      if (p.lse && g == 0)
        p.lse[row0 + r] = none ? -INFINITY : (j.m + __builtin_amdgcn_logf(j.l)) * kLn2;
    }
    return;
  }
  // the waves' parts: part[wave][row][16 blocks of 4], block x of row r at x ^ (r mod 16); then m and l
  __syncthreads();
  float* const part = smem;
  float* const ml = smem + nw * nrows * kD;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const uint32_t m = c * W + col;
    if (m >= nrows) continue;
    float* pr = part + (wave * nrows + m) * kD;
#pragma unroll
    for (int u = 0; u < NV; u += 4) {
      const Acc& a = o[c][u / NR];
      const uint32_t x = (4 * g + (u / 16) * 8 + (u % 16) / 4) ^ (m & 15);
      *reinterpret_cast<f32x4*>(pr + 4 * x) =
          f32x4{__builtin_ldexpf(a[u % NR], back), __builtin_ldexpf(a[u % NR + 1], back),
                __builtin_ldexpf(a[u % NR + 2], back), __builtin_ldexpf(a[u % NR + 3], back)};
    }
    if (g == 0) {
      ml[2 * (wave * nrows + m)] = token(c) < n ? mx[c] : kLowest;
      ml[2 * (wave * nrows + m) + 1] = token(c) < n ? sum[c] : 0.f;
    }
  }
  __syncthreads();
  for (uint32_t e = tid; e < nrows * 16; e += 64 * nw) {
    const uint32_t m = e >> 4, x = e & 15;
    float top = kLowest;
    for (uint32_t y = 0; y < nw; ++y) top = fmaxf(top, ml[2 * (y * nrows + m)]);
    f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
    for (uint32_t y = 0; y < nw; ++y) {
      const float ly = ml[2 * (y * nrows + m) + 1];
      if (ly == 0.f) continue;
      const float f = __builtin_amdgcn_exp2f(ml[2 * (y * nrows + m)] - top);
      l = fmaf(ly, f, l);
      const f32x4 oy = *reinterpret_cast<const f32x4*>(part + (y * nrows + m) * kD + 4 * (x ^ (m & 15)));
      acc += oy * f;
    }
    if (splits > 1) {
      const int64_t at = (int64_t)it * QB + m;
      put2(p.part + at * kD + 4 * x, acc[0], acc[1]);
      put2(p.part + at * kD + 4 * x + 2, acc[2], acc[3]);
      if (x == 0) put2(p.part_ml + at * 2, top, l);
    } else {
      const Joined j = finish(top, l, p.off_by_one);
      const float f = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(top - j.m) / j.l;
      const int64_t r = row_of(m);
      store4(out0 + r * kD + 4 * x, acc[0] * f, acc[1] * f, acc[2] * f, acc[3] * f);
      if (p.lse && x == 0)
        p.lse[row0 + r] = l == 0.f ? -INFINITY : (j.m + __builtin_amdgcn_logf(j.l)) * kLn2;
    }
  }
  if (splits == 1 || !p.ticket) return;
  // the last workgroup of the block to get here joins its parts
  wait_tiles<0>();  // (this thread's part is where every XCD sees it)
  __syncthreads();
  uint32_t* const drawn = reinterpret_cast<uint32_t*>(smem);
  if (tid == 0)
    *drawn = (uint32_t)__hip_atomic_fetch_add(p.ticket + bb, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (*drawn != splits - 1) return;
  if (tid == 0) __hip_atomic_store(p.ticket + bb, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  for (uint32_t e = tid; e < nrows * 16; e += 64 * nw)
    join_rows<T, QB>(p, it - split, splits, e >> 4, e & 15, row0 + row_of(e >> 4));
}

// The same in a launch of its own, where a window has no tickets for so many row blocks: more than two per
// head, which only rows cut head by head come to (p.per_head > 0; as lists a group's rows make at most a block per
// head).  16 threads per row.
template <typename T, int QB>
__global__ __launch_bounds__(256) void window_join_kernel(WindowParams p) {
  const uint32_t e = __builtin_amdgcn_workgroup_id_x() * 256 + __builtin_amdgcn_workitem_id_x();
  const uint32_t x = e & 15, m = (e >> 4) % QB, bb = (e >> 4) / QB;
  const uint32_t bh = bb / p.blocks, blk = bb - bh * p.blocks;
  if (bb >= p.items / p.splits) return;
  const uint32_t gh = blk / p.per_head, tmin = (blk - gh * p.per_head) * QB;
  const uint32_t b = bh / p.Hkv, h = bh - b * p.Hkv;
  if (m < min((uint32_t)QB, p.T - tmin))
    join_rows<T, QB>(p, bb * p.splits, p.splits, m, x,
                     (int64_t)(b * p.H + h * p.G) * p.T + gh * p.T + tmin + m);
}

}  // namespace

namespace {
// Waves that a launch is cut into where its row blocks are fewer.  8 / 16 / 32 per CU: 64 sequences' single tokens
// 15.1 / 16.0 / 18.2 us, four long sequences' 79 / 82 / 85, trees of 25 nodes 54 / 67 / 82: each wave has two
// tiles on their way, and more waves are more parts to join.
constexpr int kWavesPerCu = 8;
// 64 rows unpack a tile for twice the rows, but leave two waves per SIMD: where such blocks, a wave each, fill
// the chip.  64 / 32 rows there: a prompt of 8,192 tokens 126 / 141 us.  Short of that: the tree of 25 nodes
// 55 / 52, one of 10 nodes 37 / 32, 64 tokens of two sequences 13.8 / 8.1.  int8, whose numbers have no scaled
// conversion, would spill: prompt 315 / 175, tree 95 / 66.
int rows_of(const gca_window& w, int64_t T) {
  const int64_t G = w.H / w.Hkv, M = G * T, blocks = T >= 64 ? G * ((T + 63) / 64) : (M + 63) / 64;
  if (M <= 16) return 16;
  const bool can = w.dtype == GCA_BF16 && w.format == GCA_E4M3;
  return can && (int64_t)w.B * w.Hkv * blocks >= kWavesPerCu * device_cus() ? 64 : 32;
}
// Tiles that a row block may see.
int64_t tiles_seen(const gca_window& w, int64_t T, int rows) {
  const int64_t all = w.capacity / 64, some = tiles_of(w.window + (T < rows ? T : rows) - 1);
  return w.window && some < all ? some : all;
}
}  // namespace

WindowAttnPlan window_attn_plan(const gca_window& w, int64_t T) {
  WindowAttnPlan a;
  const int64_t G = w.H / w.Hkv, M = G * T;
  a.rows = rows_of(w, T);
  a.per_head = T >= a.rows ? (T + a.rows - 1) / a.rows : 0;
  a.blocks = a.per_head ? G * a.per_head : (M + a.rows - 1) / a.rows;
  a.groups = (int64_t)w.B * w.Hkv * a.blocks;
  const int64_t tiles = tiles_seen(w, T, a.rows), fill = kWavesPerCu * device_cus();
  a.waves = 1;
  while (a.waves < kMaxWaves && 2 * a.waves <= tiles && a.groups * a.waves < fill) a.waves *= 2;
  // more workgroups where that leaves each wave two tiles at least
  int64_t splits = 1;
  if (a.waves == kMaxWaves) {
    splits = fill / (a.groups * kMaxWaves);
    if (splits > tiles / (2 * kMaxWaves)) splits = tiles / (2 * kMaxWaves);
  }
  a.splits = (int)(splits < 1 ? 1 : splits);
  return a;
}

// Where every row sees its sequence's all, some sequences may have far more to do than others: their blocks get
// more workgroups.  The tree of 25 nodes over 16 sequences of 1 to 7,777 tokens: 54 us with as many for each,
// 41 so; of equal lengths with the same sum 33 either way.  (In workgroups of two waves 38, but of equal ones 38.)
namespace {
constexpr int kBalanceWaves = 4;  // per workgroup at least: fewer, and there are several rounds of them anyway
bool may_balance(const gca_window& w) { return w.window == 0 && w.B > 1 && w.B <= 64 && w.capacity >= 1024; }
bool balanced(const gca_window& w, const WindowAttnPlan& a) {
  return may_balance(w) && a.rows <= 32 && a.waves >= kBalanceWaves;
}
}  // namespace

size_t window_workspace(const gca_window& w, int64_t T) {
  // (what any number of row blocks of this height, or of 32, asks for: it then never falls as T grows)
  const int rows = rows_of(w, T) == 16 ? 16 : 32;
  const bool balance = may_balance(w);
  if (!balance && tiles_seen(w, T, rows) < 4 * kMaxWaves) return 0;
  // workgroups: as many waves as fill the chip, and balanced up to twice that
  const int64_t most = balance ? 2 * kWavesPerCu * device_cus() / kBalanceWaves : kWavesPerCu * device_cus() / kMaxWaves;
  return align256((size_t)most * rows * (kD + 2) * sizeof(float));
}

hipError_t launch_window_attn(const gca_window& w, const void* q, const int32_t* parents, const int32_t* lengths,
                              const float* slopes, void* out, float* lse, int64_t T, void* ws, hipStream_t stream) {
  const WindowAttnPlan a = window_attn_plan(w, T);
  WindowParams p;
  p.items = (uint32_t)(a.groups * a.splits);
  p.splits = (uint32_t)a.splits;
  p.blocks = (uint32_t)a.blocks;
  p.nw = (uint32_t)a.waves;
  p.Hkv = w.Hkv;
  p.H = w.H;
  p.B = w.B;
  p.G = w.H / w.Hkv;
  p.T = (uint32_t)T;
  p.M = (uint32_t)(p.G * T);
  p.per_head = (uint32_t)a.per_head;
  p.ring_tiles = (uint32_t)(w.capacity / 64);
  p.ring = w.window > 0;
  p.window = w.window;
  p.length = w.length;
  p.parents = parents;
  p.lengths = lengths;
  p.slopes = slopes;
  p.k = static_cast<const uint8_t*>(w.k);
  p.v = static_cast<const uint8_t*>(w.v);
  p.ks = w.k_scale;
  p.vs = w.v_scale;
  p.q = q;
  p.out = out;
  p.lse = lse;
  p.part = static_cast<float*>(ws);
  p.part_ml = p.part + (size_t)a.groups * a.splits * a.rows * kD;
  // (a window has 2 H tickets per sequence)
  p.ticket = a.blocks <= 2 * (int64_t)p.G ? w.ticket : nullptr;
  const float s = fabsf(w.attn_scale);
  p.scale = (s > 0.f ? s : 1.f) * kLog2e;
  p.unscale = s > 0.f ? 1.f / s : 1.f;
  p.negate = w.attn_scale < 0.f ? (w.dtype == GCA_BF16 ? 0x80008000u : 0x80000000u) : 0u;
  p.keep = s > 0.f ? 0xffffffffu : 0u;
  p.off_by_one = w.off_by_one;
  p.balance = balanced(w, a) && p.ticket;
  size_t lds = (size_t)a.waves * 192 * sizeof(float);
  const size_t parts = a.waves * a.splits > 1 ? (size_t)a.waves * a.rows * (kD + 2) * sizeof(float) : 0;
  if (parts > lds) lds = parts;
  const dim3 grid((p.items + 7) / 8 * 8);
  const dim3 block(64 * a.waves);
  auto run = [&](auto tag, auto i8) {
    using T_ = decltype(tag);
    constexpr bool I8 = decltype(i8)::value;
    const char* name = "window_attn_kernel";
    auto attend = [&](auto tree) {
      constexpr bool TREE = decltype(tree)::value;
      if (a.rows == 16) launch_kernel(name, window_attn_kernel<T_, I8, 16, 1, TREE>, grid, block, lds, stream, p);
      else if (a.rows == 32) launch_kernel(name, window_attn_kernel<T_, I8, 32, 1, TREE>, grid, block, lds, stream, p);
      else if constexpr (sizeof(T_) == 2 && !I8)
        launch_kernel(name, window_attn_kernel<T_, I8, 32, 2, TREE>, grid, block, lds, stream, p);
    };
    parents ? attend(std::true_type{}) : attend(std::false_type{});
    if (a.splits > 1 && !p.ticket) {
      const dim3 joins((unsigned)((a.groups * a.rows * 16 + 255) / 256)), threads(256);
      name = "window_join_kernel";
      if (a.rows == 16) launch_kernel(name, window_join_kernel<T_, 16>, joins, threads, 0, stream, p);
      else launch_kernel(name, window_join_kernel<T_, 32>, joins, threads, 0, stream, p);
    }
  };
  if (w.dtype == GCA_BF16) w.format == GCA_INT8 ? run(__bf16{}, std::true_type{}) : run(__bf16{}, std::false_type{});
  else w.format == GCA_INT8 ? run(float{}, std::true_type{}) : run(float{}, std::false_type{});
  return take_launch_error();
}

}  // namespace gca
