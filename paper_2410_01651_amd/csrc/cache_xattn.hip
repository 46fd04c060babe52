// Grouped cross attention over the 8-bit chunk cache (gca_cache_xattn): Eq. 2-3 for groups of
// any number of query rows, each group with its own list of slots.
//
// Mathematics.  For slot j of a list, K_j = kappa_j N_j and V_j = nu_j M_j with 8-bit numbers
// N, M, so  s = (attn_scale kappa_j) q N_j^T,  P = softmax(s) over the chunk's tokens, and
// out = sum_j w_j P V_j = u sum_j (w_j nu_j / u) P M_j  with u a power of two, by the list's largest
// w_j nu_j.  Every e4m3 number and every int8 is exact in bf16 and in fp16, so the scales stay out
// of the operands: q N^T is a product of exact operands with fp32 sums (fp32 queries: three
// bf16 terms, 24 bits), and the scaled probabilities (w_j nu_j / u) P < 65,473 meet M in
// fp16, 11 bits each (fp32 tensors: two fp16 terms, 22 bits).  As every chunk has a softmax of its own,
// nothing is rescaled and the slots of a list can be split over waves and added.
// One fp16 term for bf16 tensors is a choice: with it a tenth of the outputs is the neighbour of the
// bf16 that fp32 sums round to (1.67e-3 of fp64 in all, against 1.66e-3); two terms leave 2 in 10,000, but
// take, one / two, us: a token 4.5 / 4.8, 64 rows of 32 sequences 11.8 / 14.1, a 64K
// prompt 470 / 605 (a cold run).  fp32 tensors: 2.0e-7 of fp64 (fp32 sums alone: 1.5e-7).
//
// Layout.  The products are formed transposed, S^T = N Q^T and O^T = M^T P^T, on MFMA tiles of
// W x W (W = 32, or 16 for at most 16 rows): lane l = W g + c has query row c as its column.
// Row m of block a of N is not token W a + m but the token that makes a lane's accumulators
// consecutive tokens (`lane_row`): W = 32: 32 a + 16 g + (0..15); W = 16: 16 g + (0..15).  They are
// then, rounded, the operand of the second product as they stand, and what a lane needs of M
// (stored transposed: columns of a chunk's values are rows) are 16 consecutive bytes; so are
// its columns of N.  A tile is 4 loads of 16 bytes per lane straight from the cache into
// registers, unpacked two numbers per instruction (e4m3), with neither LDS nor a transpose.
// The same order of M's rows leaves a lane 16 consecutive columns of the output.
//
// Work.  One workgroup per (sequence, cached head, group, block of rows); its waves take the
// list's valid slots in turn.
//
// Bounds, 8 entries per list, bf16.  One token of 64 sequences and 16 heads: HBM, 67 MB of tiles in 13.4
// us (5.0 TB/s); of one sequence: a chain of three trips to memory, 4.5 us.  A 64K prompt of 2
// sequences and 16 heads: instruction issue, 400-415 us, 0.57 of the rate of a large matrix product (532
// vector instructions of which 32 are matrix ones per slot and 64 rows); int8 452 us (more instructions to
// unpack), fp32 800, int8 867 (2.5 times the products).
#include "cache_plan.hpp"
#include "gca_device.hpp"
#include "gca_launch.hpp"
#include "numbers8.hpp"

namespace gca {
namespace {

constexpr int kMaxWaves = 8;
constexpr int kTileBytes = kS * kD;

// (in the order of use)
struct XattnParams {
  uint32_t items, blocks;  // work items; row blocks per group
  uint32_t nw;             // waves per item
  uint32_t nQ, Hkv, Hr;
  int topk, lag, C;
  uint32_t H, G, rows, M;  // M = G rows: query rows of a group that share a cached head
  uint32_t part;           // bytes of LDS before the partial outputs
  const int32_t* idx;
  const float* sel;
  const int32_t* tokens;
  const float* ks;
  const float* vs;
  const uint8_t* k;
  const uint8_t* v;
  const void* q;
  void* out;
  float* lse;
  float* w;
  float scale;      // |attn_scale| log2 e
  uint32_t negate;  // the sign bits of one query entry (fp32) or two, if attn_scale < 0
  int off_by_one;
};

// (Indices by builtin: what is behind threadIdx and its like does not inline under this file's
// floating point flags and would be called.)
// T: type of the queries; W: MFMA tile; NC: column blocks of W query rows.
template <typename T, bool I8, int W, int NC>
__global__ __launch_bounds__(kMaxWaves * 64, 2) void cache_xattn_kernel(XattnParams p) {
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
  typedef __attribute__((ext_vector_type(NR))) float Acc;
  extern __shared__ __attribute__((aligned(16))) float smem[];

  const uint32_t it = (uint32_t)xcd_swizzle(__builtin_amdgcn_workgroup_id_x(), (p.items + 7) / 8 * 8);
  if (it >= p.items) return;
  const uint32_t tid = __builtin_amdgcn_workitem_id_x(), nw = p.nw, threads = 64 * nw;
  const int lane = tid & 63, g = lane / W, col = lane % W;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // item = ((b Hkv + h) nQ + t) blocks + block
  // (the quotients are formed on the vector unit: back to scalar registers, and with them every address)
  auto scalar = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane(x); };
  const uint32_t bt = scalar(it / p.blocks), blk = it - bt * p.blocks;
  const uint32_t bh = scalar(bt / p.nQ), t = bt - bh * p.nQ;
  const uint32_t b = scalar(bh / p.Hkv), h = bh - b * p.Hkv;
  const int K = p.topk;

  // piece (a, y) of a tile: its row lane_row + 32 a (W = 32) or + 4 a, the token (column) of this
  // lane's operand row, bytes 16 (g + NG y) ..
  const uint32_t lane_row = W == 32 ? 16 * ((col >> 2) & 1) + 4 * (col >> 3) + (col & 3)
                                    : 16 * (col >> 2) + (col & 3);
  const uint32_t lane_off = lane_row * kD + 16 * g;
  // (`there` false: nothing is wanted, and the descriptor is empty.  The loads are issued either
  // way, so that what is in flight at a wait is known and a wait for one tile does not wait for the
  // next; the address is always that of one of the cache's own tiles.)
  auto load_tile = [&](u32x4* x, const uint8_t* base, int slot, bool there) {
    const __amdgpu_buffer_rsrc_t tile = range_rsrc(
        reinterpret_cast<const char*>(base) + ((int64_t)bh * p.C + slot) * kTileBytes, there ? kTileBytes : 0);
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
      for (int y = 0; y < NX; ++y)
        x[a * NX + y] = __builtin_amdgcn_raw_buffer_load_b128(
            tile, lane_off, (W == 32 ? 32 : 4) * a * kD + 16 * NG * y, 0);
  };

  // ---- the list: lane s holds entry s.  Groups before the first list take the weights of
  // the last one, which feeds no group.
  const bool has_list = (int)t >= p.lag;
  const uint32_t list = has_list ? t - p.lag : p.nQ - 1;
  const int64_t row = ((int64_t)b * p.Hr + (p.Hr == 1 ? 0 : h)) * p.nQ + list;
  // (loads on every path, lanes behind the list's end taking its last entry's: one that a branch
  // guards is waited for before the next)
  const uint32_t mine_at = min(lane, K - 1);
  int j = scalar_ptr(p.idx + row * K)[mine_at];
  const float sv = scalar_ptr(p.sel + row * K)[mine_at];
  const bool named = lane < K && j >= 0 && j < p.C;
  j = named ? j : 0;
  const int64_t slot0 = (int64_t)bh * p.C;
  int length = scalar_ptr(p.tokens + (int64_t)b * p.C)[(uint32_t)j];
  float kscale = scalar_ptr(p.ks + slot0)[(uint32_t)j];
  float vscale = scalar_ptr(p.vs + slot0)[(uint32_t)j];

  // The first tiles that the list names for this wave are asked for at once, beside their lengths
  // and scales: it is nearly always so that they are in use.
  auto share = [&](uint64_t entries) {  // this wave's: those whose rank is its number (mod nw)
    return (uint32_t)(entries & __ballot(((uint32_t)lanes_below(entries) & (nw - 1)) == wave));
  };
  const uint32_t guess = has_list ? share(__ballot(named)) : 0;
  const int first = guess != 0 ? __builtin_amdgcn_readlane(j, __builtin_ctz(guess)) : 0;
  u32x4 kr[NA * NX], vr[NA * NX];
  load_tile(kr, p.k, first, guess != 0);
  load_tile(vr, p.v, first, guess != 0);

  // ---- the queries: lane (g, c) takes columns 16 (g + NG x) .. of row c, x < NX
  const uint32_t m0 = blk * QB;
  const bool flat = p.G == 1 || p.nQ == 1;  // a group's rows are consecutive
  const int64_t row0 = ((int64_t)(b * p.H + h * p.G) * p.nQ + t) * p.rows + (flat ? m0 : 0);
  auto ahead = [&](uint32_t m) -> int64_t {  // of the item's row m, from row0
    if (flat) return m;
    m += m0;
    return (int64_t)(m / p.rows) * p.nQ * p.rows + m % p.rows;
  };
  bf16x8 qf[NC][NK][QP];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const uint32_t m = min(uint32_t(c * W + col), p.M - 1 - m0);
    const auto* qr = scalar_ptr(reinterpret_cast<const T*>(p.q) + row0 * kD) + ahead(m) * kD;
#pragma unroll
    for (int s = 0; s < NK; ++s) {
      const auto* src = qr + 16 * (g + NG * (s >> 1)) + 8 * (s & 1);
      if constexpr (kB16) {
        u32x4 x = *reinterpret_cast<const __attribute__((address_space(1))) u32x4*>(src);
        x ^= u32x4{p.negate, p.negate, p.negate, p.negate};
        qf[c][s][0] = __builtin_bit_cast(bf16x8, x);
      } else {
#pragma unroll
        for (int m8 = 0; m8 < 8; ++m8) {
          float x = src[m8];
          x = __uint_as_float(__float_as_uint(x) ^ p.negate);
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

  // ---- fusion weights (Eq. 2)
  length = named ? max(min(length, kS), 0) : 0;
  const bool valid = length > 0;
  vscale = valid ? vscale : 0.f;  // (a free slot's scale may be anything)
  const float top = max64(valid ? sv : -INFINITY);
  const float es = valid ? expf(sv - top) : 0.f;
  const float total = sum64(es);
  const float wl = valid ? es / total : 0.f;
  if (p.w && wave == 0 && blk == 0 && (p.Hr != 1 || h == 0) && lane < K) p.w[row * K + lane] = wl;
  // c_j = w_j nu_j as mantissa and exponent, since the product may lie outside fp32's range.  All are scaled
  // by the power of two 2^(16 - top_octave) that brings the largest into [1023 / 2048, 1023 / 1024) 2^16,
  // which fp16 holds.  (By the products: a chunk that hardly counts may have any value scale.)
  const float mant = __builtin_amdgcn_frexp_mantf(wl) * __builtin_amdgcn_frexp_mantf(vscale);
  const int expo = __builtin_amdgcn_frexp_expf(wl) + __builtin_amdgcn_frexp_expf(vscale);
  const int octave = expo + __builtin_amdgcn_frexp_expf(mant * (1024.f / 1023.f));
  const int top_octave = __builtin_amdgcn_readfirstlane((int)max64(mant != 0.f ? (float)octave : -1000.f));
  const float coef = __builtin_ldexpf(mant, expo - top_octave + 16);
  const uint64_t all = __ballot(valid && has_list);
  const uint32_t count = __popcll(all);
  uint32_t mine = share(all);
  const int entry = (j << 7) | length;  // (one register for both: C <= 2^18)

  const uint32_t nrows = min((uint32_t)QB, p.M - m0);
  float* const lse_s = smem;  // [row][entry]
  if (p.lse) {
    for (uint32_t e = tid; e < nrows * K; e += threads) lse_s[e] = -INFINITY;
    __syncthreads();
  }

  // a lane's values of tokens behind the first len set to x (value u is token 32 (u / 16) + 16 g
  // + u % 16, W = 32, or 16 g + u, W = 16); opaque: compared where it happens, in the rare branch
  auto cut = [&](float* v, int len, float x) {
    const int left = opaque(len - 16 * g);
#pragma unroll
    for (int u = 0; u < NV; ++u)
      if ((W == 32 ? 32 * (u / 16) + u % 16 : u) >= left) v[u] = x;
  };

  Acc o[NC][NA];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int a = 0; a < NA; ++a) o[c][a] = Acc{};

  if (mine != 0) {
    const int jn = __builtin_amdgcn_readlane(entry, __builtin_ctz(mine)) >> 7;
    if (jn != first) {
      load_tile(kr, p.k, jn, true);
      load_tile(vr, p.v, jn, true);
    }
  }
  while (mine != 0) {
    const int s = __builtin_ctz(mine);
    mine &= mine - 1;
    const int jn = mine != 0 ? __builtin_amdgcn_readlane(entry, __builtin_ctz(mine)) >> 7 : 0;
    const int len = __builtin_amdgcn_readlane(entry, s) & 127;
    const float sc = p.scale * __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(kscale), s));
    const float cf = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(coef), s));

    // S^T = N Q^T
    Acc st[NC][NA];
#pragma unroll
    for (int a = 0; a < NA; ++a) {
#pragma unroll
      for (int c = 0; c < NC; ++c) st[c][a] = Acc{};
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        const u32x4 r = kr[a * NX + (i >> 1)];
        const bf16x8 f = to_bf16<I8>(r[2 * (i & 1)], r[2 * (i & 1) + 1]);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < QP; ++e) st[c][a] = mma(f, qf[c][i][e], st[c][a]);
      }
    }
    load_tile(kr, p.k, jn, mine != 0);

    // softmax over the chunk's tokens
    f16x8 pf[NC][NK][PP];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float v[NV];
#pragma unroll
      for (int u = 0; u < NV; ++u) v[u] = st[c][u / NR][u % NR];
      if (len < kS) cut(v, len, -INFINITY);
      float mx = fmaxf(fmaxf(v[0], v[1]), v[2]), mx2 = fmaxf(fmaxf(v[3], v[4]), v[5]);
#pragma unroll
      for (int u = 6; u + 3 < NV; u += 4) {
        mx = fmaxf(fmaxf(mx, v[u]), v[u + 1]);
        mx2 = fmaxf(fmaxf(mx2, v[u + 2]), v[u + 3]);
      }
      mx = fmaxf(fmaxf(mx, v[NV - 2]), fmaxf(mx2, v[NV - 1]));
      if constexpr (W == 16) {
        uint32_t x, y;
        pair16(__float_as_uint(mx), x, y);
        mx = fmaxf(__uint_as_float(x), __uint_as_float(y));
      }
      mx = max_xor32(mx) * sc;
      if (p.off_by_one) mx = fmaxf(mx, 0.f);
#pragma unroll
      for (int u = 0; u < NV; ++u) v[u] = __builtin_amdgcn_exp2f(fmaf(v[u], sc, -mx));
      if (len < kS) cut(v, len, 0.f);  // (a scale of zero times -inf)
      float sum = v[0], sum2 = v[1];
#pragma unroll
      for (int u = 2; u < NV; u += 2) {
        sum += v[u];
        sum2 += v[u + 1];
      }
      sum += sum2;
      if constexpr (W == 16) {
        uint32_t x, y;
        pair16(__float_as_uint(sum), x, y);
        sum = __uint_as_float(x) + __uint_as_float(y);
      }
      sum = sum_xor32(sum);
      if (p.off_by_one) sum += __builtin_amdgcn_exp2f(-mx);
      if (p.lse && g == 0 && (uint32_t)(c * W + col) < nrows)
        lse_s[(c * W + col) * K + s] = (mx + __builtin_amdgcn_logf(sum)) * kLn2;
      const float f = cf * __builtin_amdgcn_rcpf(sum);
#pragma unroll
      for (int i = 0; i < NK; ++i)
#pragma unroll
        for (int m = 0; m < 8; ++m) {
          float x = v[8 * i + m] * f;
          // (one rounding of x: the first term's and the second's must be the same number)
          if constexpr (PP == 2) asm("" : "+v"(x));
          const _Float16 hi = (_Float16)x;
          pf[c][i][0][m] = hi;
          if constexpr (PP == 2) pf[c][i][PP - 1][m] = (_Float16)(x - (float)hi);
        }
    }

    // O^T += M^T P^T (numbers behind the chunk's last token are cleared: a masked NaN stays out)
    if (len < kS) {
      const int here = opaque(len - 16 * g);
#pragma unroll
      for (int y = 0; y < NX; ++y)
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const int left = here - (16 * NG * y + 4 * d);
          const uint32_t keep = left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
#pragma unroll
          for (int a = 0; a < NA; ++a) vr[a * NX + y][d] &= keep;
        }
    }
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        const u32x4 r = vr[a * NX + (i >> 1)];
        const f16x8 f = to_f16<I8>(r[2 * (i & 1)], r[2 * (i & 1) + 1]);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < PP; ++e) o[c][a] = mma(f, pf[c][i][e], o[c][a]);
      }
    load_tile(vr, p.v, jn, mine != 0);
  }

  // ---- output: value u of a lane is column 32 (u / 16) + 16 g + u % 16 (W = 32) or 16 g + u
  const auto unscale = [&](float x) { return __builtin_ldexpf(x, top_octave - 16); };
  T* const out0 = (T*)scalar_ptr(reinterpret_cast<T*>(p.out) + row0 * kD);
  if (nw == 1) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const uint32_t m = c * W + col;
      if (m >= nrows) continue;
      T* dst = out0 + ahead(m) * kD + 16 * g;
#pragma unroll
      for (int u = 0; u < NV; u += 8) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = unscale(o[c][(u + e) / NR][(u + e) % NR]);
        store8(dst + (u / 16) * 32 + u % 16, x);
      }
    }
    if (p.lse) __syncthreads();
  } else {
    // the waves' partial sums: part[wave][row][16 blocks of 4], block x of row r at x ^ (r mod 16)
    float* const part = smem + p.part / sizeof(float);
    const uint32_t waves = min(nw, count);
    if (wave < waves) {
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
              f32x4{a[u % NR], a[u % NR + 1], a[u % NR + 2], a[u % NR + 3]};
        }
      }
    }
    __syncthreads();
    for (uint32_t e = tid; e < nrows * 16; e += threads) {
      const uint32_t m = e >> 4, x = e & 15;
      f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
      for (uint32_t y = 0; y < waves; ++y)
        acc += *reinterpret_cast<const f32x4*>(part + (y * nrows + m) * kD + 4 * (x ^ (m & 15)));
      store4(out0 + ahead(m) * kD + 4 * x, unscale(acc[0]), unscale(acc[1]), unscale(acc[2]), unscale(acc[3]));
    }
  }
  if (p.lse) {
    float* const dst = (float*)scalar_ptr(p.lse + row0 * K);
    for (uint32_t e = tid; e < nrows * K; e += threads) {
      const uint32_t m = flat ? 0 : e / K;
      dst[flat ? (int64_t)e : ahead(m) * K + (e - m * K)] = lse_s[e];
    }
  }
}

// Rows per item: 16 where a group has no more; else 32, or in bf16 64, which unpacks a tile for
// both halves but has two waves per SIMD where 32 has three (fp32 queries in three terms leave no
// registers for it).  64 where such items give every SIMD two waves and waste no half: groups of 64
// rows, 8 entries each, 32 / 64 rows per item, us: 64 groups 6.0 / 8.1, 512 12.2 / 12.7, 1,024 17.7 /
// 19.8, 2,048 30.6 / 30.4, 4,096 62.5 / 59.8, 8,192 126 / 114; of 130 rows, 768 groups 28.5 / 35.
int rows_per_item(const gca_cache& c, int64_t nQ, int64_t M) {
  if (M <= 16) return 16;
  const int64_t halves = (M + 31) / 32, groups = (int64_t)c.B * c.Hkv * nQ;
  const bool whole = halves % 2 == 0 || halves >= 8;
  return c.dtype == GCA_BF16 && whole && groups * (halves / 2) >= 8 * device_cus() ? 64 : 32;
}

}  // namespace

int64_t xattn_items(const gca_cache& c, int64_t nQ, int64_t rows) {
  const int64_t M = (int64_t)(c.H / c.Hkv) * rows, per = rows_per_item(c, nQ, M);
  return (int64_t)c.B * c.Hkv * nQ * ((M + per - 1) / per);
}

hipError_t launch_cache_xattn(const gca_cache& c, const void* q, const int32_t* idx, const float* sel, void* out,
                              float* lse, float* w, int64_t nQ, int64_t rows, int lag, hipStream_t stream) {
  const int64_t M = (int64_t)(c.H / c.Hkv) * rows;
  const int qb = rows_per_item(c, nQ, M);
  XattnParams p;
  p.k = static_cast<const uint8_t*>(c.k);
  p.v = static_cast<const uint8_t*>(c.v);
  p.ks = c.k_scale;
  p.vs = c.v_scale;
  p.tokens = c.tokens;
  p.q = q;
  p.idx = idx;
  p.sel = sel;
  p.out = out;
  p.lse = lse;
  p.w = w;
  p.items = (uint32_t)xattn_items(c, nQ, rows);
  p.blocks = (uint32_t)((M + qb - 1) / qb);
  p.nQ = (uint32_t)nQ;
  p.H = c.H;
  p.Hkv = c.Hkv;
  p.Hr = c.Hr;
  p.G = c.H / c.Hkv;
  p.rows = (uint32_t)rows;
  p.M = (uint32_t)M;
  p.topk = c.topk;
  p.lag = lag;
  p.off_by_one = c.off_by_one;
  p.C = (int)c.capacity;
  p.scale = fabsf(c.attn_scale) * kLog2e;
  p.negate = c.attn_scale < 0.f ? (c.dtype == GCA_BF16 ? 0x80008000u : 0x80000000u) : 0u;
  const int rb = (int)(M < qb ? M : qb);
  p.part = lse ? (uint32_t)((rb * c.topk * sizeof(float) + 15) & ~size_t(15)) : 0u;
  // Waves per item: enough to fill the chip's eight waves per CU, no more than the list has
  // entries, and at most 64 KiB of LDS.  At most 4 / 8 / 16 (16-row items), one token, us: one sequence of 8
  // heads, 8 entries 4.4 / 4.5 / 4.6, 16 5.6 / 5.4 / 6.2, 32 7.9 / 7.2 / 8.0; 16 sequences of 8 cached
  // heads, int8, 16 entries 6.5 / 6.5 / 7.1.
  int nw = 1;
  while (nw < kMaxWaves && 2 * nw <= c.topk && (int64_t)p.items * nw < 8 * device_cus() &&
         p.part + 2 * nw * rb * kD * sizeof(float) <= 65536)
    nw *= 2;
  p.nw = (uint32_t)nw;
  const size_t lds = p.part + (nw > 1 ? (size_t)nw * rb * kD * sizeof(float) : 0);
  const dim3 grid((p.items + 7) / 8 * 8), block(64 * nw);
  auto run = [&](auto tag, auto i8) {
    using T = decltype(tag);
    constexpr bool I8 = decltype(i8)::value;
    if (qb == 16) launch_kernel("cache_xattn_kernel", cache_xattn_kernel<T, I8, 16, 1>, grid, block, lds, stream, p);
    else if (qb == 32) launch_kernel("cache_xattn_kernel", cache_xattn_kernel<T, I8, 32, 1>, grid, block, lds, stream, p);
    else if constexpr (sizeof(T) == 2)
      launch_kernel("cache_xattn_kernel", cache_xattn_kernel<T, I8, 32, 2>, grid, block, lds, stream, p);
  };
  if (c.dtype == GCA_BF16) c.format == GCA_INT8 ? run(__bf16{}, std::true_type{}) : run(__bf16{}, std::false_type{});
  else c.format == GCA_INT8 ? run(float{}, std::true_type{}) : run(float{}, std::false_type{});
  return take_launch_error();
}

}  // namespace gca
