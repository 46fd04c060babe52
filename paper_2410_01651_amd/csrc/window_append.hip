// Appending tokens to the 8-bit token window (gca_window_append), and keeping an accepted path of
// the newest ones (gca_window_keep).
//
// Append.  Every token's 64 keys, and its 64 values, become 8-bit numbers with one scale; the values are
// kept transposed per 64 rows.  One wave per 64 positions that share a tile of rows, and per keys or
// values: lane (rg, cg) = (l / 8, l % 8) holds the 8 x 8 block of rows 8 rg .. and columns 8 cg .., so that a
// row's largest magnitude is a reduction over 8 lanes and the values' tile is byte blocks turned in
// registers.  A tile that new tokens fill only in part (a prompt's first and last)
// writes its own rows and no others.  Few tokens are taken eight to a wave instead, a row for eight lanes, and are
// read before the length that says where they go is there: eight tokens of 64 sequences, 16 heads, 5.0 us for 9.7.
// Bound: few tokens by the trips to memory; many by HBM, at 2 B Hkv T (64 (e + 1) + 4) bytes: four prompts of
// up to 8,192 tokens, 16 heads, 113 MB in 22.7 us, 5.0 TB/s, as a large copy, where the last cache still has
// what was just computed, and 121 MB in 30.6 us, 3.9 TB/s, where it has not.  (Loads that leave that cache alone:
// 27.0 us there, but 25.6 for the 22.7.)  The same prompts in int8 23 us, of fp32 tensors 31 (int8 32), without a window's
// end 24 (33).
//
// Keep.  One wave per (sequence, cached head), eight tokens at a time (64 sequences' paths, 16 heads, 6.9 us for
// 15.3 one by one); lane d moves key d and value d of each token.  As a path ascends, token i comes from a place at
// or behind i, so what later tokens come from is never overwritten.  Bound by the trips to memory (lengths and
// path, tokens, the ticket).
#include "gca_device.hpp"
#include "gca_launch.hpp"
#include "numbers8.hpp"
#include "window_plan.hpp"

namespace gca {
namespace {

constexpr int kAppendWaves = 8;
// Eight tokens to a wave / a tile to a wave: 64 sequences, 16 heads, 25 tokens 6.3 / 11.5 us, 64 tokens 10.4 / 13.5, 128
// tokens 16.6 / 16.7, 512 tokens 56 / 38; 4 sequences, 8 heads, 128 tokens 4.2 / 6.1.  (The border is where large batches
// meet; small ones pay for it up to some hundred tokens: of 129, by tiles, 4 sequences take 6.5 us, one 5.7.)
constexpr int64_t kFewTokens = 128;
constexpr int kRingTile = kS * kD;  // bytes of a tile's keys or values

struct AppendParams {
  const void* src[2];  // new keys, new values
  uint8_t* dst[2];
  float* scale[2];
  int32_t* length;
  int32_t* ticket;
  const int32_t* lengths;
  int64_t T, C;
  uint32_t seqs, per;    // sequences; workgroups of each
  uint32_t items;        // waves' items of a sequence: Hkv tiles 2
  uint32_t tiles, Hkv, stride;  // tiles of 64 (8) tokens of a sequence and head; tickets of a sequence
  int ring;
};

// The largest of 8 consecutive lanes' values.
__device__ __forceinline__ uint32_t max_row8(uint32_t x) {
  x = max(x, dpp<kDppXor1>(x));
  x = max(x, dpp<kDppXor2>(x));
  return max(x, dpp<kDppHalfMirror>(x));
}

// New tokens of sequence b.
__device__ __forceinline__ int64_t new_tokens(const int32_t* lengths, uint32_t b, int64_t T) {
  const int64_t n = lengths ? lengths[b] : T;
  return n < 0 ? 0 : n < T ? n : T;
}

// The largest magnitude of a lane's eight entries of a row, as its bits.
__device__ __forceinline__ uint32_t top_of(const Row8<__bf16>& x) {
  typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;  // (magnitudes of bf16 order as integers)
  u16x2 m = __builtin_bit_cast(u16x2, x.x[0] & 0x7fff7fffu);
#pragma unroll
  for (int c = 1; c < 4; ++c) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x.x[c] & 0x7fff7fffu));
  return (uint32_t)max(m[0], m[1]) << 16;
}
__device__ __forceinline__ uint32_t top_of(const Row8<float>& x) {
  uint32_t top = 0;
#pragma unroll
  for (int c = 0; c < 8; ++c) top = max(top, __float_as_uint(x.at(c)) & 0x7fffffffu);
  return top;
}

// A row's eight entries of this lane, of which `top` is the row's largest magnitude, as 8-bit numbers (w0, w1),
// and the row's scale.
template <bool I8, typename T>
__device__ __forceinline__ float numbers_of(const Row8<T>& x, uint32_t top, bool values, uint32_t& w0, uint32_t& w1) {
  const bool odd = top >= 0x7f800000u, nan = top > 0x7f800000u;  // anything not finite; NaN
  if (__ballot(odd) != 0) {  // the largest finite magnitude
    uint32_t fin = 0;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const uint32_t u = __float_as_uint(x.at(c)) & 0x7fffffffu;
      fin = max(fin, u < 0x7f800000u ? u : 0u);
    }
    top = max_row8(fin);
  }
  float scale;
  uint32_t w[2];
  if constexpr (I8) {
    const float amax = fmaxf(__uint_as_float(top), 0x1p-100f);
    scale = amax / 127.f;
    // As the chunk cache forms it, so that the same tokens are the same numbers in both (ties are common among bf16
    // entries, and go by the factor's last bit).  |x| inv <= 127 (1 + 2^-21): 127 at most once rounded
    const float inv = (1.f / amax) * 127.f;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      uint32_t o = 0;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float y = x.at(4 * q + c) * inv;
        if (odd) y = y == y ? fminf(fmaxf(y, -127.f), 127.f) : 0.f;
        o |= ((uint32_t)(int)__builtin_rintf(y) & 0xffu) << (8 * c);
      }
      w[q] = o;
    }
  } else {
    // 448 = 1.75 x 2^8: the least power of two s with amax / s <= 448 (at least 2^-126)
    const int e = max((int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), 1);
    scale = __uint_as_float((uint32_t)e << 23);
    const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      uint32_t o = 0;
#pragma unroll
      for (int c = 0; c < 4; c += 2) {
        float y0 = x.at(4 * q + c) * inv, y1 = x.at(4 * q + c + 1) * inv;
        if (odd) {  // infinities (a comparison with NaN is false)
          if (__builtin_fabsf(y0) > 448.f) y0 = __builtin_copysignf(448.f, y0);
          if (__builtin_fabsf(y1) > 448.f) y1 = __builtin_copysignf(448.f, y1);
          if (values) {  // (a value's number is never NaN: it would reach rows that do not see it)
            y0 = y0 == y0 ? y0 : 0.f;
            y1 = y1 == y1 ? y1 : 0.f;
          }
        }
        o = pk_e4m3(y0, y1, o, c != 0);
      }
      w[q] = o;
    }
  }
  w0 = w[0];
  w1 = w[1];
  return nan ? __builtin_nanf("") : scale;
}

// Tokens that are kept of the n new ones: [first, last).
__device__ __forceinline__ int64_t first_kept(const AppendParams& p, int64_t n) {
  return p.ring && n > p.C ? n - p.C : 0;
}
__device__ __forceinline__ int64_t last_kept(const AppendParams& p, int64_t length, int64_t n) {
  return p.ring || length + n <= p.C ? n : p.C - length;
}

// Many tokens: one tile of rows, of `tiles` of the sequence and head.
template <typename T, bool I8>
__device__ __forceinline__ void append_tile(const AppendParams& p, uint32_t b, uint32_t item, uint32_t tiles,
                                            int64_t length, int64_t n, int lane) {
  // item = (h tiles + t) 2 + which
  const uint32_t which = item & 1;
  const uint32_t h = __builtin_amdgcn_readfirstlane((item >> 1) / tiles), t = (item >> 1) - h * tiles;
  const int64_t i0 = first_kept(p, n), i1 = last_kept(p, length, n);
  const int64_t first = ((length + i0) / kS + t) * kS;  // the tile's first position
  int64_t lo = length + i0 - first, hi = length + i1 - first;  // its rows [lo, hi)
  lo = lo > 0 ? lo : 0;
  hi = hi < kS ? hi : kS;
  if (lo >= hi) return;
  const int64_t bh = (int64_t)b * p.Hkv + h;
  constexpr int kRow = kD * (int)sizeof(T);
  const __amdgpu_buffer_rsrc_t src =
      range_rsrc(reinterpret_cast<const char*>(p.src[which]) + (bh * p.T + (first + lo - length)) * kRow,
                 (uint32_t)((hi - lo) * kRow));
  const int rg = lane >> 3, cg = lane & 7;
  Row8<T> x[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const int row = 8 * rg + r;  // (rows of other positions lie behind the descriptor's end and read as zeros)
    const bool mine = row >= (int)lo && row < (int)hi;
    x[r].load(src, mine ? (uint32_t)((row - (int)lo) * kRow + cg * 8 * (int)sizeof(T)) : 0x40000000u, 0);
  }
  uint32_t w[16];  // row r: w[2 r], w[2 r + 1]
  float scale[8];
#pragma unroll
  for (int r = 0; r < 8; ++r)
    scale[r] = numbers_of<I8>(x[r], max_row8(top_of(x[r])), which, w[2 * r], w[2 * r + 1]);

  if (which) {
    // columns: w[2 c] holds rows 0-3 of column c, w[2 c + 1] rows 4-7
    uint32_t o[16];
#pragma unroll
    for (int q = 0; q < 2; ++q)      // columns 4 q ..
#pragma unroll
      for (int r = 0; r < 2; ++r)    // rows 4 r ..
        transpose4(w[8 * r + q], w[8 * r + 2 + q], w[8 * r + 4 + q], w[8 * r + 6 + q], o[8 * q + r], o[8 * q + 2 + r],
                   o[8 * q + 4 + r], o[8 * q + 6 + r]);
#pragma unroll
    for (int c = 0; c < 16; ++c) w[c] = o[c];
  }
  const int64_t row0 = bh * p.C + (p.ring ? (uint32_t)first % (uint32_t)p.C : (uint32_t)first);  // (below 2^32)
  // keys: row 8 rg + r, bytes 8 cg ..; values: column 8 cg + r, bytes 8 rg ..
  uint8_t* dst = p.dst[which] + row0 * kD + (which ? cg * 8 * kS + rg * 8 : rg * 8 * kD + cg * 8);
  const int from = max((int)lo - 8 * rg, 0), to = min((int)hi - 8 * rg, 8);  // this lane's rows
  if (which && (from > 0 || to < 8)) {
#pragma unroll
    for (int r = 0; r < 8; ++r)
      if (r >= from && r < to)
#pragma unroll
        for (int c = 0; c < 8; ++c) dst[c * kS + r] = (uint8_t)(w[2 * c + (r >> 2)] >> (8 * (r & 3)));
  } else {
#pragma unroll
    for (int r = 0; r < 8; ++r)
      if (which || (r >= from && r < to)) *reinterpret_cast<u32x2*>(dst + r * 64) = u32x2{w[2 * r], w[2 * r + 1]};
  }
  // the row's scale by lane cg = r of its group
  float s = scale[0];
#pragma unroll
  for (int r = 1; r < 8; ++r) s = cg == r ? scale[r] : s;
  if (cg >= from && cg < to) p.scale[which][row0 + 8 * rg + cg] = s;
}

// Few tokens: eight of them, a lane for eight entries of one.  What is read does not depend on
// the sequence's length, so it is asked for beside it.
template <typename T, bool I8>
__device__ __forceinline__ void append_few(const AppendParams& p, uint32_t b, uint32_t item, int lane) {
  // item = (h tiles + t) 2 + which: tokens 8 t ..
  const uint32_t which = item & 1;
  const uint32_t h = __builtin_amdgcn_readfirstlane((item >> 1) / p.tiles), t = (item >> 1) - h * p.tiles;
  const int cg = lane & 7;
  const int64_t i = 8 * t + (lane >> 3), bh = (int64_t)b * p.Hkv + h;
  constexpr int kRow = kD * (int)sizeof(T);
  Row8<T> x;
  x.load(range_rsrc(reinterpret_cast<const char*>(p.src[which]) + bh * p.T * kRow, (uint32_t)(p.T * kRow)),
         (uint32_t)(i * kRow + cg * 8 * (int)sizeof(T)), 0);
  const int64_t length = max(p.length[b], 0), n = new_tokens(p.lengths, b, p.T);
  uint32_t w0, w1;
  const float scale = numbers_of<I8>(x, max_row8(top_of(x)), which, w0, w1);
  if (i < first_kept(p, n) || i >= last_kept(p, length, n)) return;
  const uint32_t pos = (uint32_t)length + (uint32_t)i, row = p.ring ? pos % (uint32_t)p.C : pos;
  if (which) {
    uint8_t* dst = p.dst[1] + (bh * p.C + (row & ~63u)) * kD + cg * 8 * kS + (row & 63u);
#pragma unroll
    for (int c = 0; c < 8; ++c) dst[c * kS] = (uint8_t)((c < 4 ? w0 : w1) >> (8 * (c & 3)));
  } else {
    *reinterpret_cast<u32x2*>(p.dst[0] + (bh * p.C + row) * kD + cg * 8) = u32x2{w0, w1};
  }
  if (cg == 0) p.scale[which][bh * p.C + row] = scale;
}

// Whoever takes a sequence's last ticket knows that every workgroup has read its length, and writes
// the new one.  (A workgroup takes its ticket once its waves have read, at its end, when nothing waits for it.)
__device__ __forceinline__ void update_length(int32_t* length, int32_t* ticket, int32_t per, int64_t now) {
  bool last = per == 1;
  if (!last) {
    last = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == per - 1;
    if (last) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  if (last) *length = (int32_t)(now < 0x7fffffff ? now : 0x7fffffff);
}

// Many tokens of at most 64 sequences: every workgroup goes over the tiles of all of them; lane i holds sequence i's.
template <typename T, bool I8>
__device__ __forceinline__ void append_all(const AppendParams& p) {
  const int lane = threadIdx.x & 63;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const uint32_t seq = min((uint32_t)lane, p.seqs - 1);
  const int length = max(p.length[seq], 0), n = (int)new_tokens(p.lengths, seq, p.T);
  const int64_t i0 = first_kept(p, n), i1 = last_kept(p, length, n);
  const bool any = (uint32_t)lane < p.seqs && i1 > i0;
  const uint32_t tiles = any ? (uint32_t)((length + i1 - 1) / kS - (length + i0) / kS + 1) : 0;
  const uint32_t mine = tiles * p.Hkv * 2;
  uint32_t to = mine;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    const uint32_t y = (uint32_t)__shfl_up((int)to, s);
    to += lane >= s ? y : 0;
  }
  const uint32_t from = to - mine, all = (uint32_t)__builtin_amdgcn_readlane((int)to, 63);
  for (uint32_t item = blockIdx.x * waves + wave; item < all; item += gridDim.x * waves) {
    const int b = __builtin_popcountll(__ballot(from <= item)) - 1;  // (the last one that begins there: it has tiles)
    auto of = [&](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, b); };
    append_tile<T, I8>(p, (uint32_t)b, item - of(from), of(tiles), (int)of((uint32_t)length), (int)of((uint32_t)n),
                       lane);
  }
  __syncthreads();  // (the workgroup's waves have read the lengths)
  if (wave != 0) return;
  int drawn = 0;
  if (lane == 0) drawn = __hip_atomic_fetch_add(p.ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (__builtin_amdgcn_readfirstlane(drawn) != (int)gridDim.x - 1) return;
  if (lane == 0) __hip_atomic_store(p.ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if ((uint32_t)lane < p.seqs) p.length[lane] = (int)min((int64_t)length + n, (int64_t)0x7fffffff);
}

enum AppendForm { kFew, kMany, kAll };

// (Two workgroups of a tile per wave are to run on a CU: 128 registers.)
template <typename T, bool I8, AppendForm F>
__global__ __launch_bounds__(F == kFew ? 1024 : kAppendWaves * 64, 4) void window_append_kernel(AppendParams p) {
  if constexpr (F == kAll) {
    append_all<T, I8>(p);
  } else {
    const uint32_t b = blockIdx.x / p.per, part = blockIdx.x - b * p.per;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t waves = blockDim.x >> 6;
    const int64_t length = max((int)__builtin_amdgcn_readfirstlane(p.length[b]), 0);
    const int64_t n = new_tokens(p.lengths, b, p.T);
    for (uint32_t item = part * waves + wave; item < p.items; item += p.per * waves) {
      if constexpr (F == kFew) append_few<T, I8>(p, b, item, threadIdx.x & 63);
      else append_tile<T, I8>(p, b, item, p.tiles, length, n, threadIdx.x & 63);
    }
    __syncthreads();  // (the workgroup's waves have read the length)
    if (threadIdx.x == 0) update_length(p.length + b, p.ticket + (int64_t)b * p.stride, (int32_t)p.per, length + n);
  }
}

struct KeepParams {
  uint8_t* k;
  uint8_t* v;
  float* ks;
  float* vs;
  int32_t* length;
  int32_t* ticket;
  const int32_t* path;
  const int32_t* lengths;
  int64_t T, C;
  uint32_t Hkv, n, per, stride;
  int ring;
};

constexpr int kKeepWaves = 4;   // (16: 18.7 us for 6.9)
constexpr int kKeepTokens = 8;  // at a time

// One wave per (sequence, cached head).
__global__ __launch_bounds__(kKeepWaves * 64) void window_keep_kernel(KeepParams p) {
  const uint32_t b = blockIdx.x / p.per, part = blockIdx.x - b * p.per;
  const int lane = threadIdx.x & 63;
  const int length = max((int)__builtin_amdgcn_readfirstlane(p.length[b]), 0);
  const int64_t n = new_tokens(p.lengths, b, p.T);
  // lane i: entry i, in the path if every entry up to it is larger than the one before
  const int mine = lane < (int)p.n ? p.path[(int64_t)b * p.n + lane] : -1;
  const int left = __shfl_up(mine, 1);  // (by every lane: one that is not active has nothing to give)
  const int64_t base = length > n ? length - n : 0;
  // (no token past the capacity comes below it: it has no numbers)
  const bool lost = !p.ring && base + mine >= p.C && base + lane < p.C;
  const uint64_t good = __ballot(mine > (lane ? left : -1) && mine < n && !lost);
  const int m = good == ~0ull ? 64 : __builtin_ctzll(~good);
  const uint32_t h = part * (blockDim.x >> 6) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // entries that name their own place lead the path and stay
  const uint64_t moved = __ballot(lane < m && mine != lane);
  if (moved != 0 && h < p.Hkv) {
    const int64_t row0 = ((int64_t)b * p.Hkv + h) * p.C;
    // lane i: the rows that entry i comes from and goes to (-1: one is past the capacity); positions are below 2^32
    const uint32_t C = (uint32_t)p.C, src = (uint32_t)base + (uint32_t)mine, dst = (uint32_t)base + (uint32_t)lane;
    int from = (int)(p.ring ? src % C : src), to = (int)(p.ring ? dst % C : dst);
    if (lane >= m || (!p.ring && (src >= C || dst >= C))) from = to = -1;
    for (int i = __builtin_ctzll(moved); i < m; i += kKeepTokens) {
      // all that these tokens come from is read before any is written (a descriptor that is empty where
      // there is no token: nothing is asked for)
      uint8_t kb[kKeepTokens], vb[kKeepTokens];
      float sc[kKeepTokens];
#pragma unroll
      for (int e = 0; e < kKeepTokens; ++e) {
        const int f = i + e < m ? __builtin_amdgcn_readlane(from, min(i + e, 63)) : -1;
        const int64_t r = row0 + max(f, 0);
        const char* const k = reinterpret_cast<const char*>(p.k) + r * kD;
        const char* const v = reinterpret_cast<const char*>(p.v) + (r & ~(int64_t)63) * kD + (r & 63);
        kb[e] = __builtin_amdgcn_raw_buffer_load_b8(range_rsrc(k, f < 0 ? 0 : kD), lane, 0, 0);
        vb[e] = __builtin_amdgcn_raw_buffer_load_b8(range_rsrc(v, f < 0 ? 0 : kD * kS), lane * kS, 0, 0);
        sc[e] = (lane & 1 ? p.vs : p.ks)[r];
      }
#pragma unroll
      for (int e = 0; e < kKeepTokens; ++e) {
        const int t = i + e < m ? __builtin_amdgcn_readlane(to, min(i + e, 63)) : -1;
        if (t < 0) continue;
        p.k[(row0 + t) * kD + lane] = kb[e];
        p.v[(row0 + (t & ~63)) * kD + lane * kS + (t & 63)] = vb[e];
        if (lane < 2) (lane & 1 ? p.vs : p.ks)[row0 + t] = sc[e];
      }
    }
  }
  __syncthreads();  // (the workgroup's waves have read the length)
  if (threadIdx.x == 0) update_length(p.length + b, p.ticket + (int64_t)b * p.stride, (int32_t)p.per, base + m);
}

}  // namespace

hipError_t launch_window_append(const gca_window& w, const void* k, const void* v, const int32_t* lengths, int64_t T,
                                hipStream_t stream) {
  AppendParams p;
  p.src[0] = k;
  p.src[1] = v;
  p.dst[0] = static_cast<uint8_t*>(w.k);
  p.dst[1] = static_cast<uint8_t*>(w.v);
  p.scale[0] = w.k_scale;
  p.scale[1] = w.v_scale;
  p.length = w.length;
  p.ticket = w.ticket;
  p.lengths = lengths;
  p.T = T;
  p.C = w.capacity;
  p.seqs = (uint32_t)w.B;
  const bool few = T <= kFewTokens;
  p.tiles = (uint32_t)(few ? (T + 7) / 8 : tiles_of(T < w.capacity ? T : w.capacity));
  p.Hkv = (uint32_t)w.Hkv;
  p.stride = 2 * (uint32_t)w.H;
  p.items = p.Hkv * p.tiles * 2;
  // few tokens: as many waves per workgroup as go, so that one may do for a sequence and needs no ticket
  const uint32_t waves = few ? (p.items < 16 ? p.items : 16) : kAppendWaves;
  p.per = (p.items + waves - 1) / waves;
  if (!few) {  // no more workgroups than run at once: every one takes a ticket (a workgroup per 8 tiles: 34 us for 24)
    const uint32_t most = 2 * (uint32_t)device_cus() / p.seqs;
    if (p.per > most) p.per = most > 1 ? most : 1;
  }
  p.ring = w.window > 0;
  // a tile per wave and more: over all sequences' tiles, so that no workgroup is left with a long one while others are
  // through (four prompts of up to 8,192 tokens: 30.6 us for 34.8; below that one ticket for all is 1 us more)
  const bool all = !few && p.seqs > 1 && p.seqs <= 64 && p.items >= p.per * waves;
  const dim3 grid(p.seqs * p.per), block(waves * 64);
  auto run = [&](auto tag, auto i8) {
    using E = decltype(tag);
    constexpr bool I8 = decltype(i8)::value;
    auto kernel = window_append_kernel<E, I8, kMany>;
    if (few) kernel = window_append_kernel<E, I8, kFew>;
    else if (all) kernel = window_append_kernel<E, I8, kAll>;
    launch_kernel("window_append_kernel", kernel, grid, block, 0, stream, p);
  };
  if (w.dtype == GCA_BF16) w.format == GCA_INT8 ? run(__bf16{}, std::true_type{}) : run(__bf16{}, std::false_type{});
  else w.format == GCA_INT8 ? run(float{}, std::true_type{}) : run(float{}, std::false_type{});
  return take_launch_error();
}

hipError_t launch_window_keep(const gca_window& w, const int32_t* path, int64_t n, const int32_t* lengths, int64_t T,
                              hipStream_t stream) {
  KeepParams p;
  p.k = static_cast<uint8_t*>(w.k);
  p.v = static_cast<uint8_t*>(w.v);
  p.ks = w.k_scale;
  p.vs = w.v_scale;
  p.length = w.length;
  p.path = path;
  p.lengths = lengths;
  p.T = T;
  p.C = w.capacity;
  p.Hkv = (uint32_t)w.Hkv;
  p.n = (uint32_t)n;
  p.ticket = w.ticket;
  p.stride = 2 * (uint32_t)w.H;
  const uint32_t waves = p.Hkv < kKeepWaves ? p.Hkv : kKeepWaves;
  p.per = (p.Hkv + waves - 1) / waves;
  p.ring = w.window > 0;
  launch_kernel("window_keep_kernel", window_keep_kernel, dim3((unsigned)w.B * p.per), dim3(waves * 64), 0, stream, p);
  return take_launch_error();
}

}  // namespace gca
