// Appending tokens to the 8-bit token window (gca_window_append), and keeping an accepted path of
// the newest ones (gca_window_keep).
//
// Append.  Every token's 64 keys, and its 64 values, become 8-bit numbers with one scale; the values are
// kept transposed per 64 rows.  One wave per 64 positions that share a tile of rows, and per keys or
// values: lane (rg, cg) = (l / 8, l % 8) holds the 8 x 8 block of rows 8 rg .. and columns 8 cg .., so that a
// row's largest magnitude is a reduction over 8 lanes and the values' tile is byte blocks turned in
// registers.  A tile that new tokens fill only in part (a single token's, a prompt's first and last)
// writes its own rows and no others.
//
// Keep.  One wave per (sequence, cached head); lane d moves key d and value d of each token.  As a path
// ascends, token i comes from a place at or behind i, so what later tokens come from is never overwritten.
#include "gca_device.hpp"
#include "gca_launch.hpp"
#include "numbers8.hpp"
#include "window_plan.hpp"

namespace gca {
namespace {

constexpr int kAppendWaves = 4;
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
  uint32_t tiles, Hkv, stride;  // stride: tickets of a sequence
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

template <typename T, bool I8>
__device__ __forceinline__ void append_tile(const AppendParams& p, uint32_t b, uint32_t item, int64_t length,
                                            int64_t n, int lane) {
  // item = (h tiles + t) 2 + which
  const uint32_t which = item & 1;
  const uint32_t h = __builtin_amdgcn_readfirstlane((item >> 1) / p.tiles), t = (item >> 1) - h * p.tiles;
  // tokens that are kept: [i0, i1); the tile's: from position `first`
  const int64_t i0 = p.ring && n > p.C ? n - p.C : 0;
  const int64_t i1 = p.ring || length + n <= p.C ? n : p.C - length;
  const int64_t first = ((length + i0) / kS + t) * kS;
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
  for (int r = 0; r < 8; ++r) {
    uint32_t top = 0;
#pragma unroll
    for (int c = 0; c < 8; ++c) top = max(top, __float_as_uint(x[r].at(c)) & 0x7fffffffu);
    top = max_row8(top);
    const bool odd = top >= 0x7f800000u, nan = top > 0x7f800000u;
    if (__any(odd)) {  // the largest finite magnitude
      uint32_t fin = 0;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint32_t u = __float_as_uint(x[r].at(c)) & 0x7fffffffu;
        fin = max(fin, u < 0x7f800000u ? u : 0u);
      }
      top = max_row8(fin);
    }
    if constexpr (I8) {
      const float amax = fmaxf(__uint_as_float(top), 0x1p-100f);
      scale[r] = amax / 127.f;
      const float inv = 127.f / amax;  // |x| inv <= 127 (1 + 2 roundings): 127 at most once rounded
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        uint32_t o = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float y = x[r].at(4 * q + c) * inv;
          if (odd) y = y == y ? fminf(fmaxf(y, -127.f), 127.f) : 0.f;
          o |= ((uint32_t)(int)__builtin_rintf(y) & 0xffu) << (8 * c);
        }
        w[2 * r + q] = o;
      }
    } else {
      // 448 = 1.75 x 2^8: the least power of two s with amax / s <= 448 (at least 2^-126)
      const int e = max((int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), 1);
      scale[r] = __uint_as_float((uint32_t)e << 23);
      const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        uint32_t o = 0;
#pragma unroll
        for (int c = 0; c < 4; c += 2) {
          float y0 = x[r].at(4 * q + c) * inv, y1 = x[r].at(4 * q + c + 1) * inv;
          if (odd) {  // infinities (a comparison with NaN is false)
            if (__builtin_fabsf(y0) > 448.f) y0 = __builtin_copysignf(448.f, y0);
            if (__builtin_fabsf(y1) > 448.f) y1 = __builtin_copysignf(448.f, y1);
            if (which) {  // (a value's number is never NaN: it would reach rows that do not see it)
              y0 = y0 == y0 ? y0 : 0.f;
              y1 = y1 == y1 ? y1 : 0.f;
            }
          }
          o = pk_e4m3(y0, y1, o, c != 0);
        }
        w[2 * r + q] = o;
      }
    }
    if (nan) scale[r] = __builtin_nanf("");
  }

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
  const int64_t row0 = bh * p.C + (p.ring ? first % p.C : first);
  // keys: row 8 rg + r, bytes 8 cg ..; values: column 8 cg + r, bytes 8 rg ..
  uint8_t* dst = p.dst[which] + row0 * kD + (which ? cg * 8 * kS + rg * 8 : rg * 8 * kD + cg * 8);
  const int from = max((int)lo - 8 * rg, 0), to = min((int)hi - 8 * rg, 8);  // this lane's rows
  if (which && (from > 0 || to < 8)) {
    for (int r = from; r < to; ++r)
#pragma unroll
      for (int c = 0; c < 8; ++c)
        dst[c * kS + r] = (uint8_t)((r < 4 ? w[2 * c] : w[2 * c + 1]) >> (8 * (r & 3)));
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

// The last workgroup of a sequence to have read its length writes the new one: every workgroup takes a
// ticket behind its read, and who takes the last knows that nobody reads any more.
template <typename T, bool I8>
__global__ __launch_bounds__(kAppendWaves * 64) void window_append_kernel(AppendParams p) {
  __shared__ int32_t old;
  const uint32_t b = blockIdx.x / p.per, part = blockIdx.x - b * p.per;
  int32_t drawn = 0;
  if (threadIdx.x == 0) {
    int32_t len = p.length[b];
    old = len;
    if (p.per > 1) {
      asm volatile("" : "+v"(len)::"memory");  // (the value is here before the ticket is asked for)
      drawn = __hip_atomic_fetch_add(p.ticket + (int64_t)b * p.stride, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  __syncthreads();
  const int64_t length = max(old, 0);
  const int64_t n = new_tokens(p.lengths, b, p.T);
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t item = part * kAppendWaves + wave;
  if (item < p.items) append_tile<T, I8>(p, b, item, length, n, threadIdx.x & 63);
  if (threadIdx.x == 0 && drawn == (int32_t)p.per - 1) {
    const int64_t len = length + n;
    p.length[b] = (int32_t)(len < 0x7fffffff ? len : 0x7fffffff);
    if (p.per > 1) __hip_atomic_store(p.ticket + (int64_t)b * p.stride, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

struct KeepParams {
  uint8_t* k;
  uint8_t* v;
  float* ks;
  float* vs;
  int32_t* length;
  const int32_t* path;
  const int32_t* lengths;
  int64_t T, C;
  uint32_t Hkv, n;
  int ring;
};

constexpr int kKeepWaves = 8;

// One workgroup per sequence, its waves taking the cached heads in turn.
__global__ __launch_bounds__(kKeepWaves * 64) void window_keep_kernel(KeepParams p) {
  const uint32_t b = blockIdx.x;
  const int lane = threadIdx.x & 63;
  const int64_t n = new_tokens(p.lengths, b, p.T);
  const int64_t length = max(p.length[b], 0);
  // lane i: entry i, in the path if every entry up to it is larger than the one before
  const int mine = lane < (int)p.n ? p.path[(int64_t)b * p.n + lane] : -1;
  const int left = __shfl_up(mine, 1);  // (by every lane: one that is not active has nothing to give)
  const uint64_t good = __ballot(mine > (lane ? left : -1) && mine < n);
  const int m = good == ~0ull ? 64 : __builtin_ctzll(~good);
  __syncthreads();  // every wave has read the length
  const int64_t base = length > n ? length - n : 0;
  if (threadIdx.x == 0) p.length[b] = (int32_t)(base + m);
  // entries that name their own place lead the path and stay
  const uint64_t moved = __ballot(lane < m && mine != lane);
  if (moved == 0) return;
  const int first = __builtin_ctzll(moved);
  auto row_of = [&](int64_t pos) { return p.ring ? pos % p.C : pos; };
  for (uint32_t h = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); h < p.Hkv; h += kKeepWaves) {
    const int64_t row0 = ((int64_t)b * p.Hkv + h) * p.C;
    // four tokens at a time: all that they come from is read before any is written
    for (int i = first; i < m; i += 4) {
      uint8_t kb[4], vb[4];
      float sc[4];
      int64_t to[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int at = min(i + e, m - 1);
        const int64_t from = row_of(base + __builtin_amdgcn_readlane(mine, at));
        to[e] = row_of(base + at);
        // (a row past the capacity is neither there nor wanted)
        if (i + e >= m || from >= p.C || to[e] >= p.C) to[e] = -1;
        const int64_t f = to[e] < 0 ? 0 : from;
        kb[e] = p.k[(row0 + f) * kD + lane];
        vb[e] = p.v[(row0 + (f & ~63)) * kD + lane * kS + (f & 63)];
        sc[e] = lane < 2 ? (lane ? p.vs : p.ks)[row0 + f] : 0.f;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (to[e] < 0) continue;
        p.k[(row0 + to[e]) * kD + lane] = kb[e];
        p.v[(row0 + (to[e] & ~63)) * kD + lane * kS + (to[e] & 63)] = vb[e];
        if (lane < 2) (lane ? p.vs : p.ks)[row0 + to[e]] = sc[e];
      }
    }
  }
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
  p.tiles = (uint32_t)tiles_of(T < w.capacity ? T : w.capacity);
  p.Hkv = (uint32_t)w.Hkv;
  p.stride = 2 * (uint32_t)w.H;
  p.items = p.Hkv * p.tiles * 2;
  p.per = (p.items + kAppendWaves - 1) / kAppendWaves;
  p.ring = w.window > 0;
  const dim3 grid(p.seqs * p.per), block(kAppendWaves * 64);
  const bool i8 = w.format == GCA_INT8;
  if (w.dtype == GCA_BF16)
    launch_kernel("window_append_kernel", i8 ? window_append_kernel<__bf16, true> : window_append_kernel<__bf16, false>,
                  grid, block, 0, stream, p);
  else
    launch_kernel("window_append_kernel", i8 ? window_append_kernel<float, true> : window_append_kernel<float, false>,
                  grid, block, 0, stream, p);
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
  p.ring = w.window > 0;
  launch_kernel("window_keep_kernel", window_keep_kernel, dim3((unsigned)w.B), dim3(kKeepWaves * 64), 0, stream, p);
  return take_launch_error();
}

}  // namespace gca
