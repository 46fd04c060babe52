// Storing chunks in the 8-bit chunk cache (gca_cache_store): every 64 x 64 tile of new keys
// or values becomes 8-bit numbers and one scale, the values' tile transposed.
//
// One wave per tile.  Lane (rg, cg) = (l / 8, l % 8) holds the 8 x 8 block of rows 8 rg ..
// and columns 8 cg ..: a load instruction takes 16 bytes of 8 rows' 128-byte lines (bf16),
// all of a tile's loads are in flight at once, the largest magnitude is one reduction over
// the wave, and the transposed tile is 8 x 8 byte blocks turned in registers (byte
// permutes), so a tile goes through no LDS and is read and written once.
//
// Bound by HBM: a bf16 tile reads 8 KiB and writes 4 KiB.  1,024 chunks of 2 sequences and 16 heads (806 MB)
// take 154 us, 5.3 TB/s in random slots; one chunk of 32 sequences and 16 heads (12.6 MB) 4.4 us.
#include "cache_plan.hpp"
#include "gca_device.hpp"
#include "gca_launch.hpp"
#include "numbers8.hpp"

namespace gca {
namespace {

constexpr int kStoreThreads = 256;

struct StoreParams {
  const int32_t* slots;
  const int32_t* lengths;
  int32_t* tokens;
  uint32_t tiles, items;  // 2 B Hkv n tiles, then B Hr n landmark rows (none without lmk)
  uint32_t n, Hkv, Hr;
  int32_t C;
  uint32_t claimed;  // `tokens` says which chunk a slot takes
  uint32_t seqs;
  int row_bytes;  // of a landmark row
  const void* src[2];  // new keys, new values
  uint8_t* dst[2];
  float* scale[2];
  const void* lmk;
  void* lmk_dst;
};

// A slot that a sequence names twice takes the last chunk.  Up to kClaimFrom chunks per sequence every
// tile's wave looks through the slots behind its own; a longer call, where that would grow as n^2, has
// `tokens` hold kClaim + the last chunk's number while it runs, in three small launches around the store
// (clear, claim by the largest number, length).  A length is at most 64, so a chunk never
// takes another's length for its own claim.  Looking / claiming, bf16, us: 2 sequences of 16 heads, 256
// chunks each 35 / 45, 512 84 / 86, 1,024 161 / 154, 2,048 355 / 293; 16,384 chunks of 8 heads 2,045 / 619.
constexpr int kClaim = 128;
constexpr int64_t kClaimFrom = 512;

__device__ __forceinline__ uint32_t max_u64(uint32_t x) {
  x = max(x, dpp<kDppXor1>(x));
  x = max(x, dpp<kDppXor2>(x));
  x = max(x, dpp<kDppRor4>(x));
  x = max(x, dpp<kDppRor8>(x));
  uint32_t a, b;
  pair16(x, a, b);
  x = max(a, b);
  pair32(x, a, b);
  return max(a, b);
}

// Chunks with tokens among n, of a sequence of `total` new tokens.
__device__ __forceinline__ uint32_t with_tokens(uint32_t n, int total) {
  const int64_t x = ((int64_t)total + kS - 1) / kS;
  return (uint32_t)(x < 0 ? 0 : x < n ? x : n);
}

// Whether a later chunk with tokens of the sequence, before `last`, names chunk i's slot too.
__device__ __forceinline__ bool replaced(const StoreParams& p, uint32_t b, uint32_t i, uint32_t last, int slot,
                                         int lane) {
  if (i + 1 >= last) return false;
  if (p.claimed) return p.tokens[(int64_t)b * p.C + slot] != kClaim + (int)i;
  const int32_t* slots = p.slots + (int64_t)b * p.n;
  for (uint32_t e = i + 1; e < last; e += 64)
    if (__ballot(e + lane < last && slots[e + lane < last ? e + lane : i] == slot)) return true;
  return false;
}

template <typename T, bool I8>
__device__ __forceinline__ void store_tile(const StoreParams& p, uint32_t item, int lane) {
  // item = ((b Hkv + h) n + i) 2 + which
  const uint32_t which = item & 1, t = item >> 1;
  // (the quotients are formed on the vector unit: back to scalar registers, and with them every address)
  const uint32_t bh = __builtin_amdgcn_readfirstlane(t / p.n), i = t - bh * p.n;
  const uint32_t b = __builtin_amdgcn_readfirstlane(bh / p.Hkv);
  int slot = p.slots[(int64_t)b * p.n + i];
  int total = p.lengths ? p.lengths[b] : 0;
  slot = __builtin_amdgcn_readfirstlane(slot);
  total = __builtin_amdgcn_readfirstlane(total);
  const int64_t len64 = p.lengths ? (int64_t)total - 64 * (int64_t)i : kS;
  const int len = (int)(len64 < kS ? len64 : kS);
  if (len <= 0 || slot < 0 || slot >= p.C) return;
  const int rg = lane >> 3, cg = lane & 7;
  Row8<T> x[8];
  // (rows behind the last token lie past the descriptor's end and read as zeros)
  constexpr int kRow = kD * (int)sizeof(T);
  const __amdgpu_buffer_rsrc_t src =
      range_rsrc(reinterpret_cast<const char*>(p.src[which]) + (int64_t)t * (kS * kRow), (uint32_t)(len * kRow));
  const uint32_t at = rg * 8 * kRow + cg * 8 * (int)sizeof(T);
#pragma unroll
  for (int r = 0; r < 8; ++r) x[r].load(src, at, r * kRow);
  // a later chunk of the sequence that is stored in the same slot replaces this one
  if (replaced(p, b, i, p.lengths ? with_tokens(p.n, total) : p.n, slot, lane)) return;

  // the largest finite magnitude, as its bits
  uint32_t top = 0;
  bool odd = false, nan = false;  // anything not finite; NaN
  if constexpr (sizeof(T) == 2) {
    // bf16 pairs: magnitudes order as integers
    typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
    u16x2 m = u16x2{0, 0};
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int c = 0; c < 4; ++c) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x[r].x[c] & 0x7fff7fffu));
    top = (uint32_t)max(m[0], m[1]) << 16;
  } else {
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int c = 0; c < 8; ++c) top = max(top, __float_as_uint(x[r].at(c)) & 0x7fffffffu);
  }
  top = max_u64(top);
  if (top >= 0x7f800000u) {  // wave-uniform
    odd = true;
    nan = top > 0x7f800000u;
    top = 0;
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint32_t u = __float_as_uint(x[r].at(c)) & 0x7fffffffu;
        top = max(top, u < 0x7f800000u ? u : 0u);
      }
    top = max_u64(top);
  }

  uint32_t w[16];  // row r: w[2 r], w[2 r + 1]
  float scale;
  if constexpr (I8) {
    const float amax = fmaxf(__uint_as_float(top), 0x1p-100f);
    scale = nan ? __builtin_nanf("") : amax * (1.f / 127.f);
    const float inv = (1.f / amax) * 127.f;  // |x| inv <= 127 (1 + 3 roundings): 127 at most once rounded
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        uint32_t o = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float y = x[r].at(4 * q + c) * inv;
          if (odd) y = fminf(fmaxf(y, -127.f), 127.f);
          o |= ((uint32_t)(int)__builtin_rintf(y) & 0xffu) << (8 * c);
        }
        w[2 * r + q] = o;
      }
  } else {
    // 448 = 1.75 x 2^8: the least power of two s with amax / s <= 448 (at least 2^-126)
    const int e = max((int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), 1);
    scale = __uint_as_float((uint32_t)e << 23);
    const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        uint32_t o = 0;
#pragma unroll
        for (int c = 0; c < 4; c += 2) {
          float y0 = x[r].at(4 * q + c) * inv, y1 = x[r].at(4 * q + c + 1) * inv;
          if (odd) {  // infinities (a comparison with NaN is false)
            if (__builtin_fabsf(y0) > 448.f) y0 = __builtin_copysignf(448.f, y0);
            if (__builtin_fabsf(y1) > 448.f) y1 = __builtin_copysignf(448.f, y1);
          }
          o = pk_e4m3(y0, y1, o, c != 0);
        }
        w[2 * r + q] = o;
      }
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
  const int64_t tile = (int64_t)bh * p.C + slot;
  // keys: row 8 rg + r, bytes 8 cg ..; values: column 8 cg + r, bytes 8 rg ..
  uint8_t* dst = p.dst[which] + tile * (kS * kD) + (which ? cg * 8 * kS + rg * 8 : rg * 8 * kD + cg * 8);
#pragma unroll
  for (int r = 0; r < 8; ++r) *reinterpret_cast<u32x2*>(dst + r * 64) = u32x2{w[2 * r], w[2 * r + 1]};
  if (lane == 0) {
    p.scale[which][tile] = scale;
    if (which == 0 && bh == b * p.Hkv && !p.claimed) p.tokens[(int64_t)b * p.C + slot] = len;
  }
}

// Landmark row i of (sequence, retrieval head) into the same slot.
__device__ __forceinline__ void store_landmark(const StoreParams& p, uint32_t item, int lane) {
  const uint32_t bhr = __builtin_amdgcn_readfirstlane(item / p.n), i = item - bhr * p.n;
  const uint32_t b = __builtin_amdgcn_readfirstlane(bhr / p.Hr);
  const int slot = p.slots[(int64_t)b * p.n + i];
  const uint32_t last = p.lengths ? with_tokens(p.n, p.lengths[b]) : p.n;
  if (i >= last || slot < 0 || slot >= p.C || replaced(p, b, i, last, slot, lane)) return;
  const char* src = reinterpret_cast<const char*>(p.lmk) + (int64_t)item * p.row_bytes;
  char* dst = reinterpret_cast<char*>(p.lmk_dst) + ((int64_t)bhr * p.C + slot) * p.row_bytes;
  for (int x = lane * 16; x < p.row_bytes; x += 1024)
    *reinterpret_cast<u32x4*>(dst + x) = *reinterpret_cast<const u32x4*>(src + x);
}

// STEP 0, 1: before the store, slots named cleared, then claimed; 2: after it, the lengths.
template <int STEP>
__global__ __launch_bounds__(kStoreThreads) void cache_claim_kernel(StoreParams p) {
  const uint32_t at = blockIdx.x * kStoreThreads + threadIdx.x;  // b n + i
  const uint32_t b = at / p.n, i = at - b * p.n;
  if (b >= p.seqs || i >= (p.lengths ? with_tokens(p.n, p.lengths[b]) : p.n)) return;
  const int slot = p.slots[at];
  if (slot < 0 || slot >= p.C) return;
  int32_t* tokens = p.tokens + (int64_t)b * p.C + slot;
  if constexpr (STEP == 0) *tokens = 0;
  if constexpr (STEP == 1) atomicMax(tokens, kClaim + (int)i);
  if constexpr (STEP == 2) {
    const int64_t len = p.lengths ? (int64_t)p.lengths[b] - 64 * (int64_t)i : kS;
    if (*tokens == kClaim + (int)i) *tokens = (int)(len < kS ? len : kS);
  }
}

template <typename T, bool I8>
__global__ __launch_bounds__(kStoreThreads) void cache_store_kernel(StoreParams p) {
  const uint32_t item =
      __builtin_amdgcn_readfirstlane(blockIdx.x * (kStoreThreads / 64) + (threadIdx.x >> 6));
  const int lane = threadIdx.x & 63;
  if (item < p.tiles) store_tile<T, I8>(p, item, lane);
  else if (item < p.items) store_landmark(p, item - p.tiles, lane);
}

}  // namespace

hipError_t launch_cache_store(const gca_cache& c, const void* k, const void* v, const void* lmk, const int32_t* slots,
                              const int32_t* lengths, int64_t n, hipStream_t stream) {
  StoreParams p;
  p.src[0] = k;
  p.src[1] = v;
  p.dst[0] = static_cast<uint8_t*>(c.k);
  p.dst[1] = static_cast<uint8_t*>(c.v);
  p.scale[0] = c.k_scale;
  p.scale[1] = c.v_scale;
  p.lmk = lmk;
  p.lmk_dst = c.lmk;
  p.slots = slots;
  p.lengths = lengths;
  p.tokens = c.tokens;
  p.tiles = (uint32_t)(2 * (int64_t)c.B * c.Hkv * n);
  p.items = p.tiles + (lmk ? (uint32_t)((int64_t)c.B * c.Hr * n) : 0u);
  p.n = (uint32_t)n;
  p.Hkv = c.Hkv;
  p.Hr = c.Hr;
  p.C = (int)c.capacity;
  p.row_bytes = c.D * (c.dtype == GCA_BF16 ? 2 : 4);
  const int per = kStoreThreads / 64;
  const dim3 grid((p.items + per - 1) / per), block(kStoreThreads);
  const bool i8 = c.format == GCA_INT8;
  p.claimed = n > kClaimFrom;
  p.seqs = (uint32_t)c.B;
  const dim3 claims((unsigned)((c.B * n + kStoreThreads - 1) / kStoreThreads));
  if (p.claimed) {
    launch_kernel("cache_claim_kernel", cache_claim_kernel<0>, claims, block, 0, stream, p);
    launch_kernel("cache_claim_kernel", cache_claim_kernel<1>, claims, block, 0, stream, p);
  }
  if (c.dtype == GCA_BF16)
    launch_kernel("cache_store_kernel", i8 ? cache_store_kernel<__bf16, true> : cache_store_kernel<__bf16, false>,
                  grid, block, 0, stream, p);
  else
    launch_kernel("cache_store_kernel", i8 ? cache_store_kernel<float, true> : cache_store_kernel<float, false>, grid,
                  block, 0, stream, p);
  if (p.claimed) launch_kernel("cache_claim_kernel", cache_claim_kernel<2>, claims, block, 0, stream, p);
  return take_launch_error();
}

}  // namespace gca
