// 8-bit numbers on the device (gfx950), shared by the chunk cache's and the token window's
// kernels: operands from e4m3 and int8 numbers, rows of new keys and values, and byte
// transposes.
#pragma once

#include "gca_device.hpp"

namespace gca {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;

__device__ __forceinline__ f32x16 mma(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(const f16x8& a, const f16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(const f16x8& a, const f16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Eight numbers (dwords x, y) as a bf16 / fp16 operand, exactly.
template <bool I8>
__device__ __forceinline__ bf16x8 to_bf16(uint32_t x, uint32_t y) {
  if constexpr (I8) {
    bf16x8 f;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      f[m] = (__bf16)(float)(int8_t)((int)x >> (8 * m));
      f[4 + m] = (__bf16)(float)(int8_t)((int)y >> (8 * m));
    }
    return f;
  } else {
    const u32x4 r = u32x4{
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, false)),
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, true)),
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, 1.f, false)),
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, 1.f, true))};
    return __builtin_bit_cast(bf16x8, r);
  }
}
// Eight e4m3 numbers times a power of two (by its exponent) as a bf16 operand: exact from 2^-117 up.
__device__ __forceinline__ bf16x8 to_bf16_times(uint32_t x, uint32_t y, float pow2) {
  const u32x4 r = u32x4{
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, pow2, false)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, pow2, true)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, pow2, false)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, pow2, true))};
  return __builtin_bit_cast(bf16x8, r);
}
template <bool I8>
__device__ __forceinline__ f16x8 to_f16(uint32_t x, uint32_t y) {
  if constexpr (I8) {
    // n + 128 in the low mantissa bits of 1024: fp16 1152 + n
    auto two = [](uint32_t u, uint32_t sel) {
      const f16x2 m = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, sel));
      return __builtin_bit_cast(uint32_t, m - f16x2{(_Float16)1152, (_Float16)1152});
    };
    x ^= 0x80808080u;
    y ^= 0x80808080u;
    return __builtin_bit_cast(
        f16x8, u32x4{two(x, 0x04010400), two(x, 0x04030402), two(y, 0x04010400), two(y, 0x04030402)});
  } else {
    const u32x4 r = u32x4{
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.f, false)),
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.f, true)),
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(y, 1.f, false)),
        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(y, 1.f, true))};
    return __builtin_bit_cast(f16x8, r);
  }
}

// Eight e4m3 numbers times 2^-9 as an fp16 operand (below 1, and exact).
__device__ __forceinline__ f16x8 to_f16_small(uint32_t x, uint32_t y) {
  constexpr float k = 0x1p-9f;
  const u32x4 r = u32x4{
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, k, false)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, k, true)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(y, k, false)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(y, k, true))};
  return __builtin_bit_cast(f16x8, r);
}

__device__ __forceinline__ void store8(__bf16* p, const float* x) {
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (__bf16)x[e];
  *reinterpret_cast<bf16x8*>(p) = r;
}
__device__ __forceinline__ void store8(float* p, const float* x) {
  reinterpret_cast<f32x4*>(p)[0] = f32x4{x[0], x[1], x[2], x[3]};
  reinterpret_cast<f32x4*>(p)[1] = f32x4{x[4], x[5], x[6], x[7]};
}

// A wave-uniform address in scalar registers.  (As a pointer to global memory: through an integer it would
// lose that, and a wait for a load that might be from elsewhere is a wait for all loads.)
template <typename T>
__device__ __forceinline__ __attribute__((address_space(1))) T* scalar_ptr(T* x) {
  return reinterpret_cast<__attribute__((address_space(1))) T*>(uniform_addr(x));
}

// One row's 8 entries of a lane.
template <typename T> struct Row8;
template <> struct Row8<__bf16> {
  u32x4 x;  // pairs of bf16
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t src, uint32_t at, int row) {
    x = __builtin_amdgcn_raw_buffer_load_b128(src, at, row, 0);
  }
  __device__ __forceinline__ float at(int c) const {
    const uint32_t w = x[c >> 1];
    return __uint_as_float((c & 1) ? (w & 0xffff0000u) : (w << 16));
  }
};
template <> struct Row8<float> {
  f32x4 lo, hi;
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t src, uint32_t at, int row) {
    lo = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(src, at, row, 0));
    hi = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(src, at + 16, row, 0));
  }
  __device__ __forceinline__ float at(int c) const { return c < 4 ? lo[c] : hi[c - 4]; }
};

// 8 x 8 bytes, row r in (x[2 r], x[2 r + 1]), transposed in place: four 4 x 4 blocks, each
// turned by two levels of byte permutes.
__device__ __forceinline__ void transpose4(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t& o0, uint32_t& o1,
                                           uint32_t& o2, uint32_t& o3) {
  // v_perm_b32(hi, lo, sel): selector 0-3 takes a byte of lo, 4-7 of hi
  const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602);
  const uint32_t cd0 = __builtin_amdgcn_perm(d, c, 0x05010400), cd1 = __builtin_amdgcn_perm(d, c, 0x07030602);
  o0 = __builtin_amdgcn_perm(cd0, ab0, 0x05040100);
  o1 = __builtin_amdgcn_perm(cd0, ab0, 0x07060302);
  o2 = __builtin_amdgcn_perm(cd1, ab1, 0x05040100);
  o3 = __builtin_amdgcn_perm(cd1, ab1, 0x07060302);
}

// Two numbers to e4m3 (round to nearest even), into one half of w.
__device__ __forceinline__ uint32_t pk_e4m3(float a, float b, uint32_t w, bool hi) {
  return hi ? (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)w, true)
            : (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)w, false);
}

}  // namespace gca
