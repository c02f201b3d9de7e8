// Device-side helpers of the 8-bit cache kernels (gfx950, wave64).
#pragma once

#include "cache8.h"
#include "cache_device.h"

namespace stepkv {

constexpr int kLeast8 = -117, kMost8 = 119;  // exponents of a scale

typedef short i16x2_t __attribute__((ext_vector_type(2)));

// Four codes of a word times the power of two whose exponent field s has, in
// bf16, exactly: one instruction for two. NaN codes give NaN.
__device__ __forceinline__ u32x2_t spread4(uint32_t w, float s) {
  u32x2_t r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true));
  return r;
}
__device__ __forceinline__ u32x4_t spread8(uint32_t w0, uint32_t w1, float s) {
  const u32x2_t a = spread4(w0, s), b = spread4(w1, s);
  return u32x4_t{a[0], a[1], b[0], b[1]};
}

// The codes of four bf16 values divided by the power of two in s: rounded to the
// nearest, ties to even; NaN above 464 s and for what is not finite.
__device__ __forceinline__ uint32_t round4(uint32_t x0, uint32_t x1, float s) {
  i16x2_t w = {0, 0};
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2_t, x0), s, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2_t, x1), s, true);
  return __builtin_bit_cast(uint32_t, w);
}

__device__ __forceinline__ float pow2_of(int e) { return __int_as_float((e + 127) << 23); }
// e of a scale 2^e, whatever its sign and mantissa bits hold.
__device__ __forceinline__ int exponent_of(float s) {
  return (int)((__float_as_uint(s) >> 23) & 255u) - 127;
}

// x[i] with a wave-uniform i, of an array that stays unchanged for the whole
// launch: a scalar load.
__device__ __forceinline__ float read_const(const float* x, size_t i) {
  return ((const __attribute__((address_space(4))) float*)x)[i];
}

// Index of the first scale of sequence s, whose rows start at row0.
__device__ __forceinline__ int first_block(int row0, int s) { return row0 / kBlock8 + s; }

}  // namespace stepkv
