// Device-side helpers of the 4-bit cache kernels (gfx950, wave64).
#pragma once

#include "cache4.h"
#include "cache_device.h"

namespace stepkv {

// Two elements (byte SEL of w) times the power of two whose exponent field s
// has (its sign and mantissa are not looked at; exponent 255 gives NaN), in
// bf16, exactly: one instruction.
template <int SEL>
__device__ __forceinline__ uint32_t spread2(uint32_t w, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, SEL));
}

// The eight values of one word of codes.
__device__ __forceinline__ u32x4_t spread8(uint32_t w, float s) {
  u32x4_t r;
  r[0] = spread2<0>(w, s);
  r[1] = spread2<1>(w, s);
  r[2] = spread2<2>(w, s);
  r[3] = spread2<3>(w, s);
  return r;
}

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

}  // namespace stepkv
