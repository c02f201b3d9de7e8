// Device-side helpers of the 4-bit cache kernels (gfx950, wave64).
#pragma once

#include "cache4.h"
#include "common.h"

namespace stepkv {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// STEPKV_FLAG_* bits that the calls on a cache report.
constexpr uint32_t kFlagNonFinite4 = 2u, kFlagOutRows4 = 4u;

__device__ __forceinline__ float bf16_float(uint32_t b) { return __uint_as_float(b << 16); }

// Tokens of sequence s that the cache holds: lens[s] within its room.
__device__ __forceinline__ int held_tokens(const Cache4View& c, int s) {
  return min(max(c.lens[s], 0), c.cu_rows[s + 1] - c.cu_rows[s]);
}

// x[i] of an array that stays unchanged for the whole launch, read through the
// constant address space: with a wave-uniform index the load is a scalar one,
// which does not queue behind the rows that the compute unit streams.
__device__ __forceinline__ int read_const(const int32_t* x, int i) {
  return ((const __attribute__((address_space(4))) int32_t*)x)[i];
}
// held_tokens of a wave-uniform sequence, where the launch does not write lens.
__device__ __forceinline__ int held_const(const Cache4View& c, int s) {
  return min(max(read_const(c.lens, s), 0), read_const(c.cu_rows, s + 1) - read_const(c.cu_rows, s));
}

// Reports a sequence with more tokens than room (called by one wave of a launch).
__device__ __forceinline__ void report_rooms(const Cache4View& c) {
  if (c.status == nullptr) return;
  bool over = false;
  for (int s = threadIdx.x & 63; s < c.S; s += kWave)
    over |= c.lens[s] > c.cu_rows[s + 1] - c.cu_rows[s];
  if (over) atomicOr(c.status, kFlagOutRows4);
}

// Inclusive prefix sum over the wave's lanes on the vector unit (DPP row shifts
// within 16 lanes, then the row totals); the wave's total is lane 63's.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);  // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);  // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);  // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31
  return x;
}
__device__ __forceinline__ int wave_total(int scanned) {
  return __builtin_amdgcn_readlane(scanned, kWave - 1);
}

// The item `at` of a list that holds count(s) items of each sequence in order:
// its sequence, and the first item of that sequence; s_out = -1 past the
// list's end (grids are sized by bounds that the host knows). Wave-uniform.
template <typename F>
__device__ __forceinline__ void locate_item(int S, int at, F count, int& s_out, int& first_out) {
  const int lane = threadIdx.x & 63;
  int base = 0;
  for (int s0 = 0; s0 < S; s0 += kWave) {
    const int cnt = s0 + lane < S ? count(s0 + lane) : 0;
    const int incl = wave_scan(cnt);
    const int total = wave_total(incl);
    if (at < base + total) {
      const int k = __builtin_ctzll(ballot(base + incl > at));
      s_out = s0 + k;
      first_out = base + __builtin_amdgcn_readlane(incl - cnt, k);
      return;
    }
    base += total;
  }
  s_out = -1;
  first_out = base;
}

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
