// Device-side helpers of the quantised caches' kernels (gfx950, wave64).
#pragma once

#include "common.h"

namespace stepkv {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((__vector_size__(4 * sizeof(float))));

// STEPKV_FLAG_* bits that the calls on a cache report.
constexpr uint32_t kFlagNonFinite4 = 2u, kFlagOutRows4 = 4u;

__device__ __forceinline__ float bf16_float(uint32_t b) { return __uint_as_float(b << 16); }

// Tokens of sequence s that a cache holds: lens[s] within its room.
template <typename View>
__device__ __forceinline__ int held_tokens(const View& c, int s) {
  return min(max(c.lens[s], 0), c.cu_rows[s + 1] - c.cu_rows[s]);
}

// x[i] of an array that stays unchanged for the whole launch, read through the
// constant address space: with a wave-uniform index the load is a scalar one,
// which does not queue behind the rows that the compute unit streams.
__device__ __forceinline__ int read_const(const int32_t* x, int i) {
  return ((const __attribute__((address_space(4))) int32_t*)x)[i];
}
// held_tokens of a wave-uniform sequence, where the launch does not write lens.
template <typename View>
__device__ __forceinline__ int held_const(const View& c, int s) {
  return min(max(read_const(c.lens, s), 0), read_const(c.cu_rows, s + 1) - read_const(c.cu_rows, s));
}

// Reports a sequence with more tokens than room (called by one wave of a launch).
template <typename View>
__device__ __forceinline__ void report_rooms(const View& c) {
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

// ---------------------------------------------------------------- attention
// The value of lane l ^ 16 and of lane l ^ 32 (permlane swaps).
__device__ __forceinline__ float xor16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return __uint_as_float(((threadIdx.x >> 4) & 1) ? r[0] : r[1]);
}
__device__ __forceinline__ float xor32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return __uint_as_float(((threadIdx.x >> 5) & 1) ? r[0] : r[1]);
}

// Eight probabilities as bf16 operands whose sum they are, exactly: three parts
// of 8 bits of the significand each, by truncation (the rest is exact in fp32).
// Groups of at most 5 heads lie in the operand's 16 rows three times (C = 3), and
// each copy takes its own part: one product instead of three (8 layers x 8 heads
// x 131071 rows, G 4: 200 -> 187 us; two copies of at most 8 heads and two
// products: no faster).
template <int C>
struct Parts {
  static constexpr int N = 3 / C;
  bf16x8_t x[N];
};
__device__ __forceinline__ uint32_t upper(uint32_t b, uint32_t a) {  // the upper halves of a, b
  return __builtin_amdgcn_perm(b, a, 0x07060302u);
}
// x less its bits in mask (the upper half, or none).
__device__ __forceinline__ uint32_t below(uint32_t x, uint32_t mask) {
  return __float_as_uint(__uint_as_float(x) - __uint_as_float(x & mask));
}
template <int C>
__device__ __forceinline__ Parts<C> split_parts(const float (&p)[8], int copy) {
  constexpr uint32_t F = 0xffff0000u;
  const uint32_t m1 = copy >= 1 ? F : 0u, m2 = copy >= 2 ? F : 0u;
  u32x4_t w[Parts<C>::N];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = __float_as_uint(p[2 * i]), b = __float_as_uint(p[2 * i + 1]);
    if constexpr (C == 3) {
      w[0][i] = upper(below(below(b, m1), m2), below(below(a, m1), m2));
    } else {
      const uint32_t a1 = below(a, F), b1 = below(b, F);
      w[0][i] = upper(b, a);
      w[1][i] = upper(b1, a1);
      w[2][i] = upper(below(b1, F), below(a1, F));
    }
  }
  Parts<C> r;
#pragma unroll
  for (int k = 0; k < Parts<C>::N; ++k) r.x[k] = __builtin_bit_cast(bf16x8_t, w[k]);
  return r;
}

}  // namespace stepkv
