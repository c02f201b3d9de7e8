// Writing and reading the 4-bit cache (the format: include/stepkv_cache4.h).
//
// write4_kernel quantises bf16 rows into cache rows, gathered by the retained
// positions of a boundary or appended token by token; read4_kernel gives rows
// back in bf16. Both are bound by memory: 4d bytes of bf16 and d + d/16 bytes
// of codes and scales a row (K and V), a handful of operations a value. The
// conversions are one instruction per two values (their rounding, ties to the
// even code and saturation at 6, is the format's).
#include "cache4_device.h"

namespace stepkv {
namespace {

constexpr int kThreads = 256;

// max(x, x of lane ^ 1) and ^ 2 (quad permutes): the maximum of four lanes.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true));
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true));
}

// min and max that keep a NaN.
__device__ __forceinline__ float min_nan(float a, float b) { return a < b || a != a ? a : b; }
__device__ __forceinline__ float max_nan(float a, float b) { return a > b || a != a ? a : b; }

// Eight values of a group (the other 24 in the other lanes of the quad):
// their codes, and the group's scale byte. With the largest magnitude
// 1.m * 2^E in bf16 bits (E and the 7 bits of m), max <= 7 * 2^e means
// e = E - 2 for 1.m <= 1.75 (m <= 96) and E - 1 above: a carry into E.
__device__ __forceinline__ uint32_t quantise8(u32x4_t x, uint32_t& byte) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    top = max(top, max(x[i] & 0x7fffu, (x[i] >> 16) & 0x7fffu));
  top = quad_max(top);
  if (top >= 0x7f80u) {  // a NaN or an infinity in the group
    byte = 255u;
    return 0u;
  }
  byte = (uint32_t)min(max((int)((top + 31u) >> 7) - 2, 3), 252);
  const float s = scale_of(byte);
  // (a bit cast of a vector's element takes the vector's first: elements are copied)
  const uint32_t x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, x0), s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, x1), s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, x2), s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, x3), s, 3);
  return w;
}

// The tokens [j0, j1) of sequence s that a call writes (j0 may be negative:
// more new tokens than the sequence has), and the source row of token j0.
__device__ __forceinline__ void span_of(const Write4Args& a, int s, int& j0, int& j1, int& src0) {
  const int room = a.c.cu_rows[s + 1] - a.c.cu_rows[s];
  src0 = a.cu_src[s];
  if (a.idx) {
    j0 = 0;
    j1 = min(min(a.cu_retained[s + 1] - a.cu_retained[s], a.cu_src[s + 1] - src0), room);
  } else {
    const int len = max(a.c.lens[s], 0);
    j0 = len - max(a.cu_src[s + 1] - src0, 0);
    j1 = min(len, room);
  }
}

// One workgroup per (layer, KV head, block of 64 tokens): a lane holds 16
// bytes (8 channels) of a row, a quad of lanes a group. The block's bounds of
// K are taken from the values as quantised.
template <int D>
__global__ __launch_bounds__(kThreads) void write4_kernel(Write4Args a) {
  constexpr int PR = D / 8;             // pieces of 8 channels a row
  constexpr int RP = kThreads / PR;     // rows a pass
  constexpr int NP = kBlock4 / RP;      // passes
  constexpr int NS = D / kGroup4;
  constexpr int NWV = kThreads / kWave;
  __shared__ float red[NWV][2][D];
  const int tid = threadIdx.x;
  const Cache4View& c = a.c;
  if (blockIdx.x == 0 && tid == 0) {
    if (a.idx) {
      bool over = false;
      for (int s = 0; s < c.S; ++s) {
        const int n = max(a.cu_retained[s + 1] - a.cu_retained[s], 0);
        c.lens[s] = n;
        over |= n > c.cu_rows[s + 1] - c.cu_rows[s];
      }
      if (over && c.status) atomicOr(c.status, kFlagOutRows4);
    } else {
      report_rooms(c);
    }
  }
  if (a.nblocks == 0) return;
  const int lh = blockIdx.x / a.nblocks;
  const int l = lh / c.H, h = lh - l * c.H;
  int s, first;
  locate_item(c.S, (int)(blockIdx.x - lh * a.nblocks), [&](int sq) {
    int j0, j1, src0;
    span_of(a, sq, j0, j1, src0);
    j0 = max(j0, 0);
    return j1 > j0 ? (j1 - 1) / kBlock4 - j0 / kBlock4 + 1 : 0;
  }, s, first);
  if (s < 0) return;  // past the last block: uniform over the workgroup
  int j0, j1, src0;
  span_of(a, s, j0, j1, src0);
  const int blk = max(j0, 0) / kBlock4 + ((int)(blockIdx.x - lh * a.nblocks) - first);
  const int seq_rows = a.idx ? a.cu_src[s + 1] - src0 : 0;
  const int32_t* __restrict__ idx =
      a.idx ? a.idx + (a.shared_idx ? 0 : (size_t)lh * a.nsrc) + src0 : nullptr;
  const int sub = tid / PR, piece = tid % PR;
  int src[NP];  // source row, or -1
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int j = blk * kBlock4 + p * RP + sub;
    src[p] = -1;
    if (j >= j0 && j < j1) {
      if (idx) {
        const int pos = idx[j];
        if (pos >= 0 && pos < seq_rows) src[p] = src0 + pos;
      } else if (src0 + (j - j0) >= 0 && src0 + (j - j0) < a.nsrc) {
        src[p] = src0 + (j - j0);
      }
    }
  }
  const uint16_t* __restrict__ kb = a.k + l * a.k_layer + h * a.k_head + 8 * piece;
  const uint16_t* __restrict__ vb = a.v + l * a.v_layer + h * a.v_head + 8 * piece;
  u32x4_t kx[NP], vx[NP];
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    kx[p] = vx[p] = u32x4_t{};
    if (src[p] < 0) continue;
    kx[p] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(kb + src[p] * a.k_row));
    vx[p] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(vb + src[p] * a.v_row));
  }
  const size_t row0 = (size_t)lh * c.rows + c.cu_rows[s] + (size_t)blk * kBlock4;
  float lo[8], hi[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo[i] = INFINITY;
    hi[i] = -INFINITY;
  }
  uint32_t flags = 0;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    uint32_t kbyte, vbyte;  // every lane: the quad exchanges need all four
    const uint32_t kw = quantise8(kx[p], kbyte), vw = quantise8(vx[p], vbyte);
    if (src[p] < 0) continue;
    if (kbyte == 255u || vbyte == 255u) flags |= kFlagNonFinite4;
    const size_t row = row0 + p * RP + sub;
    reinterpret_cast<uint32_t*>(c.k_codes + row * (D / 2))[piece] = kw;
    reinterpret_cast<uint32_t*>(c.v_codes + row * (D / 2))[piece] = vw;
    if (piece % 4 == 0) {
      c.k_scales[row * NS + piece / 4] = (uint8_t)kbyte;
      c.v_scales[row * NS + piece / 4] = (uint8_t)vbyte;
    }
    if (c.k_bounds) {
      const u32x4_t y = spread8(kw, scale_of(kbyte));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float y0 = bf16_float(y[i] & 0xffffu), y1 = bf16_float(y[i] >> 16);
        lo[2 * i] = min_nan(lo[2 * i], y0);
        hi[2 * i] = max_nan(hi[2 * i], y0);
        lo[2 * i + 1] = min_nan(lo[2 * i + 1], y1);
        hi[2 * i + 1] = max_nan(hi[2 * i + 1], y1);
      }
    }
  }
  report_flags(c.status, flags);
  if (!c.k_bounds) return;
  // over the rows of the wave (lanes of one piece), then over the waves
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int off = PR; off < kWave; off <<= 1) {
      lo[i] = min_nan(lo[i], __shfl_xor(lo[i], off, kWave));
      hi[i] = max_nan(hi[i], __shfl_xor(hi[i], off, kWave));
    }
  if ((tid & 63) < PR) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      red[tid >> 6][0][8 * piece + i] = lo[i];
      red[tid >> 6][1][8 * piece + i] = hi[i];
    }
  }
  __syncthreads();
  uint16_t* __restrict__ bounds =
      c.k_bounds + ((size_t)lh * c.nblk + c.cu_rows[s] / kBlock4 + s + blk) * 2 * D;
  const bool opened = blk * kBlock4 >= j0;  // the block's first token is among the new ones
  if (tid < D) {
    const int which = tid / (D / 2), ch = 2 * (tid % (D / 2));
    float x0 = red[0][which][ch], x1 = red[0][which][ch + 1];
    auto join = [&](float y0, float y1) {
      x0 = which ? max_nan(x0, y0) : min_nan(x0, y0);
      x1 = which ? max_nan(x1, y1) : min_nan(x1, y1);
    };
#pragma unroll
    for (int w = 1; w < NWV; ++w) join(red[w][which][ch], red[w][which][ch + 1]);
    uint32_t* at = reinterpret_cast<uint32_t*>(bounds + which * D + ch);
    if (!opened) join(bf16_float(*at & 0xffffu), bf16_float(*at >> 16));
    // exact: the values are bf16
    *at = (__float_as_uint(x0) >> 16) | (__float_as_uint(x1) & 0xffff0000u);
  }
}

__global__ void advance4_kernel(Cache4View c, const int32_t* __restrict__ cu_new) {
  for (int s = blockIdx.x * blockDim.x + threadIdx.x; s < c.S; s += gridDim.x * blockDim.x)
    c.lens[s] += max(cu_new[s + 1] - cu_new[s], 0);
}

// A thread per 8 channels of a row: one word of codes and a scale byte in, 16
// bytes out, several rows in flight per thread.
constexpr int kReadPasses = 2;

template <int D>
__global__ __launch_bounds__(kThreads) void read4_kernel(Read4Args a) {
  constexpr int PR = D / 8;
  constexpr int RP = kThreads / PR;
  constexpr int RB = RP * kReadPasses;
  constexpr int NS = D / kGroup4;
  const Cache4View& c = a.c;
  const int nb = (a.out_rows + RB - 1) / RB;
  const int lh = blockIdx.x / nb, rb = blockIdx.x - lh * nb;
  const int total = min(a.out_rows, a.cu_out[c.S]);
  const int sub = threadIdx.x / PR, piece = threadIdx.x % PR;
  int64_t row[kReadPasses];  // cache row, or -1
#pragma unroll
  for (int p = 0; p < kReadPasses; ++p) {
    const int o = rb * RB + p * RP + sub;
    row[p] = -1;
    if (o >= total) continue;
    const int s = segment_of(a.cu_out, c.S, o);
    const int i = o - a.cu_out[s], n = a.cu_out[s + 1] - a.cu_out[s];
    const int j = max(c.lens[s], 0) - n + i;
    if (i >= 0 && i < n && j >= 0 && j < held_tokens(c, s))
      row[p] = (int64_t)lh * c.rows + c.cu_rows[s] + j;
  }
  uint32_t kw[kReadPasses], vw[kReadPasses], ks[kReadPasses], vs[kReadPasses];
#pragma unroll
  for (int p = 0; p < kReadPasses; ++p) {
    if (row[p] < 0) continue;
    if (a.k_out) {
      kw[p] = reinterpret_cast<const uint32_t*>(c.k_codes + row[p] * (D / 2))[piece];
      ks[p] = c.k_scales[row[p] * NS + piece / 4];
    }
    if (a.v_out) {
      vw[p] = reinterpret_cast<const uint32_t*>(c.v_codes + row[p] * (D / 2))[piece];
      vs[p] = c.v_scales[row[p] * NS + piece / 4];
    }
  }
#pragma unroll
  for (int p = 0; p < kReadPasses; ++p) {
    if (row[p] < 0) continue;
    const size_t dst = ((size_t)lh * a.out_rows + rb * RB + p * RP + sub) * D;
    if (a.k_out)
      __builtin_nontemporal_store(spread8(kw[p], scale_of(ks[p])),
                                  reinterpret_cast<u32x4_t*>(a.k_out + dst) + piece);
    if (a.v_out)
      __builtin_nontemporal_store(spread8(vw[p], scale_of(vs[p])),
                                  reinterpret_cast<u32x4_t*>(a.v_out + dst) + piece);
  }
}

}  // namespace

hipError_t launch_write4(const Write4Args& a, hipStream_t st) {
  // one workgroup at least: the compaction sets lens
  const dim3 grid(a.nblocks > 0 ? (unsigned)(a.c.L * a.c.H) * (unsigned)a.nblocks : 1u);
  if (a.c.d == 128)
    hipLaunchKernelGGL(write4_kernel<128>, grid, dim3(kThreads), 0, st, a);
  else
    hipLaunchKernelGGL(write4_kernel<64>, grid, dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_advance4(const Cache4View& c, const int32_t* cu_new, hipStream_t st) {
  hipLaunchKernelGGL(advance4_kernel, dim3((c.S + 255) / 256), dim3(256), 0, st, c, cu_new);
  return hipGetLastError();
}

hipError_t launch_read4(const Read4Args& a, hipStream_t st) {
  const int rb = kThreads / (a.c.d / 8) * kReadPasses;
  const dim3 grid((unsigned)(a.c.L * a.c.H) * (unsigned)((a.out_rows + rb - 1) / rb));
  if (a.c.d == 128)
    hipLaunchKernelGGL(read4_kernel<128>, grid, dim3(kThreads), 0, st, a);
  else
    hipLaunchKernelGGL(read4_kernel<64>, grid, dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace stepkv
