// Writing and reading the 8-bit cache (the format: include/stepkv_cache8.h).
//
// write8_kernel quantises bf16 rows into cache rows, gathered by the retained
// positions of a boundary or appended token by token; read8_kernel gives rows
// back in bf16. Both are bound by memory: 4d bytes of bf16 and 2d bytes of
// codes a row (K and V), a handful of operations a value. The conversions are
// one instruction per two values (their rounding and their NaN are the
// format's).
#include "cache8_device.h"

#include <type_traits>

namespace stepkv {
namespace {

constexpr int kThreads = 256;
constexpr int kWavesW = kThreads / kWave;
static_assert(kWavesW == 4, "the waves' results are looked at one by one");

typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pk_max_u16(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, a),
                                                                __builtin_bit_cast(u16x2_t, b)));
}

// Halves of a word that hold a finite magnitude stay, others become 0.
__device__ __forceinline__ uint32_t finite_halves(uint32_t mag) {
  return ((mag & 0xffffu) >= 0x7f80u ? 0u : mag & 0xffffu) |
         (mag >= 0x7f800000u ? 0u : mag & 0xffff0000u);
}

// The largest magnitudes (two halves) of eight bf16 values; `bad` if one is not
// finite (then the others count).
__device__ __forceinline__ uint32_t top_of(u32x4_t x, bool& bad) {
  constexpr uint32_t M = 0x7fff7fffu;
  const uint32_t x0 = x[0] & M, x1 = x[1] & M, x2 = x[2] & M, x3 = x[3] & M;
  uint32_t t = pk_max_u16(pk_max_u16(x0, x1), pk_max_u16(x2, x3));
  if ((t & 0xffffu) >= 0x7f80u || t >= 0x7f800000u) {
    bad = true;
    t = pk_max_u16(pk_max_u16(finite_halves(x0), finite_halves(x1)),
                   pk_max_u16(finite_halves(x2), finite_halves(x3)));
  }
  return t;
}

// The exponent that a largest magnitude 1.m * 2^(E - 127) in bf16 bits needs:
// E - 135 for 1.m <= 1.8125 (m <= 104, 464 = 1.8125 * 2^8) and E - 134 above: a
// carry into E.
__device__ __forceinline__ int need_of(uint32_t top) {
  return min(max((int)((top + 23u) >> 7) - 135, kLeast8), kMost8);
}

// Eight codes. With the greatest scale a finite magnitude past 448 of it is held
// as 448 (below that scale none is past 464, which rounds to 448).
__device__ __forceinline__ u32x2_t codes_of(u32x4_t x, int e) {
  if (e == kMost8) {
    constexpr uint32_t top = 0x7f60u;  // 448 * 2^119
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t lo = x[i] & 0x7fffu, hi = (x[i] >> 16) & 0x7fffu;
      lo = lo > top && lo < 0x7f80u ? top : lo;
      hi = hi > top && hi < 0x7f80u ? top : hi;
      x[i] = (x[i] & 0x80008000u) | lo | hi << 16;
    }
  }
  const float s = pow2_of(e);
  return u32x2_t{round4(x[0], x[1], s), round4(x[2], x[3], s)};
}

// Eight codes of one power of two, rounded to a greater one.
__device__ __forceinline__ u32x2_t regrid(u32x2_t w, float from, float to) {
  const u32x4_t x = spread8(w[0], w[1], from);
  return u32x2_t{round4(x[0], x[1], to), round4(x[2], x[3], to)};
}

// The tokens [j0, j1) of sequence s that a call writes (j0 may be negative:
// more new tokens than the sequence has), and the source row of token j0.
__device__ __forceinline__ void span_of(const Write8Args& a, int s, int& j0, int& j1) {
  const int room = a.c.cu_rows[s + 1] - a.c.cu_rows[s];
  const int n = a.cu_src[s + 1] - a.cu_src[s];
  if (a.cu_retained) {
    j0 = 0;
    j1 = min(min(a.cu_retained[s + 1] - a.cu_retained[s], n), room);
  } else {
    const int len = max(a.c.lens[s], 0);
    j0 = len - max(n, 0);
    j1 = min(len, room);
  }
}

// The span of one sequence, wave-uniform: scalar loads.
struct Span8 {
  int j0, j1, src0, src1, row0;
};
__device__ __forceinline__ Span8 span_const(const Write8Args& a, int s) {
  Span8 x;
  x.row0 = read_const(a.c.cu_rows, s);
  const int room = read_const(a.c.cu_rows, s + 1) - x.row0;
  x.src0 = read_const(a.cu_src, s);
  x.src1 = read_const(a.cu_src, s + 1);
  if (a.cu_retained) {
    x.j0 = 0;
    x.j1 = min(min(read_const(a.cu_retained, s + 1) - read_const(a.cu_retained, s),
                   x.src1 - x.src0), room);
  } else {
    const int len = max(read_const(a.c.lens, s), 0);
    x.j0 = len - max(x.src1 - x.src0, 0);
    x.j1 = min(len, room);
  }
  return x;
}

// One workgroup per (layer, KV head, block of 64 tokens): a lane holds 16 bytes
// (8 channels) of a row of K and of V, the largest magnitudes of the block meet
// in LDS, and its scales are written once. A token of the call without a source
// keeps its codes. Chains of loads bound it (the block's sequence, the positions, the
// rows), so a workgroup has all its rows in flight at once; blocks go to the XCDs in
// turn. 32 layers x 8 heads x 1536 gathered rows of d 128 66 us, 308 MB at 4.7 TB/s; 8100 new tokens of 8 heads 11 us
// (50 MB), one token of each of 28 sequences 4.5.
template <int D>
__global__ __launch_bounds__(kThreads) void write8_kernel(Write8Args a) {
  constexpr int PR = D / 8;          // pieces of 8 channels a row
  constexpr int RP = kThreads / PR;  // rows a pass
  constexpr int NP = kBlock8 / RP;   // passes
  __shared__ uint32_t tops[kWavesW];
  __shared__ int some[kWavesW];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const Cache8View& c = a.c;
  if (blockIdx.x == 0 && tid < kWave) {
    if (a.cu_retained) {
      bool over = false;
      for (int s = tid; s < c.S; s += kWave) {
        const int n = max(a.cu_retained[s + 1] - a.cu_retained[s], 0);
        const int there = a.cu_src[s + 1] - a.cu_src[s];  // no more tokens than the source has
        c.lens[s] = min(n, there);
        c.seen[s] = there;
        over |= n > min(there, c.cu_rows[s + 1] - c.cu_rows[s]);
      }
      if (over && c.status) atomicOr(c.status, kFlagOutRows4);
    } else {
      report_rooms(c);
      // offsets that count more tokens than the call gives
      report_flags(c.status, read_const(a.cu_src, c.S) > a.nsrc ? kFlagOutRows4 : 0u);
    }
  }
  if (a.nblocks == 0) return;
  const int lh = uniform(blockIdx.x / a.nblocks);
  const int at = uniform(blockIdx.x - lh * a.nblocks);
  const int l = uniform(lh / c.H), h = lh - l * c.H;
  int s = 0, first = 0;  // the block's sequence, and the blocks of those before it
  if (c.S > 1)
    locate_item(c.S, at, [&](int sq) {
      int b0, b1;
      span_of(a, sq, b0, b1);
      b0 = max(b0, 0);
      return b1 > b0 ? (b1 - 1) / kBlock8 - b0 / kBlock8 + 1 : 0;
    }, s, first);
  if (s < 0) return;  // uniform over the workgroup, as all that follow
  const Span8 x = span_const(a, s);
  const int blk = max(x.j0, 0) / kBlock8 + (at - first);
  if (x.j1 <= max(x.j0, 0) || blk * kBlock8 >= x.j1) return;
  const int b0 = blk * kBlock8;
  const bool anew = b0 >= x.j0;  // the block's first token is among the call's
  const size_t scale_at = (size_t)lh * c.nblk + first_block(x.row0, s) + blk;
  int ek = kLeast8, ev = kLeast8;  // what the block's scales are at least
  float k_old = 0.f, v_old = 0.f;
  if (!anew) {
    k_old = c.k_scales[scale_at];
    v_old = c.v_scales[scale_at];
  }
  const int32_t* __restrict__ idx =
      a.idx ? a.idx + (a.shared_idx ? 0 : (size_t)lh * a.nsrc) + x.src0 : nullptr;
  const int sub = tid / PR, piece = tid % PR;
  int src[NP];  // source row, or -1
  uint32_t flags = 0u;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int j = b0 + p * RP + sub;
    src[p] = -1;
    if (j >= x.j0 && j < x.j1) {
      if (idx) {
        const int pos = idx[j];
        if (pos >= 0 && pos < x.src1 - x.src0) src[p] = x.src0 + pos;
      } else {
        const int64_t from = (int64_t)x.src0 + j - x.j0;
        if (from >= 0 && from < a.nsrc) src[p] = (int)from;
      }
      if (src[p] < 0) flags |= kFlagOutRows4;
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
  uint32_t kt = 0u, vt = 0u;
  bool bad = false;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    kt = pk_max_u16(kt, top_of(kx[p], bad));
    vt = pk_max_u16(vt, top_of(vx[p], bad));
  }
  if (bad) flags |= kFlagNonFinite4;
  report_flags(c.status, flags);
  kt = max(kt & 0xffffu, kt >> 16);
  vt = max(vt & 0xffffu, vt >> 16);
  uint32_t both = kt << 16 | vt;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1)
    both = pk_max_u16(both, (uint32_t)__shfl_xor((int)both, off, kWave));
  if (lane == 0) tops[wave] = both;
  bool writes = false;
#pragma unroll
  for (int p = 0; p < NP; ++p) writes |= src[p] >= 0;
  const uint64_t writing = ballot(writes);
  if (lane == 0) some[wave] = writing != 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWavesW; ++w) both = pk_max_u16(both, tops[w]);
  if (!some[0] && !some[1] && !some[2] && !some[3]) return;  // nothing is written into the block
  ek = need_of(both >> 16);
  ev = need_of(both & 0xffffu);
  if (!anew) {
    ek = max(ek, exponent_of(k_old));
    ev = max(ev, exponent_of(v_old));
    ek = uniform(min(max(ek, kLeast8), kMost8));
    ev = uniform(min(max(ev, kLeast8), kMost8));
  }
  if (tid == 0) {
    c.k_scales[scale_at] = pow2_of(ek);
    c.v_scales[scale_at] = pow2_of(ev);
  }
  const size_t row = (size_t)lh * c.rows + x.row0 + b0;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    if (src[p] < 0) continue;
    const size_t r = row + p * RP + sub;
    __builtin_nontemporal_store(codes_of(kx[p], ek), reinterpret_cast<u32x2_t*>(c.k_codes + r * D) + piece);
    __builtin_nontemporal_store(codes_of(vx[p], ev), reinterpret_cast<u32x2_t*>(c.v_codes + r * D) + piece);
    if (piece == 0 && c.weights) {
      c.weights[r] = a.gathered ? a.gathered[(size_t)lh * a.nsrc + src[p]] : 0.f;
      const int j = b0 + p * RP + sub;
      c.positions[r] = idx ? src[p] - x.src0
                           : read_const(c.seen, s) - (max(read_const(c.lens, s), 0) - j);
    }
  }
  // The block's other tokens, where a scale grew.
  const bool grow_k = !anew && ek > exponent_of(k_old), grow_v = !anew && ev > exponent_of(v_old);
  if (!grow_k && !grow_v) return;
#pragma nounroll
  for (int p = 0; p < NP; ++p) {
    const int j = b0 + p * RP + sub;
    if (src[p] >= 0 || j >= x.j1) continue;
    const size_t r = row + p * RP + sub;
    if (grow_k) {
      u32x2_t* w = reinterpret_cast<u32x2_t*>(c.k_codes + r * D) + piece;
      *w = regrid(*w, k_old, pow2_of(ek));
    }
    if (grow_v) {
      u32x2_t* w = reinterpret_cast<u32x2_t*>(c.v_codes + r * D) + piece;
      *w = regrid(*w, v_old, pow2_of(ev));
    }
  }
}

__global__ void advance8_kernel(Cache8View c, const int32_t* __restrict__ cu_new) {
  for (int s = blockIdx.x * blockDim.x + threadIdx.x; s < c.S; s += gridDim.x * blockDim.x) {
    const int n = max(cu_new[s + 1] - cu_new[s], 0);
    c.lens[s] += n;
    c.seen[s] += n;
  }
}

// A thread per 8 channels of a row: 8 bytes of codes in, 16 bytes out, PASSES
// rows in flight per thread. A workgroup's rows almost always belong to one
// sequence, whose bounds are then found once, with scalar loads. 28 layers x 4 heads x
// 28812 rows of d 128 in 16 sequences: 392 us, 2.48 GB at 6.3 TB/s (a copy of as many
// bytes: 377).
template <int D, int PASSES>
__global__ __launch_bounds__(kThreads) void read8_kernel(Read8Args a) {
  constexpr int PR = D / 8;
  constexpr int RP = kThreads / PR;
  constexpr int RB = RP * PASSES;
  const Cache8View& c = a.c;
  const int nb = (a.out_rows + RB - 1) / RB;
  const int bid = blockIdx.x;
  const int lh = uniform(bid / nb), o0 = (bid - lh * nb) * RB;
  if (lh >= c.L * c.H) return;
  const int total = min(a.out_rows, read_const(a.cu_out, c.S));
  if (o0 >= total) return;
  const int sub = threadIdx.x / PR, piece = threadIdx.x % PR;
  // row i of sequence s's rows is token len - n + i, in cache row row0 + shift + o
  int lo = 0, hi = c.S;  // cu_out[lo] <= o0 < cu_out[hi] where cu_out is in order
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (read_const(a.cu_out, mid) <= o0) lo = mid;
    else hi = mid;
  }
  const bool one = o0 + RB <= read_const(a.cu_out, lo + 1) || lo + 1 == c.S;
  const int r0 = read_const(a.cu_out, lo), r1 = read_const(a.cu_out, lo + 1);
  const int row0 = read_const(c.cu_rows, lo), len = max(read_const(c.lens, lo), 0);
  const int held = min(len, read_const(c.cu_rows, lo + 1) - row0);
  int64_t row[PASSES];  // cache row, or -1
  int blk[PASSES];      // its block
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int o = o0 + p * RP + sub;
    row[p] = -1;
    blk[p] = 0;
    if (o >= total) continue;
    if (!one && o >= r1) {
      const int s = segment_of(a.cu_out, c.S, o);
      const int64_t j = (int64_t)o - a.cu_out[s + 1] + max(c.lens[s], 0);
      if (o >= a.cu_out[s] && o < a.cu_out[s + 1] && j >= 0 && j < held_tokens(c, s)) {
        row[p] = (int64_t)lh * c.rows + c.cu_rows[s] + j;
        blk[p] = first_block(c.cu_rows[s], s) + (int)(j / kBlock8);
      }
    } else {
      const int64_t j = (int64_t)o - r1 + len;
      if (o >= r0 && o < r1 && j >= 0 && j < held) {
        row[p] = (int64_t)lh * c.rows + row0 + j;
        blk[p] = first_block(row0, lo) + (int)j / kBlock8;
      }
    }
  }
  u32x2_t kw[PASSES], vw[PASSES];
  float ks[PASSES], vs[PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    if (row[p] < 0) continue;
    const size_t sc = (size_t)lh * c.nblk + blk[p];
    if (a.k_out) {
      kw[p] = __builtin_nontemporal_load(
          reinterpret_cast<const u32x2_t*>(c.k_codes + row[p] * D) + piece);
      ks[p] = c.k_scales[sc];
    }
    if (a.v_out) {
      vw[p] = __builtin_nontemporal_load(
          reinterpret_cast<const u32x2_t*>(c.v_codes + row[p] * D) + piece);
      vs[p] = c.v_scales[sc];
    }
  }
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    if (row[p] < 0) continue;
    const size_t dst = ((size_t)lh * a.out_rows + o0 + p * RP + sub) * D;
    if (a.k_out)
      __builtin_nontemporal_store(spread8(kw[p][0], kw[p][1], ks[p]),
                                  reinterpret_cast<u32x4_t*>(a.k_out + dst) + piece);
    if (a.v_out)
      __builtin_nontemporal_store(spread8(vw[p][0], vw[p][1], vs[p]),
                                  reinterpret_cast<u32x4_t*>(a.v_out + dst) + piece);
  }
}

// Workgroups of a read with `passes` rows a thread.
int64_t read_workgroups(const Read8Args& a, int passes) {
  const int64_t rows = (int64_t)kThreads / (a.c.d / 8) * passes;
  return (int64_t)a.c.L * a.c.H * ((a.out_rows + rows - 1) / rows);
}

}  // namespace

bool write8_fits(const Write8Args& a) {
  return grid_fits((int64_t)a.c.L * a.c.H * a.nblocks, kThreads);
}

hipError_t launch_write8(const Write8Args& a, hipStream_t st) {
  // one workgroup at least: the compaction sets lens
  const dim3 grid(a.nblocks > 0 ? (unsigned)(a.c.L * a.c.H) * (unsigned)a.nblocks : 1u);
  if (a.c.d == 128)
    hipLaunchKernelGGL(write8_kernel<128>, grid, dim3(kThreads), 0, st, a);
  else
    hipLaunchKernelGGL(write8_kernel<64>, grid, dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_advance8(const Cache8View& c, const int32_t* cu_new, hipStream_t st) {
  hipLaunchKernelGGL(advance8_kernel, dim3((c.S + 255) / 256), dim3(256), 0, st, c, cu_new);
  return hipGetLastError();
}

bool read8_fits(const Read8Args& a) { return grid_fits(read_workgroups(a, 4), kThreads); }

hipError_t launch_read8(const Read8Args& a, hipStream_t st) {
  const int64_t one = read_workgroups(a, 1);
  auto run = [&](auto passes) {
    constexpr int P = decltype(passes)::value;
    const dim3 grid((unsigned)read_workgroups(a, P));
    if (a.c.d == 128)
      hipLaunchKernelGGL((read8_kernel<128, P>), grid, dim3(kThreads), 0, st, a);
    else
      hipLaunchKernelGGL((read8_kernel<64, P>), grid, dim3(kThreads), 0, st, a);
  };
  if (!grid_fits(one, kThreads)) run(std::integral_constant<int, 4>{});
  else run(std::integral_constant<int, 1>{});
  return hipGetLastError();
}

}  // namespace stepkv
