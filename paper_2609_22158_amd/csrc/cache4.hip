// Writing and reading the 4-bit cache (the format: include/stepkv_cache4.h).
//
// write4_kernel quantises bf16 rows into cache rows, gathered by the retained
// positions of a boundary or appended token by token; read4_kernel gives rows
// back in bf16. Both are bound by memory: 4d bytes of bf16 and d + d/16 bytes
// of codes and scales a row (K and V), a handful of operations a value. The
// conversions are one instruction per two values (their rounding, ties to the
// even code and saturation at 6, is the format's).
#include "cache4_device.h"

#include <type_traits>

namespace stepkv {
namespace {

constexpr int kThreads = 256;

typedef short i16x2_t __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pk_max_u16(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, a),
                                                                __builtin_bit_cast(u16x2_t, b)));
}
__device__ __forceinline__ uint32_t pk_max_i16(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(i16x2_t, a),
                                                                __builtin_bit_cast(i16x2_t, b)));
}
__device__ __forceinline__ uint32_t pk_min_i16(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(i16x2_t, a),
                                                                __builtin_bit_cast(i16x2_t, b)));
}
// Two bf16 patterns as 16-bit integers in the order of their values, and back
// (its own inverse): negative ones have their magnitude bits inverted.
__device__ __forceinline__ uint32_t pk_sortable(uint32_t x) {
  const i16x2_t v = __builtin_bit_cast(i16x2_t, x);
  return x ^ (__builtin_bit_cast(uint32_t, v >> 15) & 0x7fff7fffu);
}

// Eight values of a group (the other 24 in the other lanes of the quad):
// their codes, and the group's scale byte. With the largest magnitude
// 1.m * 2^E in bf16 bits (E and the 7 bits of m), max <= 7 * 2^e means
// e = E - 2 for 1.m <= 1.75 (m <= 96) and E - 1 above: a carry into E.
__device__ __forceinline__ uint32_t quantise8(u32x4_t x, uint32_t& byte) {
  // copied: a bit cast of a vector's element takes the vector's first
  const uint32_t x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];
  uint32_t two = pk_max_u16(pk_max_u16(x0 & 0x7fff7fffu, x1 & 0x7fff7fffu),
                            pk_max_u16(x2 & 0x7fff7fffu, x3 & 0x7fff7fffu));
  // over the quad's lanes (^ 1, ^ 2)
  two = pk_max_u16(two, (uint32_t)__builtin_amdgcn_mov_dpp((int)two, 0xB1, 0xf, 0xf, true));
  two = pk_max_u16(two, (uint32_t)__builtin_amdgcn_mov_dpp((int)two, 0x4E, 0xf, 0xf, true));
  const uint32_t top = max(two & 0xffffu, two >> 16);
  const bool bad = top >= 0x7f80u;  // a NaN or an infinity in the group
  byte = bad ? 255u : (uint32_t)min(max((int)((top + 31u) >> 7) - 2, 3), 252);
  const float s = scale_of(byte);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, x0), s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, x1), s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, x2), s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, x3), s, 3);
  return bad ? 0u : w;
}

// The tokens [j0, j1) of sequence s that a call writes (j0 may be negative:
// more new tokens than the sequence has), and the source row of token j0.
__device__ __forceinline__ void span_of(const Write4Args& a, int s, int& j0, int& j1, int& src0) {
  const int room = a.c.cu_rows[s + 1] - a.c.cu_rows[s];
  src0 = a.cu_src[s];
  if (a.cu_retained) {
    j0 = 0;
    j1 = min(min(a.cu_retained[s + 1] - a.cu_retained[s], a.cu_src[s + 1] - src0), room);
  } else {
    const int len = max(a.c.lens[s], 0);
    j0 = len - max(a.cu_src[s + 1] - src0, 0);
    j1 = min(len, room);
  }
}

// The span of one sequence, wave-uniform: scalar loads.
__device__ __forceinline__ void span_const(const Write4Args& a, int s, int& j0, int& j1,
                                           int& src0, int& src1, int& row0) {
  row0 = read_const(a.c.cu_rows, s);
  const int room = read_const(a.c.cu_rows, s + 1) - row0;
  src0 = read_const(a.cu_src, s);
  src1 = read_const(a.cu_src, s + 1);
  if (a.cu_retained) {
    j0 = 0;
    j1 = min(min(read_const(a.cu_retained, s + 1) - read_const(a.cu_retained, s), src1 - src0),
             room);
  } else {
    const int len = max(read_const(a.c.lens, s), 0);
    j0 = len - max(src1 - src0, 0);
    j1 = min(len, room);
  }
}

// A block of 64 tokens that a call's spans touch, and the span of its sequence.
struct Block4 {
  int s, blk, j0, j1, src0, src1, row0;
};

// Block `at` of those that the spans touch, in the order of the sequences; false
// past the last. Wave-uniform.
__device__ __forceinline__ bool find_block(const Write4Args& a, int at, Block4& x) {
  int first = 0;
  x.s = 0;
  if (a.c.S > 1)
    locate_item(a.c.S, at, [&](int sq) {
      int b0, b1, unused;
      span_of(a, sq, b0, b1, unused);
      b0 = max(b0, 0);
      return b1 > b0 ? (b1 - 1) / kBlock4 - b0 / kBlock4 + 1 : 0;
    }, x.s, first);
  if (x.s < 0) return false;
  span_const(a, x.s, x.j0, x.j1, x.src0, x.src1, x.row0);
  x.blk = max(x.j0, 0) / kBlock4 + (at - first);
  return x.j1 > max(x.j0, 0) && x.blk * kBlock4 < x.j1;  // of the only sequence: up to its last
}

// The least and greatest of 8 channels of K over a lane's rows, from the values
// as quantised, as ordered 16-bit integers two at a time; a NaN is a flag.
struct Bounds4 {
  uint32_t lo[4], hi[4];
  bool bad = false;
  __device__ __forceinline__ Bounds4() {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = 0x7f807f80u;  // +inf, and -inf as it sorts
      hi[i] = pk_sortable(0xff80ff80u);
    }
  }
  __device__ __forceinline__ void add(uint32_t codes, uint32_t byte) {
    if (byte == 255u) {
      bad = true;
      return;
    }
    const u32x4_t y = spread8(codes, scale_of(byte));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t t = pk_sortable(y[i]);
      lo[i] = pk_min_i16(lo[i], t);
      hi[i] = pk_max_i16(hi[i], t);
    }
  }
};

// The block's bounds from those of the workgroup's lanes, with the ones there are
// where the block's first token is not the call's. red, bad_s: LDS.
template <int D>
__device__ __forceinline__ void store_bounds(const Cache4View& c, int lh, const Block4& x,
                                             Bounds4 m,
                                             uint32_t (&red)[kThreads / kWave][2][D / 2],
                                             int (&bad_s)[kThreads / kWave][D / 8]) {
  constexpr int PR = D / 8, NWV = kThreads / kWave;
  const int tid = threadIdx.x, piece = tid % PR;
  // over the rows of the wave (lanes of one piece), then over the waves
#pragma unroll
  for (int off = PR; off < kWave; off <<= 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m.lo[i] = pk_min_i16(m.lo[i], (uint32_t)__shfl_xor((int)m.lo[i], off, kWave));
      m.hi[i] = pk_max_i16(m.hi[i], (uint32_t)__shfl_xor((int)m.hi[i], off, kWave));
    }
  }
  const uint64_t bads = ballot(m.bad);
  if ((tid & 63) < PR) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      red[tid >> 6][0][4 * piece + i] = m.lo[i];
      red[tid >> 6][1][4 * piece + i] = m.hi[i];
    }
    uint64_t lanes = 0;  // those that hold this piece
#pragma unroll
    for (int off = 0; off < kWave; off += PR) lanes |= uint64_t(1) << off;
    bad_s[tid >> 6][piece] = (bads & (lanes << piece)) != 0;
  }
  __syncthreads();
  uint16_t* __restrict__ bounds =
      c.k_bounds + ((size_t)lh * c.nblk + x.row0 / kBlock4 + x.s + x.blk) * 2 * D;
  if (tid < D) {
    const int which = tid / (D / 2), two = tid % (D / 2);  // channels 2 two, 2 two + 1
    uint32_t v = red[0][which][two];
    bool nan0 = false, nan1;
#pragma unroll
    for (int w = 0; w < NWV; ++w) {
      v = which ? pk_max_i16(v, red[w][which][two]) : pk_min_i16(v, red[w][which][two]);
      nan0 |= bad_s[w][two / 4] != 0;
    }
    nan1 = nan0;
    uint32_t* out = reinterpret_cast<uint32_t*>(bounds + which * D) + two;
    if (x.blk * kBlock4 < x.j0) {  // the block's first token is not among the new ones
      const uint32_t old = *out, t = pk_sortable(old);
      nan0 |= (old & 0x7fffu) > 0x7f80u;
      nan1 |= (old >> 16 & 0x7fffu) > 0x7f80u;
      v = which ? pk_max_i16(v, t) : pk_min_i16(v, t);
    }
    v = pk_sortable(v);
    if (nan0) v = (v & 0xffff0000u) | 0x7fc0u;
    if (nan1) v = (v & 0xffffu) | 0x7fc00000u;
    *out = v;
  }
}

// One workgroup per (layer, KV head, block of 64 tokens): a lane holds 16
// bytes (8 channels) of a row, a quad of lanes a group. A token of the call
// without a source keeps what its row holds, and the block's bounds count that
// like the rows that are written. 32 layers x 8 heads x 1536 rows gathered from
// 32768 take 52 to 54 us (255 MB, 4.7 to 4.9 TB/s), bound by the gather's reads in
// flight: 64 rows of K and V a workgroup, 32 KB. Code stores are non-temporal
// (measured at one time: 51 us, with ordinary ones 54, with 16-byte stores of
// words exchanged within the quads 60).
template <int D>
__global__ __launch_bounds__(kThreads) void write4_kernel(Write4Args a) {
  constexpr int PR = D / 8;             // pieces of 8 channels a row
  constexpr int RP = kThreads / PR;     // rows a pass
  constexpr int NP = kBlock4 / RP;      // passes
  constexpr int NS = D / kGroup4;
  constexpr int NWV = kThreads / kWave;
  __shared__ uint32_t red[NWV][2][D / 2];
  __shared__ int bad_s[NWV][PR];
  const int tid = threadIdx.x;
  const Cache4View& c = a.c;
  // offsets of an append that count more tokens than it gives
  const bool short_of = !a.cu_retained && read_const(a.cu_src, c.S) > a.nsrc;
  if (blockIdx.x == 0 && tid < kWave) {
    if (a.cu_retained) {
      bool over = false;
      for (int s = tid; s < c.S; s += kWave) {
        const int n = max(a.cu_retained[s + 1] - a.cu_retained[s], 0);
        const int there = a.cu_src[s + 1] - a.cu_src[s];  // no more tokens than the source has
        c.lens[s] = min(n, there);
        over |= n > min(there, c.cu_rows[s + 1] - c.cu_rows[s]);
      }
      if (over && c.status) atomicOr(c.status, kFlagOutRows4);
    } else {
      report_rooms(c);
      report_flags(c.status, short_of ? kFlagOutRows4 : 0u);
    }
  }
  if (a.nblocks == 0) return;
  const int lh = uniform(blockIdx.x / a.nblocks);
  int at = uniform(blockIdx.x - lh * a.nblocks);
  const int l = uniform(lh / c.H), h = lh - l * c.H;
  Block4 x;
  if (!find_block(a, at, x)) return;  // uniform over the workgroup
  const int32_t* __restrict__ idx =
      a.idx ? a.idx + (a.shared_idx ? 0 : (size_t)lh * a.nsrc) + x.src0 : nullptr;
  const int sub = tid / PR, piece = tid % PR;
  int src[NP];      // source row, or -1
  int missing = 0;  // bit p: a token of the call that has none
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int j = x.blk * kBlock4 + p * RP + sub;
    src[p] = -1;
    if (j >= x.j0 && j < x.j1) {
      if (idx) {
        const int pos = idx[j];
        if (pos >= 0 && pos < x.src1 - x.src0) src[p] = x.src0 + pos;
      } else if (x.src0 + (j - x.j0) >= 0 && x.src0 + (j - x.j0) < a.nsrc) {
        src[p] = x.src0 + (j - x.j0);
      }
      if (src[p] < 0) missing |= 1 << p;
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
  const size_t head_row = (size_t)lh * c.rows;
  const size_t first_row = head_row + x.row0 + (size_t)x.blk * kBlock4;
  Bounds4 m;
  uint32_t flags = missing ? kFlagOutRows4 : 0u;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    uint32_t kbyte, vbyte;  // every lane: the quad exchanges need all four
    const uint32_t kw = quantise8(kx[p], kbyte), vw = quantise8(vx[p], vbyte);
    if (src[p] < 0) continue;
    if (kbyte == 255u || vbyte == 255u) flags |= kFlagNonFinite4;
    const size_t row = first_row + p * RP + sub;
    __builtin_nontemporal_store(kw, reinterpret_cast<uint32_t*>(c.k_codes + row * (D / 2)) + piece);
    __builtin_nontemporal_store(vw, reinterpret_cast<uint32_t*>(c.v_codes + row * (D / 2)) + piece);
    if (piece % 4 == 0) {
      c.k_scales[row * NS + piece / 4] = (uint8_t)kbyte;
      c.v_scales[row * NS + piece / 4] = (uint8_t)vbyte;
    }
    m.add(kw, kbyte);
  }
  report_flags(c.status, flags);
  if (!c.k_bounds) return;
  auto add_stored = [&](size_t row) __attribute__((always_inline)) {
    m.add(reinterpret_cast<const uint32_t*>(c.k_codes + row * (D / 2))[piece],
          c.k_scales[row * NS + piece / 4]);
  };
  if (ballot(missing != 0)) {  // rare
#pragma nounroll
    for (int p = 0; p < NP; ++p)
      if (missing >> p & 1) add_stored(first_row + p * RP + sub);
  }
  store_bounds<D>(c, lh, x, m, red, bad_s);
  // Then the grid has fewer workgroups than there are blocks: those past it hold
  // no token that is given (these come first), and only need their bounds.
  if (!short_of) return;
  for (at += a.nblocks; find_block(a, at, x); at += a.nblocks) {
    __syncthreads();  // red and bad_s are read above
    m = Bounds4();
#pragma nounroll
    for (int p = 0; p < NP; ++p) {
      const int j = x.blk * kBlock4 + p * RP + sub;
      if (j >= x.j0 && j < x.j1) add_stored(head_row + x.row0 + j);
    }
    store_bounds<D>(c, lh, x, m, red, bad_s);
  }
}

__global__ void advance4_kernel(Cache4View c, const int32_t* __restrict__ cu_new) {
  for (int s = blockIdx.x * blockDim.x + threadIdx.x; s < c.S; s += gridDim.x * blockDim.x)
    c.lens[s] += max(cu_new[s + 1] - cu_new[s], 0);
}

// A thread per 8 channels of a row: one word of codes and a scale byte in, 16
// bytes out, PASSES rows in flight per thread. A workgroup's rows almost always
// belong to one sequence, whose bounds are then found once, with scalar loads.

template <int D, int PASSES>
__global__ __launch_bounds__(kThreads) void read4_kernel(Read4Args a) {
  constexpr int PR = D / 8;
  constexpr int RP = kThreads / PR;
  constexpr int RB = RP * PASSES;
  constexpr int NS = D / kGroup4;
  const Cache4View& c = a.c;
  const int nb = (a.out_rows + RB - 1) / RB;
  const int bid = blockIdx.x;
  const int lh = uniform(bid / nb), o0 = (bid - lh * nb) * RB;
  if (lh >= c.L * c.H) return;
  const int total = min(a.out_rows, read_const(a.cu_out, c.S));
  if (o0 >= total) return;
  const int sub = threadIdx.x / PR, piece = threadIdx.x % PR;
  // row i of sequence s's rows is token len - n + i, in cache row shift + o
  int lo = 0, hi = c.S;  // cu_out[lo] <= o0 < cu_out[hi] where cu_out is in order
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (read_const(a.cu_out, mid) <= o0) lo = mid;
    else hi = mid;
  }
  auto span = [&](int s, int& b, int& e, int64_t& shift) {  // rows [b, e) have tokens
    const int r0 = read_const(a.cu_out, s), r1 = read_const(a.cu_out, s + 1);
    const int row0 = read_const(c.cu_rows, s);
    const int len = max(read_const(c.lens, s), 0);
    const int held = min(len, read_const(c.cu_rows, s + 1) - row0);
    // token of row o: o - r1 + len, within [0, held)
    b = (int)max((int64_t)r0, (int64_t)r1 - len);
    e = (int)min((int64_t)r1, (int64_t)r1 - len + held);
    shift = (int64_t)row0 + len - r1;
  };
  int b, e;
  int64_t shift;
  span(lo, b, e, shift);
  const bool one = o0 + RB <= read_const(a.cu_out, lo + 1) || lo + 1 == c.S;
  int64_t row[PASSES];  // cache row, or -1
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int o = o0 + p * RP + sub;
    row[p] = -1;
    if (o >= total) continue;
    if (!one && o >= read_const(a.cu_out, lo + 1)) {
      const int s = segment_of(a.cu_out, c.S, o);
      const int r1 = a.cu_out[s + 1], len = max(c.lens[s], 0);
      const int64_t j = (int64_t)o - r1 + len;
      if (o >= a.cu_out[s] && o < r1 && j >= 0 && j < held_tokens(c, s))
        row[p] = (int64_t)lh * c.rows + c.cu_rows[s] + j;
    } else if (o >= b && o < e) {
      row[p] = (int64_t)lh * c.rows + shift + o;
    }
  }
  uint32_t kw[PASSES], vw[PASSES], ks[PASSES], vs[PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    if (row[p] < 0) continue;
    if (a.k_out) {
      kw[p] = __builtin_nontemporal_load(
          reinterpret_cast<const uint32_t*>(c.k_codes + row[p] * (D / 2)) + piece);
      ks[p] = c.k_scales[row[p] * NS + piece / 4];
    }
    if (a.v_out) {
      vw[p] = __builtin_nontemporal_load(
          reinterpret_cast<const uint32_t*>(c.v_codes + row[p] * (D / 2)) + piece);
      vs[p] = c.v_scales[row[p] * NS + piece / 4];
    }
  }
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    if (row[p] < 0) continue;
    const size_t dst = ((size_t)lh * a.out_rows + o0 + p * RP + sub) * D;
    if (a.k_out)
      __builtin_nontemporal_store(spread8(kw[p], scale_of(ks[p])),
                                  reinterpret_cast<u32x4_t*>(a.k_out + dst) + piece);
    if (a.v_out)
      __builtin_nontemporal_store(spread8(vw[p], scale_of(vs[p])),
                                  reinterpret_cast<u32x4_t*>(a.v_out + dst) + piece);
  }
}

}  // namespace

bool write4_fits(const Write4Args& a) {
  return grid_fits((int64_t)a.c.L * a.c.H * a.nblocks, kThreads);
}

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

namespace {

// Workgroups of a read with `passes` rows a thread.
int64_t read_workgroups(const Read4Args& a, int passes) {
  const int64_t rows = (int64_t)kThreads / (a.c.d / 8) * passes;
  return (int64_t)a.c.L * a.c.H * ((a.out_rows + rows - 1) / rows);
}

}  // namespace

bool read4_fits(const Read4Args& a) { return grid_fits(read_workgroups(a, 4), kThreads); }

hipError_t launch_read4(const Read4Args& a, hipStream_t st) {
  // One row per thread keeps the most workgroups in flight, and the smallest
  // calls short (32 layers x 8 heads x 1536 rows 42 us, with four rows 47; 85
  // rows 4.1 and 6.0). With many rows of several sequences the search for the
  // sequence counts: four rows share it (28 layers x 4 heads x 16 sequences,
  // 28800 rows in all: 358 us, with one row 380). Four rows also keep the largest
  // reads of one sequence within a launch (2^28 rows of d 128, all heads together).
  const int64_t one = read_workgroups(a, 1);
  auto run = [&](auto passes) {
    constexpr int P = decltype(passes)::value;
    const dim3 grid((unsigned)read_workgroups(a, P));
    if (a.c.d == 128)
      hipLaunchKernelGGL((read4_kernel<128, P>), grid, dim3(kThreads), 0, st, a);
    else
      hipLaunchKernelGGL((read4_kernel<64, P>), grid, dim3(kThreads), 0, st, a);
  };
  if ((a.c.S > 1 && one >= 8 * 2048) || !grid_fits(one, kThreads)) run(std::integral_constant<int, 4>{});
  else run(std::integral_constant<int, 1>{});
  return hipGetLastError();
}

}  // namespace stepkv
