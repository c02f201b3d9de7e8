// The blocks that a decode step attends to (stepkv_cache4_select_blocks).
//
// score4_kernel: the score of every block that is ranked,
//   sum_i a_i kmax_i + b_i kmin_i,  a = sum_g max(q_g, 0), b = sum_g min(q_g, 0),
// which is sum_g sum_i max(q_gi kmin_i, q_gi kmax_i): one product per channel
// and bound, whatever the group. 4d bytes of bounds a block bound it. The sums
// are kept in 64 bits, so that two scores compare as their exact values do
// (32-bit sums would rank close blocks by the order of their additions).
// select4_kernel: one workgroup per (layer, sequence, KV head) finds the
// threshold by radix passes over the ordered keys and lists the blocks.
#include "cache4_device.h"

namespace stepkv {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 128;  // blocks a workgroup scores

__device__ __forceinline__ int blocks_of(const Cache4View& c, int s) {
  return (held_tokens(c, s) + kBlock4 - 1) / kBlock4;
}

// Doubles as unsigned integers in the same order; NaN as -inf, -0 as +0.
__device__ __forceinline__ uint64_t ordered(double x) {
  if (x != x) x = -INFINITY;
  const uint64_t b = __builtin_bit_cast(uint64_t, x + 0.0);
  return b >> 63 ? ~b : b | (uint64_t(1) << 63);
}

// Eight lanes a block; lane i holds pieces i, i + 8, .. (16 bytes) of the
// block's minima, then maxima, and the coefficients of those channels.
template <int D>
__global__ __launch_bounds__(kThreads) void score4_kernel(Select4Args a) {
  constexpr int NP = D / 64;  // pieces a lane holds of each bound
  const Cache4View& c = a.c;
  const int lh = blockIdx.x / a.chunks;
  const int l = lh / c.H, h = lh - l * c.H;
  int s, first;
  locate_item(c.S, (int)(blockIdx.x - lh * a.chunks), [&](int sq) {
    const int nb = blocks_of(c, sq);
    return nb > a.n ? (nb + kChunk - 1) / kChunk : 0;  // shorter ones are not ranked
  }, s, first);
  if (s < 0) return;
  const int b0 = ((int)(blockIdx.x - lh * a.chunks) - first) * kChunk;
  const int b1 = min(blocks_of(c, s), b0 + kChunk);
  const int i = threadIdx.x & 7;
  double up[NP][8] = {}, down[NP][8] = {};
  const uint16_t* __restrict__ q = a.q + (((size_t)l * c.S + s) * a.Hq + h * a.G) * D + 8 * i;
  for (int g = 0; g < a.G; ++g)
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const u32x4_t w = *reinterpret_cast<const u32x4_t*>(q + (size_t)g * D + 64 * p);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = bf16_float(e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xffffu);
        up[p][e] += x > 0.f ? (double)x : 0.0;  // a NaN adds nothing
        down[p][e] += x < 0.f ? (double)x : 0.0;
      }
    }
  const size_t at = (size_t)lh * c.nblk + c.cu_rows[s] / kBlock4 + s;
  for (int b = b0 + (int)(threadIdx.x >> 3); b < b0 + kChunk; b += kThreads / 8) {
    const uint16_t* __restrict__ x = c.k_bounds + (at + min(b, b1 - 1)) * 2 * D + 8 * i;
    double sum = 0.0;
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const u32x4_t w = __builtin_nontemporal_load(
            reinterpret_cast<const u32x4_t*>(x + which * D + 64 * p));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const double y = bf16_float(e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xffffu);
          sum = fma(y, which ? up[p][e] : down[p][e], sum);
        }
      }
#pragma unroll
    for (int off = 1; off < 8; off <<= 1) sum += __shfl_xor(sum, off, kWave);
    if (i == 0 && b < b1) a.keys[at + b] = ordered(sum);
  }
}

__global__ __launch_bounds__(kThreads) void select4_kernel(Select4Args a) {
  __shared__ uint64_t lo_s[kThreads / kWave], hi_s[kThreads / kWave];
  __shared__ int hist[256], wsum[2][kThreads / kWave], bin_s, above_s;
  const Cache4View& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int h = blockIdx.x % c.H;
  const int s = (blockIdx.x / c.H) % c.S;
  const int l = blockIdx.x / (c.H * c.S);
  int32_t* __restrict__ out = a.blocks + (size_t)blockIdx.x * a.n;
  const int nb = blocks_of(c, s);
  if (nb <= a.n) {
    for (int i = tid; i < a.n; i += kThreads) out[i] = i < nb ? i : -1;
    return;
  }
  const uint64_t* __restrict__ keys =
      a.keys + (size_t)(l * c.H + h) * c.nblk + c.cu_rows[s] / kBlock4 + s;
  // candidates [b0, b1), of which `want` are taken: those with key >> shift
  // above `bin`, all or the first `ties` of those with key >> shift == bin
  const int b0 = a.first, b1 = nb - a.last, want = a.n - a.first - a.last;
  int shift = 0, ties = 0;
  uint64_t bin = 0;
  if (want > 0) {
    uint64_t lo = ~uint64_t(0), hi = 0;
    for (int b = b0 + tid; b < b1; b += kThreads) {
      lo = min(lo, keys[b]);
      hi = max(hi, keys[b]);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
      lo = min(lo, (uint64_t)__shfl_xor((unsigned long long)lo, off, kWave));
      hi = max(hi, (uint64_t)__shfl_xor((unsigned long long)hi, off, kWave));
    }
    if (lane == 0) {
      lo_s[wave] = lo;
      hi_s[wave] = hi;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / kWave; ++w) {
      lo = min(lo, lo_s[w]);
      hi = max(hi, hi_s[w]);
    }
    // digits of 8 bits from the highest bit in which the keys differ
    int top = lo == hi ? 0 : 64 - __builtin_clzll(lo ^ hi);  // bits that differ
    shift = max(top - 8, 0);
    uint64_t prefix = top == 64 ? 0 : hi >> top;  // of the candidates left, at `top`
    ties = want;
    for (;;) {  // at most 8 rounds: top falls by 8 each
      hist[tid] = 0;
      __syncthreads();
      for (int b = b0 + tid; b < b1; b += kThreads) {
        const uint64_t k = keys[b];
        if (top == 64 || k >> top == prefix)
          atomicAdd(&hist[(k >> shift) & ((1 << (top - shift)) - 1)], 1);
      }
      __syncthreads();
      // thread t: digit 255 - t; an inclusive prefix from the greatest digit
      const int mine = hist[255 - tid];
      int incl = mine;
#pragma unroll
      for (int off = 1; off < kWave; off <<= 1) {
        const int x = __shfl_up(incl, off, kWave);
        if (lane >= off) incl += x;
      }
      if (lane == kWave - 1) wsum[0][wave] = incl;
      __syncthreads();
      for (int w = 0; w < wave; ++w) incl += wsum[0][w];
      if (incl >= ties && incl - mine < ties) {  // one thread
        bin_s = 255 - tid;
        above_s = incl - mine;
      }
      __syncthreads();
      const int digit = bin_s, in_bin = hist[digit];
      ties -= above_s;
      prefix = top == 64 ? (uint64_t)digit : (prefix << (top - shift)) | (uint64_t)digit;
      bin = prefix;
      if (in_bin == ties || shift == 0) break;  // uniform
      top = shift;
      shift = max(top - 8, 0);
      __syncthreads();  // hist and bin_s are read above
    }
  }
  // listed ascending: forced ones and those above the bin, then ties in order
  int done = 0, tied = 0;  // blocks listed, ties met so far
  for (int r0 = 0; r0 < nb; r0 += kThreads) {
    const int b = r0 + tid;
    bool in = b < nb && (b < b0 || b >= b1), tie = false;
    if (!in && b < nb && want > 0) {
      const uint64_t k = keys[b] >> shift;
      in = k > bin;
      tie = k == bin;
    }
    const uint64_t tmask = ballot(tie);
    __syncthreads();
    if (lane == 0) wsum[0][wave] = __popcll(tmask);
    __syncthreads();
    int t = tied + lanes_below(tmask);
    for (int w = 0; w < wave; ++w) t += wsum[0][w];
    for (int w = 0; w < kThreads / kWave; ++w) tied += wsum[0][w];
    in |= tie && t < ties;
    const uint64_t imask = ballot(in);
    if (lane == 0) wsum[1][wave] = __popcll(imask);
    __syncthreads();
    int at = done + lanes_below(imask);
    for (int w = 0; w < wave; ++w) at += wsum[1][w];
    for (int w = 0; w < kThreads / kWave; ++w) done += wsum[1][w];
    if (in && at < a.n) out[at] = b;
  }
}

}  // namespace

int score4_chunks(const int32_t* cu_rows_host, int S) {
  int64_t n = 0;
  for (int s = 0; s < S; ++s) {
    const int64_t nb = ((int64_t)(cu_rows_host[s + 1] - cu_rows_host[s]) + kBlock4 - 1) / kBlock4;
    n += (nb + kChunk - 1) / kChunk;
  }
  return (int)n;
}

hipError_t launch_select4(const Select4Args& a, hipStream_t st) {
  if (a.chunks > 0) {
    const dim3 grid((unsigned)(a.c.L * a.c.H) * (unsigned)a.chunks);
    if (a.c.d == 128) hipLaunchKernelGGL(score4_kernel<128>, grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL(score4_kernel<64>, grid, dim3(kThreads), 0, st, a);
  }
  hipLaunchKernelGGL(select4_kernel, dim3((unsigned)(a.c.L * a.c.S) * (unsigned)a.c.H),
                     dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace stepkv
