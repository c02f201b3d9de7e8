// The blocks that a decode step attends to (stepkv_cache4_select_blocks): the
// score of every block that is ranked,
//   sum_i a_i kmax_i + b_i kmin_i,  a = sum_g max(q_g, 0), b = sum_g min(q_g, 0),
// which is sum_g sum_i max(q_gi kmin_i, q_gi kmax_i) with one product per
// channel and bound whatever the group, and the threshold among them. 4d bytes
// of bounds a block bound it. The sums are kept in 64 bits and taken in one order
// for every block: the products are exact, so are sums of values within some 2^30
// of each other, and equal bounds give equal scores whatever their size (32-bit
// sums would rank close blocks by their roundings).
//
// select4_kernel: one workgroup per (layer, sequence, KV head) scores its blocks
// into LDS, finds the threshold by radix passes over the ordered keys and lists
// the blocks; where that would take long, score4_kernel scores them all over the
// chip, through the workspace.
#include "cache4_device.h"

#include <algorithm>

namespace stepkv {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 64;        // blocks a workgroup of score4_kernel scores
constexpr int kLdsBlocks = 4096;  // keys that select4_kernel holds itself

__device__ __forceinline__ int blocks_of(const Cache4View& c, int s) {
  return (held_tokens(c, s) + kBlock4 - 1) / kBlock4;
}

__device__ __forceinline__ int blocks_const(const Cache4View& c, int s) {  // of a uniform s
  return (held_const(c, s) + kBlock4 - 1) / kBlock4;
}

// Doubles as unsigned integers in the same order; NaN as -inf, -0 as +0.
__device__ __forceinline__ uint64_t ordered(double x) {
  if (x != x) x = -INFINITY;
  const uint64_t b = __builtin_bit_cast(uint64_t, x + 0.0);
  return b >> 63 ? ~b : b | (uint64_t(1) << 63);
}

// The least x of the wave: within 16 lanes by DPP exchanges, then the four rows.
template <int CTRL>
__device__ __forceinline__ uint64_t dpp_min(uint64_t x) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(x >> 32), CTRL, 0xf, 0xf, true);
  return min(x, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ uint64_t wave_min(uint64_t x) {
  x = dpp_min<0xB1>(x);
  x = dpp_min<0x4E>(x);
  x = dpp_min<0x141>(x);
  x = dpp_min<0x140>(x);
  uint64_t r = ~uint64_t(0);
#pragma unroll
  for (int row = 0; row < 4; ++row) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)x, 16 * row);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), 16 * row);
    r = min(r, (uint64_t)hi << 32 | lo);
  }
  return r;
}

// x plus that of the lanes which hold the same block (D / 8 of them): DPP
// exchanges within 4, 8 and 16 lanes.
template <int CTRL>
__device__ __forceinline__ double dpp_add(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)u, CTRL, 0xf, 0xf, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(u >> 32), CTRL, 0xf, 0xf, true);
  return x + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int D>
__device__ __forceinline__ double block_sum(double x) {
  x = dpp_add<0xB1>(x);   // lane ^ 1
  x = dpp_add<0x4E>(x);   // lane ^ 2
  x = dpp_add<0x141>(x);  // row_half_mirror: the other four of 8
  if constexpr (D == 128) x = dpp_add<0x140>(x);  // row_mirror: the other eight of 16
  return x;
}

// Scores blocks [b0, b1) of a sequence (bounds x, of block 0) for the G query
// heads at q, keys to keys[b]; coef: LDS. D / 8 lanes a block: a lane holds 8
// channels of its minima and maxima and their coefficients, and the next
// rounds' bounds. Every thread of the workgroup calls it.
template <int D, int THREADS>
__device__ __forceinline__ void score_blocks(const uint16_t* __restrict__ q, int G,
                                             const uint16_t* __restrict__ x, int b0, int b1,
                                             uint64_t* keys, double (&coef)[2][D]) {
  constexpr int LB = D / 8, STEP = THREADS / LB;  // lanes a block, blocks a round
  constexpr int AHEAD = 4;
  const int i = threadIdx.x % LB;
  x += 8 * i;
  u32x4_t w[AHEAD][2];
  auto load = [&](u32x4_t (&v)[2], int b) __attribute__((always_inline)) {
    const uint16_t* __restrict__ p = x + (size_t)min(b, b1 - 1) * 2 * D;
    v[0] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
    v[1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p + D));
  };
  const int mine = b0 + (int)(threadIdx.x / LB);
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) load(w[u], mine + u * STEP);  // while the coefficients are summed
  if (threadIdx.x < D) {
    double up = 0.0, down = 0.0;
#pragma unroll 8
    for (int g = 0; g < G; ++g) {
      const float y = bf16_float(q[(size_t)g * D + threadIdx.x]);
      up += !(y <= 0.f) ? (double)y : 0.0;  // a NaN too: it makes every score one
      down += y < 0.f ? (double)y : 0.0;
    }
    coef[0][threadIdx.x] = down;  // of the minimum
    coef[1][threadIdx.x] = up;
  }
  __syncthreads();
  double c[2][8];
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int e = 0; e < 8; ++e) c[which][e] = coef[which][8 * i + e];
  for (int r = b0; r < b1; r += AHEAD * STEP) {  // uniform over the workgroup
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int b = mine + (r - b0) + u * STEP;
      double sum[2] = {0.0, 0.0};
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int which = 0; which < 2; ++which) {
          const uint32_t v = w[u][which][e / 2];
          sum[which] = fma((double)__uint_as_float(e & 1 ? v & 0xffff0000u : v << 16),
                           c[which][e], sum[which]);
        }
      if (r + AHEAD * STEP + u * STEP < b1) load(w[u], b + AHEAD * STEP);  // uniform
      const double total = block_sum<D>(sum[0] + sum[1]);
      if (i == 0 && b < b1) keys[b] = ordered(total);
    }
  }
}

template <int D>
__global__ __launch_bounds__(kThreads) void score4_kernel(Select4Args a) {
  __shared__ double coef[2][D];
  const Cache4View& c = a.c;
  const int lh = uniform(blockIdx.x / a.chunks), at = uniform(blockIdx.x - lh * a.chunks);
  const int l = uniform(lh / c.H), h = lh - l * c.H;
  int s = 0, first = 0;
  if (c.S == 1 && at * kChunk >= (blocks_const(c, 0) > a.n ? blocks_const(c, 0) : 0)) return;
  if (c.S > 1) locate_item(c.S, at, [&](int sq) {
    const int nb = blocks_of(c, sq);
    return nb > a.n ? (nb + kChunk - 1) / kChunk : 0;  // shorter ones are not ranked
  }, s, first);
  if (s < 0) return;
  const int b0 = (at - first) * kChunk;
  const size_t base = (size_t)lh * c.nblk + read_const(c.cu_rows, s) / kBlock4 + s;
  score_blocks<D, kThreads>(a.q + (((size_t)l * c.S + s) * a.Hq + h * a.G) * D, a.G,
                            c.k_bounds + base * 2 * D, b0, min(blocks_const(c, s), b0 + kChunk),
                            a.keys + base, coef);
}

// HERE: scores the blocks itself, into LDS (at most KEYS); otherwise score4_kernel did.
template <int D, int THREADS, bool HERE, int KEYS>
__global__ __launch_bounds__(THREADS) void select4_kernel(Select4Args a) {
  constexpr int W = THREADS / kWave;
  __shared__ uint64_t own[KEYS];
  __shared__ double coef[2][HERE ? D : 1];
  __shared__ uint64_t lo_s[W], hi_s[W];
  __shared__ int hist[256], bin_s, ties_s, in_s, cnt[2][W];
  const Cache4View& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int h = uniform(blockIdx.x % c.H);
  const int s = uniform((blockIdx.x / c.H) % c.S), l = uniform(blockIdx.x / (c.H * c.S));
  int32_t* __restrict__ out = a.blocks + (size_t)blockIdx.x * a.n;
  const int nb = blocks_const(c, s);
  if (nb <= a.n) {
    for (int i = tid; i < a.n; i += THREADS) out[i] = i < nb ? i : -1;
    return;
  }
  const size_t base = (size_t)(l * c.H + h) * c.nblk + read_const(c.cu_rows, s) / kBlock4 + s;
  const uint64_t* keys = a.keys + base;
  // candidates [b0, b1), of which `want` are taken: those with key >> shift
  // above `bin`, and the first `ties` of those with key >> shift == bin
  const int b0 = a.first, b1 = nb - a.last, want = a.n - a.first - a.last;
  if constexpr (HERE) {
    if (want > 0)
      score_blocks<D, THREADS>(a.q + (((size_t)l * c.S + s) * a.Hq + h * a.G) * D, a.G,
                               c.k_bounds + base * 2 * D, b0, b1, own, coef);
    keys = own;
    __syncthreads();
  } else if (nb <= KEYS) {
    for (int b = tid; b < nb; b += THREADS) own[b] = keys[b];
    keys = own;
    __syncthreads();
  }
  int shift = 0, ties = 0;
  uint64_t bin = 0;
  if (want > 0) {
    if (tid < 256) hist[tid] = 0;
    uint64_t lo = ~uint64_t(0), hi = 0;
    for (int b = b0 + tid; b < b1; b += THREADS) {
      const uint64_t k = keys[b];
      lo = min(lo, k);
      hi = max(hi, k);
    }
    lo = wave_min(lo);
    hi = ~wave_min(~hi);
    if (lane == 0) {
      lo_s[wave] = lo;
      hi_s[wave] = hi;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) {
      lo = min(lo, lo_s[w]);
      hi = max(hi, hi_s[w]);
    }
    // digits of 8 bits from the highest bit in which the keys differ
    int top = lo == hi ? 0 : 64 - __builtin_clzll(lo ^ hi);  // bits that differ
    uint64_t prefix = top == 64 ? 0 : hi >> top;  // of the candidates left, at `top`
    ties = want;
    for (;;) {  // at most 8 rounds: top falls by 8 each
      shift = max(top - 8, 0);
      for (int b = b0 + tid; b < b1; b += THREADS) {
        const uint64_t k = keys[b];
        if (top == 64 || k >> top == prefix)
          atomicAdd(&hist[(k >> shift) & ((1 << (top - shift)) - 1)], 1);
      }
      __syncthreads();
      if (wave == 0) {
        // lane t: digits 255 - 4 t .. 252 - 4 t, counted from the greatest
        int n[4], sum = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          n[k] = hist[255 - 4 * lane - k];
          hist[255 - 4 * lane - k] = 0;  // for the next round
          sum += n[k];
        }
        int above = wave_scan(sum) - sum;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (above < ties && above + n[k] >= ties) {  // one lane, one digit
            bin_s = 255 - 4 * lane - k;
            ties_s = ties - above;
            in_s = n[k];
          }
          above += n[k];
        }
      }
      __syncthreads();
      ties = ties_s;
      prefix = top == 64 ? (uint64_t)bin_s : (prefix << (top - shift)) | (uint64_t)bin_s;
      top = shift;
      if (in_s == ties || shift == 0) break;  // uniform
      __syncthreads();  // bin_s and the others are read above
    }
    bin = prefix;
  }
  // listed ascending, each wave a run of blocks: counted, then written
  const int run = (nb + THREADS - 1) / THREADS * kWave;
  const int r0 = wave * run, r1 = min(nb, r0 + run);
  auto look = [&](int b, bool& in, bool& tie) __attribute__((always_inline)) {
    in = b < r1 && (b < b0 || b >= b1);
    tie = false;
    if (b < r1 && !in && want > 0) {
      const uint64_t k = keys[b] >> shift;
      in = k > bin;
      tie = k == bin;
    }
  };
  int nin = 0, ntie = 0;
  bool in, tie;
  for (int b = r0; b < r1; b += kWave) {
    look(b + lane, in, tie);
    nin += __popcll(ballot(in));
    ntie += __popcll(ballot(tie));
  }
  if (lane == 0) {
    cnt[0][wave] = nin;
    cnt[1][wave] = ntie;
  }
  __syncthreads();
  int done = 0, tied = 0;  // listed, and ties met, before this wave's run
  for (int w = 0; w < wave; ++w) {
    done += cnt[0][w] + min(max(ties - tied, 0), cnt[1][w]);
    tied += cnt[1][w];
  }
  for (int b = r0; b < r1; b += kWave) {
    look(b + lane, in, tie);
    const uint64_t tmask = ballot(tie);
    in |= tie && tied + lanes_below(tmask) < ties;
    const uint64_t imask = ballot(in);
    const int at = done + lanes_below(imask);
    if (in && at < a.n) out[at] = b + lane;
    done += __popcll(imask);
    tied += __popcll(tmask);
  }
}

}  // namespace

// A workgroup that scores a whole sequence has its bounds' products to do alone
// (about 10 ns a block), which saves a launch and the keys' way through memory for
// up to kAlone blocks, and for up to kLdsBlocks where there are sequences and
// heads for every compute unit (28 layers x 4 heads x 16 sequences of up to 128
// blocks: 24 us, in two launches 30). Otherwise score4_kernel spreads them (64
// heads x 2048 blocks 25 us, alone 31; 8 heads x 512: 11.5 and 13.4, but the
// second launch costs its host more).
void plan_select4(Select4Args& a, const int32_t* cu_rows_host) {
  constexpr int kAlone = 768;
  int64_t n = 0, most = 0;
  for (int s = 0; s < a.c.S; ++s) {
    const int64_t nb = ((int64_t)(cu_rows_host[s + 1] - cu_rows_host[s]) + kBlock4 - 1) / kBlock4;
    n += (nb + kChunk - 1) / kChunk;
    most = std::max(most, nb);
  }
  const int64_t rows = (int64_t)a.c.L * a.c.S * a.c.H;
  a.most = (int)most;
  a.chunks = most <= kAlone || (most <= kLdsBlocks && rows >= 512) ? 0 : (int)n;
}

namespace {

// Threads of a workgroup of select4_kernel, and whether it holds few keys: with
// many rows of short sequences more workgroups share a compute unit.
bool few_keys(const Select4Args& a) {
  return a.chunks == 0 && (int64_t)a.c.L * a.c.S * a.c.H >= 512 && a.most <= 1024;
}
int select_threads(const Select4Args& a) {
  return a.chunks > 0 ? 512 : few_keys(a) ? kThreads : 1024;
}

template <int D>
void launch_select(const Select4Args& a, hipStream_t st) {
  const dim3 rows((unsigned)(a.c.L * a.c.S) * (unsigned)a.c.H), threads(select_threads(a));
  if (a.chunks > 0) {
    hipLaunchKernelGGL(score4_kernel<D>, dim3((unsigned)(a.c.L * a.c.H) * (unsigned)a.chunks),
                       dim3(kThreads), 0, st, a);
    hipLaunchKernelGGL((select4_kernel<D, 512, false, kLdsBlocks>), rows, threads, 0, st, a);
  } else if (few_keys(a)) {
    hipLaunchKernelGGL((select4_kernel<D, kThreads, true, 1024>), rows, threads, 0, st, a);
  } else {
    hipLaunchKernelGGL((select4_kernel<D, 1024, true, kLdsBlocks>), rows, threads, 0, st, a);
  }
}

}  // namespace

bool select4_fits(const Select4Args& a) {
  return grid_fits((int64_t)a.c.L * a.c.H * a.chunks, kThreads) &&
         grid_fits((int64_t)a.c.L * a.c.S * a.c.H, select_threads(a));
}

hipError_t launch_select4(const Select4Args& a, hipStream_t st) {
  if (a.c.d == 128) launch_select<128>(a, st);
  else launch_select<64>(a, st);
  return hipGetLastError();
}

}  // namespace stepkv
