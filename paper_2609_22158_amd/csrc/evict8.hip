// Eviction from the 8-bit cache by gathered weight (include/stepkv_cache8.h):
// of the n tokens of a (layer, KV head, sequence) the `keep` best stay, and those
// of them in rows `keep` and above move into the rows below that become free. So
// only as many rows move as tokens leave, none is read and written by different
// waves, and nothing waits for anything: sources lie at `keep` and above,
// destinations below.
//
// evict8_kernel: one workgroup per (layer, KV head, sequence) finds the key of the
// keep-th best token by radix search over the weights' bits, and lists the moves.
// move8_kernel: a wave per 64-token block that rows move into: the power of two
// that they need, the rounding of the block's other tokens if its scale grows, then
// the rows, their weights and positions. A block partly below `keep` is one that
// rows leave and others enter: its scales as they were are kept by the selection.
#include "cache8_device.h"

#include <algorithm>

namespace stepkv {
namespace {

constexpr int kThreads = 1024;
constexpr int kWavesS = kThreads / kWave;
constexpr int kMoveThreads = 256;

// Tokens that stay in any case hold this key, above every weight's (+inf: 0xFF800000).
constexpr uint32_t kStays = 0xFFFFFFFFu;

// Order-preserving key of a weight: NaN -> -inf and -0 -> +0 in float arithmetic,
// then the sign flip.
__device__ __forceinline__ uint32_t order_key(float p) {
  const uint32_t u = __float_as_uint(fmaxf(p, -INFINITY) + 0.0f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

struct Ranks {  // before a thread's token: free rows, moving ones, ties
  int free, move, tie;
};

__global__ __launch_bounds__(kThreads) void evict8_kernel(Evict8Args a) {
  __shared__ uint32_t hist[256];
  __shared__ int wave_n[3][kWavesS];
  __shared__ uint32_t found[2];  // bin, rank within it
  const Cache8View& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  if (blockIdx.x == 0 && wave == 0) report_rooms(c);
  const int lh = uniform(blockIdx.x / c.S), s = uniform(blockIdx.x - lh * c.S);
  const int n = held_const(c, s);
  const int keep = a.keeps ? max(1, read_const(a.keeps, s)) : a.keep;
  Evict8Head* const head = a.heads + blockIdx.x;
  if (n <= keep) {  // uniform
    if (tid == 0) *head = Evict8Head{0, -1, 0.f, 0.f};
    return;
  }
  const int row0 = read_const(c.cu_rows, s);
  const float* __restrict__ w = c.weights + (size_t)lh * c.rows + row0;
  const int32_t* __restrict__ pos = c.positions + (size_t)lh * c.rows + row0;
  const int64_t recent = (int64_t)read_const(c.seen, s) - a.recent;  // from this position on
  auto key_of = [&](int j) {
    const int p = pos[j];
    return p < a.first || p >= recent ? kStays : order_key(w[j]);
  };
  // the key of the keep-th greatest, 8 bits at a time
  uint32_t prefix = 0u;
  int rank = keep;  // within the keys that share the prefix
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0u;
    __syncthreads();
    for (int j = tid; j < n; j += kThreads) {
      const uint32_t k = key_of(j);
      if (shift == 24 || (k ^ prefix) >> (shift + 8) == 0u) atomicAdd(&hist[(k >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (wave == 0) {  // lane l: bins 255 - 4 l .. 252 - 4 l, from the top
      uint32_t own = 0u;
#pragma unroll
      for (int i = 0; i < 4; ++i) own += hist[255 - 4 * lane - i];
      int above = wave_scan((int)own) - (int)own;
      if (above < rank && rank <= above + (int)own) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int bin = 255 - 4 * lane - i, cnt = (int)hist[bin];
          if (above < rank && rank <= above + cnt) {
            found[0] = (uint32_t)bin;
            found[1] = (uint32_t)(rank - above);
          }
          above += cnt;
        }
      }
    }
    __syncthreads();
    prefix |= found[0] << shift;
    rank = (int)found[1];
  }
  // the moves: the i-th row to be freed and the i-th token that moves
  int2* const moves = a.moves + (size_t)lh * (c.rows / 2) + row0 / 2;
  Ranks base{0, 0, 0};
  for (int j0 = 0; j0 < n; j0 += kThreads) {
    const int j = j0 + tid;
    const uint32_t k = j < n ? key_of(j) : 0u;
    const bool tie = j < n && k == prefix;
    const uint64_t ties = ballot(tie);
    if (lane == 0) wave_n[2][wave] = __popcll(ties);
    __syncthreads();
    int tb = base.tie, tt = 0;
    for (int v = 0; v < kWavesS; ++v) {
      if (v < wave) tb += wave_n[2][v];
      tt += wave_n[2][v];
    }
    const bool stays = j < n && (k > prefix || (tie && tb + lanes_below(ties) < rank));
    const uint64_t frees = ballot(j < keep && !stays), goes = ballot(j >= keep && stays);
    if (lane == 0) {
      wave_n[0][wave] = __popcll(frees);
      wave_n[1][wave] = __popcll(goes);
    }
    __syncthreads();
    int fb = base.free, ft = 0, gb = base.move, gt = 0;
    for (int v = 0; v < kWavesS; ++v) {
      if (v < wave) {
        fb += wave_n[0][v];
        gb += wave_n[1][v];
      }
      ft += wave_n[0][v];
      gt += wave_n[1][v];
    }
    if (j < keep && !stays) moves[fb + lanes_below(frees)].x = j;
    if (j >= keep && stays) moves[gb + lanes_below(goes)].y = j;
    base.tie += tt;
    base.free += ft;
    base.move += gt;
    __syncthreads();  // wave_n is read
  }
  if (tid == 0) {
    const size_t sc = (size_t)lh * c.nblk + first_block(row0, s) + keep / kBlock8;
    *head = Evict8Head{base.move, keep, c.k_scales[sc], c.v_scales[sc]};
  }
}

// The exponent that e4m3 codes with these largest magnitude bits need, as
// elements of a block with exponent e: of 1.m * 2^(E - 7), E - 15 + e for
// 1.m <= 1.8125 and one more above.
__device__ __forceinline__ int need_of_code(uint32_t top, int e) {
  if (top == 0u) return kLeast8;
  int x;
  if (top >= 8u) {
    x = (int)(top >> 3) - 15 + ((top & 7u) == 7u ? 1 : 0);
  } else {  // m * 2^-9: 7 = 1.75 * 2^2 needs no more than 4
    x = 31 - __builtin_clz(top) - 9 - 8;
  }
  return min(max(x + e, kLeast8), kMost8);
}

// The largest magnitude of the four codes of a word, NaN apart.
__device__ __forceinline__ uint32_t top_code(uint32_t w, uint32_t top) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t m = (w >> (8 * i)) & 0x7fu;
    top = m == 0x7fu ? top : max(top, m);
  }
  return top;
}

__device__ __forceinline__ u32x4_t regrid16(u32x4_t w, float from, float to) {
  u32x4_t r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const u32x2_t x = spread4(w[i], from);
    r[i] = round4(x[0], x[1], to);
  }
  return r;
}

// A wave per block that rows move into. Lanes hold 16 bytes of a row.
template <int D>
__global__ __launch_bounds__(kMoveThreads) void move8_kernel(Evict8Args a) {
  constexpr int PR = D / 16;      // pieces of a row
  constexpr int RP = kWave / PR;  // rows at a time
  const Cache8View& c = a.c;
  const int lane = threadIdx.x & 63;
  const int64_t worker = (int64_t)blockIdx.x * (kMoveThreads / kWave) + uniform(threadIdx.x >> 6);
  const int at = uniform((int)(worker / a.workers));  // (layer, KV head) and sequence
  const int part = uniform((int)(worker - (int64_t)at * a.workers));
  if (at >= c.L * c.H * c.S) return;
  const int lh = uniform(at / c.S), s = uniform(at - lh * c.S);
  const Evict8Head head = a.heads[at];
  if (head.keep < 0) return;
  if (lh == 0 && part == 0 && lane == 0) c.lens[s] = head.keep;
  const int row0 = read_const(c.cu_rows, s);
  const int2* __restrict__ moves = a.moves + (size_t)lh * (c.rows / 2) + row0 / 2;
  const int blocks = (head.keep + kBlock8 - 1) / kBlock8;
  const int b_first = (int)((int64_t)blocks * part / a.workers);
  const int b_end = (int)((int64_t)blocks * (part + 1) / a.workers);
  // the first move into block b_first or above
  int lo = 0, hi = head.moves;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (moves[mid].x < b_first * kBlock8) lo = mid + 1;
    else hi = mid;
  }
  const size_t base = (size_t)lh * c.rows + row0;
  const size_t scales = (size_t)lh * c.nblk + first_block(row0, s);
  const int sub = lane / PR, piece = lane % PR;
  for (int i = uniform(lo); i < head.moves;) {  // moves i .. i + count - 1 into one block
    const int b = uniform(moves[i].x / kBlock8);
    if (b >= b_end) return;
    int2 m = make_int2(-1, -1);
    if (i + lane < head.moves) m = moves[i + lane];
    const bool mine = m.x >= 0 && m.x / kBlock8 == b;
    const int count = __popcll(ballot(mine));  // they are ascending: the first lanes
    const float k_old = c.k_scales[scales + b], v_old = c.v_scales[scales + b];
    // this lane's move's scales, as they were before any row moved
    float ks = 1.f, vs = 1.f;
    if (mine) {
      const bool edge = m.y / kBlock8 == head.keep / kBlock8;
      ks = edge ? head.k_scale : c.k_scales[scales + m.y / kBlock8];
      vs = edge ? head.v_scale : c.v_scales[scales + m.y / kBlock8];
    }
    uint64_t taken = mine ? 1ull << (m.x % kBlock8) : 0ull;  // rows that are replaced
    int ek = kLeast8, ev = kLeast8;
    for (int j0 = 0; j0 < count; j0 += RP) {
      const int j = min(j0 + sub, count - 1);
      const int from = __shfl(m.y, j, kWave);
      const float fk = __shfl(ks, j, kWave), fv = __shfl(vs, j, kWave);
      const u32x4_t kw = reinterpret_cast<const u32x4_t*>(c.k_codes + (base + from) * D)[piece];
      const u32x4_t vw = reinterpret_cast<const u32x4_t*>(c.v_codes + (base + from) * D)[piece];
      uint32_t kt = 0u, vt = 0u;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        kt = top_code(kw[q], kt);
        vt = top_code(vw[q], vt);
      }
      ek = max(ek, need_of_code(kt, exponent_of(fk)));
      ev = max(ev, need_of_code(vt, exponent_of(fv)));
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
      ek = max(ek, __shfl_xor(ek, off, kWave));
      ev = max(ev, __shfl_xor(ev, off, kWave));
      taken |= (uint64_t)__shfl_xor((unsigned long long)taken, off, kWave);
    }
    const int ok = uniform(exponent_of(k_old)), ov = uniform(exponent_of(v_old));
    ek = uniform(min(max(ek, ok), kMost8));
    ev = uniform(min(max(ev, ov), kMost8));
    if (ek > ok || ev > ov) {  // the block's other tokens
      const float kn = pow2_of(ek), vn = pow2_of(ev);
      for (int j0 = 0; j0 < kBlock8; j0 += RP) {
        const int j = j0 + sub;
        if (b * kBlock8 + j >= head.keep || (taken >> j & 1ull)) continue;
        const size_t r = base + (size_t)b * kBlock8 + j;
        if (ek > ok) {
          u32x4_t* p = reinterpret_cast<u32x4_t*>(c.k_codes + r * D) + piece;
          *p = regrid16(*p, k_old, kn);
        }
        if (ev > ov) {
          u32x4_t* p = reinterpret_cast<u32x4_t*>(c.v_codes + r * D) + piece;
          *p = regrid16(*p, v_old, vn);
        }
      }
      if (lane == 0) {
        c.k_scales[scales + b] = kn;
        c.v_scales[scales + b] = vn;
      }
    }
    for (int j0 = 0; j0 < count; j0 += RP) {
      const int j = j0 + sub;
      const int from = __shfl(m.y, min(j, count - 1), kWave), to = __shfl(m.x, min(j, count - 1), kWave);
      const float fk = __shfl(ks, min(j, count - 1), kWave), fv = __shfl(vs, min(j, count - 1), kWave);
      if (j >= count) continue;
      const u32x4_t kw = reinterpret_cast<const u32x4_t*>(c.k_codes + (base + from) * D)[piece];
      const u32x4_t vw = reinterpret_cast<const u32x4_t*>(c.v_codes + (base + from) * D)[piece];
      reinterpret_cast<u32x4_t*>(c.k_codes + (base + to) * D)[piece] = regrid16(kw, fk, pow2_of(ek));
      reinterpret_cast<u32x4_t*>(c.v_codes + (base + to) * D)[piece] = regrid16(vw, fv, pow2_of(ev));
    }
    if (mine) {
      c.weights[base + m.x] = c.weights[base + m.y];
      c.positions[base + m.x] = c.positions[base + m.y];
    }
    i += count;
  }
}

int64_t move_workgroups(const Evict8Args& a) {
  return ((int64_t)a.c.L * a.c.H * a.c.S * a.workers + kMoveThreads / kWave - 1) / (kMoveThreads / kWave);
}

}  // namespace

// Waves that move rows: 16 for each compute unit, but no more than a sequence can
// have blocks.
void plan_evict8(Evict8Args& a, const int32_t* cu_rows_host) {
  int64_t longest = 0;
  for (int s = 0; s < a.c.S; ++s)
    longest = std::max<int64_t>(longest, cu_rows_host[s + 1] - cu_rows_host[s]);
  const int64_t heads = (int64_t)a.c.L * a.c.H * a.c.S;
  a.workers = (int)std::max<int64_t>(
      1, std::min<int64_t>((4096 + heads - 1) / heads, (longest + kBlock8 - 1) / kBlock8));
}

bool evict8_fits(const Evict8Args& a) {
  return grid_fits((int64_t)a.c.L * a.c.H * a.c.S, kThreads) &&
         grid_fits(move_workgroups(a), kMoveThreads);
}

hipError_t launch_evict8(const Evict8Args& a, hipStream_t st) {
  hipLaunchKernelGGL(evict8_kernel, dim3((unsigned)(a.c.L * a.c.H) * (unsigned)a.c.S), dim3(kThreads),
                     0, st, a);
  const dim3 grid((unsigned)move_workgroups(a));
  if (a.c.d == 128)
    hipLaunchKernelGGL(move8_kernel<128>, grid, dim3(kMoveThreads), 0, st, a);
  else
    hipLaunchKernelGGL(move8_kernel<64>, grid, dim3(kMoveThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace stepkv
