// Eviction from the 8-bit cache by gathered weight (include/stepkv_cache8.h):
// of the n tokens of a (layer, KV head, sequence) the `keep` best stay, and those
// of them in rows `keep` and above move into the rows below that become free. So
// only as many rows move as tokens leave, none is read and written by different
// waves, and nothing waits for anything: sources lie at `keep` and above,
// destinations below.
//
// evict8_kernel: one workgroup per (layer, KV head, sequence) finds the key of the
// keep-th best token by radix search over the weights' bits, and lists the moves.
// A wave holds a run of consecutive rows, 64 at a time, one key a lane and
// register; so which of them stay is a mask in scalar registers, and what waves
// have to tell each other is a few totals. The weights and positions, 8 bytes a
// token, are read once (rows past 1024 x 80: once a phase).
// move8_kernel: the rows, their weights and positions, 16 moves a wave; a wave has
// all the moves into a block, so that it can round the block's other tokens if
// its scale grows. A block partly below `keep` is one that rows leave and others
// enter: its scales as they were are kept by the selection.
#include "cache8_device.h"

#include <algorithm>
#include <type_traits>

namespace stepkv {
namespace {

constexpr int kMoveThreads = 256;
constexpr int kMoveChunk = 16;  // moves that a wave takes at a time, about

// Tokens that stay in any case hold this key, above every weight's (+inf: 0xFF800000).
constexpr uint32_t kStays = 0xFFFFFFFFu;
constexpr int kDigit = 11;
constexpr int kBins = 1 << kDigit;

// Order-preserving key of a weight: NaN -> -inf and -0 -> +0 in float arithmetic,
// then the sign flip. At least 0x007FFFFF; rows past the sequence hold 0.
__device__ __forceinline__ uint32_t order_key(float p) {
  const uint32_t u = __float_as_uint(fmaxf(p, -INFINITY) + 0.0f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

template <int W>
struct Scratch8 {
  uint32_t hist[kBins];
  uint32_t total[W];
  int count[3][W];   // of every wave: rows to be freed, rows that move, ties
  uint32_t found[3];  // bin, rank within it, keys in it
};

// The bin of sh.hist that holds the rank-th greatest key (and clears sh.hist):
// thread t looks at bins kBins - 1 - PB t and the PB - 1 below, so that the prefix
// in thread order counts from the top.
template <int W>
__device__ __forceinline__ void find_bin(Scratch8<W>& sh, uint32_t rank) {
  constexpr int PB = kBins / (W * kWave);
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int top = kBins - 1 - PB * tid;
  uint32_t n[PB], own = 0u;
#pragma unroll
  for (int i = 0; i < PB; ++i) {
    n[i] = sh.hist[top - i];
    own += n[i];
  }
#pragma unroll
  for (int i = 0; i < PB; ++i) sh.hist[top - i] = 0u;
  const uint32_t incl = (uint32_t)wave_scan((int)own);
  if (lane == kWave - 1) sh.total[wave] = incl;
  __syncthreads();
  uint32_t above = incl - own;
#pragma unroll
  for (int v = 0; v < W; ++v) above += v < wave ? sh.total[v] : 0u;
  if (above < rank && rank <= above + own) {
#pragma unroll
    for (int i = 0; i < PB; ++i) {
      if (above < rank && rank <= above + n[i]) {
        sh.found[0] = (uint32_t)(top - i);
        sh.found[1] = rank - above;
        sh.found[2] = n[i];
      }
      above += n[i];
    }
  }
  __syncthreads();
}

// Adds one to the bin of every lane with `in`: lanes of one bin as one, where they
// are many (equal weights; atomics on one word run one after another).
__device__ __forceinline__ void add_to_bins(uint32_t* hist, bool in, uint32_t bin, int lane) {
  const uint64_t active = ballot(in);
  if (active == 0ull) return;
  const int lead = __builtin_ctzll(active);
  const uint64_t same = ballot(in && bin == (uint32_t)__builtin_amdgcn_readlane((int)bin, lead));
  if (__popcll(same) >= 8) {  // uniform
    if (lane == lead) atomicAdd(&hist[bin], (uint32_t)__popcll(same));
    in = in && !(same >> lane & 1ull);
  }
  if (in) atomicAdd(&hist[bin], 1u);
}

// W waves, NB keys a lane (STREAM: read again in every phase, NB at a time).
template <int W, int NB, bool STREAM>
__global__ __launch_bounds__(W * kWave) void evict8_kernel(Evict8Args a) {
  __shared__ Scratch8<W> sh;
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
  const bool some_stay = a.first > 0 || a.recent > 0;
  // this wave's rows: nb groups of 64 from row j0
  const int nb = (n + W * kWave - 1) / (W * kWave);
  const int j0 = wave * nb * kWave;
  constexpr int kBatch = NB < 8 ? NB : 8;  // loads in flight
  uint32_t keys[NB];
  auto load = [&](int b0, int count) __attribute__((always_inline)) {  // groups b0 .. of this wave
#pragma unroll
    for (int b = 0; b < NB; b += kBatch) {
      if (b >= count) {  // uniform
#pragma unroll
        for (int i = 0; i < kBatch; ++i) keys[b + i] = 0u;
        continue;
      }
      float x[kBatch];
      int p[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int j = min(j0 + (b0 + b + i) * kWave + lane, n - 1);
        x[i] = w[j];
        p[i] = some_stay ? pos[j] : 0;
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int j = j0 + (b0 + b + i) * kWave + lane;
        const bool stays = some_stay && (p[i] < a.first || p[i] >= recent);
        keys[b + i] = b + i < count && j < n ? (stays ? kStays : order_key(x[i])) : 0u;
      }
    }
  };
  // f(group, key) over this wave's rows, in their order
  auto each = [&](auto&& f) __attribute__((always_inline)) {
    if constexpr (STREAM) {
      for (int b0 = 0; b0 < nb; b0 += NB) {
        load(b0, nb - b0);
#pragma unroll
        for (int b = 0; b < NB; ++b) f(b0 + b, keys[b]);
      }
    } else {
#pragma unroll
      for (int b = 0; b < NB; b += kBatch) {
        if (b >= nb) break;  // uniform
#pragma unroll
        for (int i = 0; i < kBatch; ++i) f(b + i, keys[b + i]);
      }
    }
  };
  if constexpr (!STREAM) load(0, nb);
  for (int i = tid; i < kBins; i += W * kWave) sh.hist[i] = 0u;
  __syncthreads();
  // tokens that stay in any case are counted apart: they are many of one key
  int always = 0;
  each([&](int, uint32_t k) __attribute__((always_inline)) {
    always += __popcll(ballot(k == kStays));
    add_to_bins(sh.hist, k != 0u && k != kStays, k >> (32 - kDigit), lane);
  });
  if (lane == 0) sh.count[0][wave] = always;
  __syncthreads();
  always = 0;
#pragma unroll
  for (int v = 0; v < W; ++v) always += sh.count[0][v];
  // keys above t_sure stay, and the first `need` of those equal to it + 1
  uint32_t t_sure;
  int need = 0;
  if (always >= keep) {
    t_sure = kStays - 1u;
    need = keep < always ? keep : 0;
  } else {
    uint32_t prefix = 0u, rank = (uint32_t)(keep - always);
    int shift = 32 - kDigit;
    for (;;) {
      find_bin<W>(sh, rank);
      prefix |= sh.found[0] << shift;
      rank = sh.found[1];
      const bool all = rank == sh.found[2];  // every key of the bin stays
      if (all || shift == 0) {
        t_sure = prefix - 1u;
        need = all ? 0 : (int)rank;
        break;
      }
      const int up = shift, down = max(shift - kDigit, 0);
      each([&](int, uint32_t k) __attribute__((always_inline)) {
        add_to_bins(sh.hist, (k ^ prefix) >> up == 0u && k != kStays, (k & ((1u << up) - 1u)) >> down, lane);
      });
      shift = down;
      __syncthreads();
    }
  }
  const bool all_ties = need == 0;  // ties: keys equal to t_sure + 1, if they do not all stay
  int tie0 = 0;
  if (!all_ties) {
    int ties = 0;
    each([&](int, uint32_t k) __attribute__((always_inline)) { ties += __popcll(ballot(k == t_sure + 1u)); });
    if (lane == 0) sh.count[2][wave] = ties;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < W; ++v) tie0 += v < wave ? sh.count[2][v] : 0;
  }
  // f(first row of 64, rows to be freed, rows that move) of this wave
  auto moves_of = [&](auto&& f) __attribute__((always_inline)) {
    int before = tie0;
    each([&](int b, uint32_t k) __attribute__((always_inline)) {
      uint64_t stay;
      if (all_ties) {  // uniform
        stay = ballot(k > t_sure);
      } else {
        const uint64_t ties = ballot(k == t_sure + 1u);
        stay = ballot(k > t_sure + 1u || (k == t_sure + 1u && before + lanes_below(ties) < need));
        before += __popcll(ties);
      }
      const int j = j0 + b * kWave;
      if (b >= nb) return;  // uniform: a batch may end past the wave's rows
      const uint64_t low = keep - j >= kWave ? ~0ull : (keep > j ? (1ull << (keep - j)) - 1ull : 0ull);
      f(j, ~stay & low, stay & ~low);
    });
  };
  int frees = 0, goes = 0;
  moves_of([&](int, uint64_t free, uint64_t go) __attribute__((always_inline)) {
    frees += __popcll(free);
    goes += __popcll(go);
  });
  __syncthreads();  // sh.count is read above
  if (lane == 0) {
    sh.count[0][wave] = frees;
    sh.count[1][wave] = goes;
  }
  __syncthreads();
  int fb = 0, gb = 0, all = 0;
#pragma unroll
  for (int v = 0; v < W; ++v) {
    fb += v < wave ? sh.count[0][v] : 0;
    gb += v < wave ? sh.count[1][v] : 0;
    all += sh.count[1][v];
  }
  // the moves: the i-th row to be freed and the i-th token that moves
  int2* const moves = a.moves + (size_t)lh * (c.rows / 2) + row0 / 2;
  if (frees + goes > 0)  // uniform over the wave
    moves_of([&](int j, uint64_t free, uint64_t go) __attribute__((always_inline)) {
      if ((free | go) == 0ull) return;
      if (free >> lane & 1ull) moves[fb + lanes_below(free)].x = j + lane;
      if (go >> lane & 1ull) moves[gb + lanes_below(go)].y = j + lane;
      fb += __popcll(free);
      gb += __popcll(go);
    });
  if (tid == 0) {
    const size_t sc = (size_t)lh * c.nblk + first_block(row0, s) + keep / kBlock8;
    *head = Evict8Head{all, keep, c.k_scales[sc], c.v_scales[sc]};
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

// The largest magnitude code of 16 codes.
__device__ __forceinline__ uint32_t top_of16(u32x4_t w) {
  uint32_t t = 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) t = top_code(w[i], t);
  return t;
}

// Chunks of kMoveChunk moves a wave, from the first move into a block to the last
// one: a block's moves are one wave's. Lane i holds move i of up to 64 of a chunk;
// lanes hold 16 bytes of a row.
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
  const size_t base = (size_t)lh * c.rows + row0;
  const size_t scales = (size_t)lh * c.nblk + first_block(row0, s);
  const int sub = lane / PR, piece = lane % PR;
  const int edge = head.keep / kBlock8;
  for (int64_t chunk = part; chunk * kMoveChunk < head.moves; chunk += a.workers) {
    // moves lo .. end - 1: from the first that begins a block at or past the chunk's
    // start to the last of the block that its last move is into
    const int c0 = (int)(chunk * kMoveChunk), c1 = min(c0 + kMoveChunk, head.moves);
    const int prev = c0 > 0 ? moves[c0 - 1].x / kBlock8 : -1;
    const int last = moves[c1 - 1].x / kBlock8;
    if (prev == last) continue;  // all of them another chunk's
    // a block has 64 rows at most, and the chunk begins within one and ends within one
    for (int i = c0; i < head.moves;) {  // lanes: moves i .. i + 63
      int2 m = make_int2(-1, -1);
      if (i + lane < head.moves) m = moves[i + lane];
      const int b = m.x < 0 ? -1 : m.x / kBlock8;
      // of these, those into the chunk's blocks whose last move is among them too
      // (the block of the 64th may go on: it is taken up again from its first move)
      const int b63 = __builtin_amdgcn_readlane(b, kWave - 1);
      const int b0 = __builtin_amdgcn_readfirstlane(b);
      const bool whole = b63 < 0 || b63 != b || i + kWave >= head.moves || b63 == b0;
      const bool mine = b > prev && b <= last && b >= 0 && whole;
      const uint64_t mask = ballot(mine);
      const uint64_t passed = ballot(b >= 0 && (b <= prev || mine));  // these and what is before them
      const int step = __popcll(passed);
      if (mask == 0ull) {
        if (step == 0) break;
        i += step;
        continue;
      }
      const int i0 = __builtin_ctzll(mask), count = __popcll(mask);  // consecutive lanes
      // scales as they were: of the blocks moved into, and of those moved out of
      float kd = 1.f, vd = 1.f, ks = 1.f, vs = 1.f;
      if (mine) {
        kd = c.k_scales[scales + b];
        vd = c.v_scales[scales + b];
        const int f = m.y / kBlock8;
        ks = f == edge ? head.k_scale : c.k_scales[scales + f];
        vs = f == edge ? head.v_scale : c.v_scales[scales + f];
      }
      // what the rows need, and whether a block's scale is less
      int ek = kLeast8, ev = kLeast8;
      for (int j0 = 0; j0 < count; j0 += RP) {
        const int j = i0 + min(j0 + sub, count - 1);
        const int from = __shfl(m.y, j, kWave);
        uint32_t kt = top_of16(reinterpret_cast<const u32x4_t*>(c.k_codes + (base + from) * D)[piece]);
        uint32_t vt = top_of16(reinterpret_cast<const u32x4_t*>(c.v_codes + (base + from) * D)[piece]);
#pragma unroll
        for (int off = PR / 2; off > 0; off >>= 1) {
          kt = max(kt, (uint32_t)__shfl_xor((int)kt, off, kWave));
          vt = max(vt, (uint32_t)__shfl_xor((int)vt, off, kWave));
        }
        // to the lane of the move: its row is the (lane - i0 - j0)-th of these
        const int back = (lane - i0 - j0) * PR;
        const uint32_t kb = (uint32_t)__shfl((int)kt, back & 63, kWave);
        const uint32_t vb = (uint32_t)__shfl((int)vt, back & 63, kWave);
        if (back >= 0 && back < kWave && mine) {
          ek = need_of_code(kb, exponent_of(ks));
          ev = need_of_code(vb, exponent_of(vs));
        }
      }
      const bool grows = mine && (ek > exponent_of(kd) || ev > exponent_of(vd));
      for (uint64_t left = ballot(grows); left != 0ull;) {  // blocks that grow: rare
        const int lead = __builtin_ctzll(left);
        const int gbk = __builtin_amdgcn_readlane(b, lead);
        const bool here = mine && b == gbk;
        left &= ~ballot(here);
        int nk = here ? ek : kLeast8, nv = here ? ev : kLeast8;
        uint64_t taken = here ? 1ull << (m.x % kBlock8) : 0ull;  // rows that are replaced
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
          nk = max(nk, __shfl_xor(nk, off, kWave));
          nv = max(nv, __shfl_xor(nv, off, kWave));
          taken |= (uint64_t)__shfl_xor((unsigned long long)taken, off, kWave);
        }
        const float k_old = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(kd), lead));
        const float v_old = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(vd), lead));
        const int ok = uniform(exponent_of(k_old)), ov = uniform(exponent_of(v_old));
        nk = uniform(min(max(nk, ok), kMost8));
        nv = uniform(min(max(nv, ov), kMost8));
        const float kn = nk > ok ? pow2_of(nk) : k_old, vn = nv > ov ? pow2_of(nv) : v_old;
        for (int j0 = 0; j0 < kBlock8; j0 += RP) {  // the block's other tokens
          const int j = j0 + sub;
          if (gbk * kBlock8 + j >= head.keep || (taken >> j & 1ull)) continue;
          const size_t r = base + (size_t)gbk * kBlock8 + j;
          if (nk > ok) {
            u32x4_t* p = reinterpret_cast<u32x4_t*>(c.k_codes + r * D) + piece;
            *p = regrid16(*p, k_old, kn);
          }
          if (nv > ov) {
            u32x4_t* p = reinterpret_cast<u32x4_t*>(c.v_codes + r * D) + piece;
            *p = regrid16(*p, v_old, vn);
          }
        }
        if (lane == lead) {
          c.k_scales[scales + gbk] = kn;
          c.v_scales[scales + gbk] = vn;
        }
        if (here) {
          kd = kn;
          vd = vn;
        }
      }
      for (int j0 = 0; j0 < count; j0 += RP) {
        const int j = i0 + min(j0 + sub, count - 1);
        const int from = __shfl(m.y, j, kWave), to = __shfl(m.x, j, kWave);
        const float fk = __shfl(ks, j, kWave), fv = __shfl(vs, j, kWave);
        const float tk = __shfl(kd, j, kWave), tv = __shfl(vd, j, kWave);
        if (j0 + sub >= count) continue;
        const u32x4_t kw = reinterpret_cast<const u32x4_t*>(c.k_codes + (base + from) * D)[piece];
        const u32x4_t vw = reinterpret_cast<const u32x4_t*>(c.v_codes + (base + from) * D)[piece];
        reinterpret_cast<u32x4_t*>(c.k_codes + (base + to) * D)[piece] = regrid16(kw, fk, tk);
        reinterpret_cast<u32x4_t*>(c.v_codes + (base + to) * D)[piece] = regrid16(vw, fv, tv);
      }
      if (mine) {
        c.weights[base + m.x] = c.weights[base + m.y];
        c.positions[base + m.x] = c.positions[base + m.y];
      }
      i += step;
    }
  }
}

int64_t move_workgroups(const Evict8Args& a) {
  return ((int64_t)a.c.L * a.c.H * a.c.S * a.workers + kMoveThreads / kWave - 1) / (kMoveThreads / kWave);
}

}  // namespace

// Waves that move rows: as many as the chip holds, but no more than there can be
// chunks of moves.
void plan_evict8(Evict8Args& a, const int32_t* cu_rows_host) {
  a.longest = 0;
  for (int s = 0; s < a.c.S; ++s) a.longest = std::max(a.longest, cu_rows_host[s + 1] - cu_rows_host[s]);
  const int64_t heads = (int64_t)a.c.L * a.c.H * a.c.S;
  a.workers = (int)std::max<int64_t>(
      1, std::min<int64_t>((8192 + heads - 1) / heads, (a.longest / 2 + kMoveChunk - 1) / kMoveChunk));
}

bool evict8_fits(const Evict8Args& a) {
  return grid_fits((int64_t)a.c.L * a.c.H * a.c.S, 16 * kWave) &&
         grid_fits(move_workgroups(a), kMoveThreads);
}

hipError_t launch_evict8(const Evict8Args& a, hipStream_t st) {
  const dim3 rows((unsigned)(a.c.L * a.c.H) * (unsigned)a.c.S);
  auto run = [&](auto waves, auto nb, auto stream) {
    constexpr int W = decltype(waves)::value, NB = decltype(nb)::value;
    hipLaunchKernelGGL((evict8_kernel<W, NB, decltype(stream)::value>), rows, dim3(W * kWave), 0, st, a);
  };
  using std::integral_constant;
  const integral_constant<bool, false> once{};
  if (a.longest <= 4 * 64 * 8) run(integral_constant<int, 4>{}, integral_constant<int, 8>{}, once);
  else if (a.longest <= 4 * 64 * 40) run(integral_constant<int, 4>{}, integral_constant<int, 40>{}, once);
  else if (a.longest <= 16 * 64 * 32) run(integral_constant<int, 16>{}, integral_constant<int, 32>{}, once);
  else if (a.longest <= 16 * 64 * 80) run(integral_constant<int, 16>{}, integral_constant<int, 80>{}, once);
  else run(integral_constant<int, 16>{}, integral_constant<int, 16>{}, integral_constant<bool, true>{});
  const dim3 grid((unsigned)move_workgroups(a));
  if (a.c.d == 128)
    hipLaunchKernelGGL(move8_kernel<128>, grid, dim3(kMoveThreads), 0, st, a);
  else
    hipLaunchKernelGGL(move8_kernel<64>, grid, dim3(kMoveThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace stepkv
