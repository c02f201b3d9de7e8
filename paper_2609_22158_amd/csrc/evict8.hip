// Eviction from the 8-bit cache by gathered weight (include/stepkv_cache8.h):
// of the n tokens of a (layer, KV head, sequence) the `keep` best stay, and those
// of them in rows `keep` and above move into the rows below that become free. So
// only as many rows move as tokens leave, none is read and written by different
// waves, and nothing waits for anything: sources lie at `keep` and above,
// destinations below.
//
// evict8_kernel: one workgroup per (layer, KV head, sequence) finds the key of the
// keep-th best token by radix search over the weights' bits, and lists the moves.
// A wave holds a run of consecutive rows in registers, four a lane, and what waves
// have to tell each other is a few totals. The weights and positions, 8 bytes a
// token, are read once (of rooms past 81920 rows once a phase). Loading takes half
// its time, then LDS atomics and the chain of phases on the CU that holds a row: 28
// layers x 4 heads x 16 sequences of 700 to 8192 rows 30 us (64 MB; 14 of them
// loading), 64 rows of 67584 38 us (12; a quarter of the chip).
// move8_kernel: the rows, their weights and positions, 16 moves a wave; a wave has
// all the moves into a block, so that it can round the block's other tokens if
// its scale grows. A block partly below `keep` is one that rows leave and others
// enter: its scales as they were are kept by the selection. Rows of 128 bytes from
// all over the cache and their chain of three loads bound it: 64 x 2048 moves 25 us
// (69 MB), one in each of 1792 heads 10.
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

constexpr int kList = 256;  // keys of one bin that are ranked by comparing them all

template <int W>
struct Scratch8 {
  uint32_t hist[kBins];
  __attribute__((aligned(16))) uint32_t list[kList];
  uint32_t total[W];
  int count[3][W];   // of every wave: rows to be freed, rows that move, ties
  uint32_t found[3];  // bin, rank within it, keys in it; then key, rank, keys equal to it
  uint32_t listed;
};

// The bin of sh.hist that holds the rank-th greatest key (and clears sh.hist):
// thread t looks at bins kBins - 1 - PB t and the PB - 1 below, so that the prefix
// in thread order counts from the top.
template <int W>
__device__ __forceinline__ void find_bin(Scratch8<W>& sh, uint32_t rank) {
  constexpr int PB = kBins / (W * kWave);
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int low = kBins - PB - PB * tid;
  uint32_t n[PB], own = 0u;
  uint32_t* const h = sh.hist + low;
  __builtin_memcpy(n, h, sizeof(n));
  const uint32_t zero[PB] = {};
  __builtin_memcpy(h, zero, sizeof(n));
#pragma unroll
  for (int i = 0; i < PB; ++i) own += n[i];
  const uint32_t incl = (uint32_t)wave_scan((int)own);
  if (lane == kWave - 1) sh.total[wave] = incl;
  __syncthreads();
  uint32_t above = incl - own;
#pragma unroll
  for (int v = 0; v < W; ++v) above += v < wave ? sh.total[v] : 0u;
  if (above < rank && rank <= above + own) {
#pragma unroll
    for (int i = PB - 1; i >= 0; --i) {
      if (above < rank && rank <= above + n[i]) {
        sh.found[0] = (uint32_t)(low + i);
        sh.found[1] = rank - above;
        sh.found[2] = n[i];
        sh.listed = 0u;
      }
      above += n[i];
    }
  }
  __syncthreads();
}

// W waves, NG groups of 4 keys a lane: a group is 256 consecutive rows of a wave's,
// four a lane (STREAM: read again in every phase, NG groups at a time).
template <int W, int NG, bool STREAM>
__global__ __launch_bounds__(W * kWave) __attribute__((amdgpu_waves_per_eu(4)))
void evict8_kernel(Evict8Args a) {
  constexpr int kGroup = 4 * kWave;
  __shared__ __attribute__((aligned(16))) Scratch8<W> sh;
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
  const size_t edge = (size_t)lh * c.nblk + first_block(row0, s) + keep / kBlock8;
  const float k_edge = read_const(c.k_scales, edge), v_edge = read_const(c.v_scales, edge);
  const char* __restrict__ w = reinterpret_cast<const char*>(c.weights + (size_t)lh * c.rows + row0);
  const char* __restrict__ pos = reinterpret_cast<const char*>(c.positions + (size_t)lh * c.rows + row0);
  // Positions that may go: first .. first + width - 1, where position - first, taken
  // as unsigned, is below width (a position below `first` wraps to 2^31 and above).
  const int64_t recent = (int64_t)read_const(c.seen, s) - a.recent;
  const uint32_t width = (uint32_t)max(recent - a.first, (int64_t)0);
  const bool some_stay = a.first > 0 || a.recent > 0;
  // this wave's rows: ng groups from row j0
  const int ng = (n + W * kGroup - 1) / (W * kGroup);
  const int j0 = wave * ng * kGroup;
  uint32_t keys[4 * NG];
  // the keys of a group, whose first row of this lane is j; 0 for rows past the sequence
  auto load = [&](int j, uint32_t* k) __attribute__((always_inline)) {
    float x[4];
    int p[4] = {};
    if (j - 4 * lane + kGroup <= n) {  // uniform; 32-bit byte offsets: there are less than 2^30 rows
      __builtin_memcpy(x, w + 4u * (uint32_t)j, 16);
      if (some_stay) __builtin_memcpy(p, pos + 4u * (uint32_t)j, 16);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t at = 4u * (uint32_t)min(j + e, n - 1);
        x[e] = *reinterpret_cast<const float*>(w + at);
        if (some_stay) p[e] = *reinterpret_cast<const int*>(pos + at);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      k[e] = some_stay && (uint32_t)(p[e] - a.first) >= width ? kStays : order_key(x[e]);
      if (j + e >= n) k[e] = 0u;
    }
  };
  // f(first row of the group, its keys) over this wave's groups, in the rows' order
  auto each = [&](auto&& f) __attribute__((always_inline)) {
    if constexpr (STREAM) {
      for (int g = 0; g < ng; g += NG) {
#pragma unroll
        for (int i = 0; i < NG; ++i)
          if (g + i < ng) load(j0 + (g + i) * kGroup + 4 * lane, keys + 4 * i);
#pragma unroll
        for (int i = 0; i < NG; ++i)
          if (g + i < ng) f(j0 + (g + i) * kGroup, keys + 4 * i);
      }
    } else {
      // compares made anew in every phase, not masks held across them
#pragma unroll
      for (int j = 0; j < 4 * NG; ++j) asm volatile("" : "+v"(keys[j]));
#pragma unroll
      for (int g = 0; g < NG; ++g)
        if (g < ng) f(j0 + g * kGroup, keys + 4 * g);  // uniform
    }
  };
  if constexpr (!STREAM) {
#pragma unroll
    for (int g = 0; g < NG; ++g)
      if (g < ng) load(j0 + g * kGroup + 4 * lane, keys + 4 * g);
  }
  // Tokens that stay in any case, and the least and greatest key of the others.
  uint32_t least1 = 0xFFFFFFFFu, most1 = 0u;  // least - 1, and most + 1
  int always = 0;
  each([&](int, const uint32_t* k) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // 0 - 1 and kStays + 1 wrap out of the way
      least1 = min(least1, k[e] - 1u);
      most1 = max(most1, k[e] + 1u);
      always += k[e] == kStays;
    }
  });
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    least1 = min(least1, (uint32_t)__shfl_xor((int)least1, off, kWave));
    most1 = max(most1, (uint32_t)__shfl_xor((int)most1, off, kWave));
  }
  always = wave_total(wave_scan(always));
  if (lane == 0) {
    sh.count[0][wave] = (int)least1;
    sh.count[1][wave] = (int)most1;
    sh.count[2][wave] = always;
  }
  for (int i = tid; i < kBins; i += W * kWave) sh.hist[i] = 0u;
  __syncthreads();
  always = 0;
#pragma unroll
  for (int v = 0; v < W; ++v) {
    least1 = min(least1, (uint32_t)sh.count[0][v]);
    most1 = max(most1, (uint32_t)sh.count[1][v]);
    always += sh.count[2][v];
  }
  // The key tau of the keep-th greatest, and how many of those equal to it stay: keys
  // lo .. lo + span in 2048 bins, then those of the bin that holds it.
  uint32_t tau, rank, ties;
  if (always >= keep) {
    tau = kStays;
    rank = (uint32_t)keep;
    ties = (uint32_t)always;
  } else {
    uint32_t lo = least1 + 1u, span = most1 - 1u - lo;
    tau = lo;
    rank = (uint32_t)(keep - always);
    ties = (uint32_t)(n - always);
    while (span > 0u) {
      const int shift = max(32 - kDigit - __builtin_clz(span), 0);
      each([&](int, const uint32_t* k) __attribute__((always_inline)) {
        uint32_t d[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) d[e] = k[e] - lo;
        // Many lanes of one bin (equal weights) are added as one: atomics on one
        // word run one after another.
        const uint64_t act = ballot(d[0] <= span);
        bool clustered = false;
        if (act != 0ull) {
          const uint32_t lead = (uint32_t)__builtin_amdgcn_readlane((int)d[0], __builtin_ctzll(act));
          clustered = __popcll(ballot(d[0] >> shift == lead >> shift)) >= 16;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          bool add = d[e] <= span;
          const uint32_t bin = d[e] >> shift;
          if (clustered) {  // uniform
            const uint64_t on = ballot(add);
            if (on == 0ull) continue;
            const int lead = __builtin_ctzll(on);
            const uint64_t same = ballot(add && bin == (uint32_t)__builtin_amdgcn_readlane((int)bin, lead));
            if (lane == lead) atomicAdd(&sh.hist[bin], (uint32_t)__popcll(same));
            add = add && !(same >> lane & 1ull);
          }
          if (add) atomicAdd(&sh.hist[bin], 1u);
        }
      });
      __syncthreads();
      find_bin<W>(sh, rank);
      lo += (uint32_t)uniform((int)sh.found[0]) << shift;
      span = (1u << shift) - 1u;
      tau = lo;
      rank = (uint32_t)uniform((int)sh.found[1]);
      ties = (uint32_t)uniform((int)sh.found[2]);
      if (rank == ties) break;  // every key of the bin stays
      if (span > 0u && ties <= kList) {  // its keys, in any order, compared with each other
        each([&](int, const uint32_t* k) __attribute__((always_inline)) {
          uint32_t d[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) d[e] = k[e] - lo;
          if (min(min(d[0], d[1]), min(d[2], d[3])) <= span) {  // few lanes hold one
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (d[e] <= span) sh.list[atomicAdd(&sh.listed, 1u)] = k[e];
          }
        });
        __syncthreads();
        const int m = (int)ties;
        if (tid < m) {
          const uint32_t mine = sh.list[tid];
          uint32_t gt = 0u, ge = 0u;
          for (int i = 0; i < m; ++i) {
            const uint32_t o = sh.list[i];
            gt += o > mine;
            ge += o >= mine;
          }
          if (gt < rank && rank <= ge) {  // equal keys write the same
            sh.found[0] = mine;
            sh.found[1] = rank - gt;
            sh.found[2] = ge - gt;
          }
        }
        __syncthreads();
        tau = (uint32_t)uniform((int)sh.found[0]);
        rank = (uint32_t)uniform((int)sh.found[1]);
        ties = (uint32_t)uniform((int)sh.found[2]);
        break;
      }
    }
  }
  // keys above t_sure stay; of those equal to tau the first `need`, or (need 0) all
  const uint32_t t_sure = rank == ties ? tau - 1u : tau;
  const uint32_t need = rank == ties ? 0u : rank;
  uint32_t tie0 = 0u;  // ties in the rows before this wave's
  __syncthreads();     // sh.count is read
  if (need > 0u) {
    int here = 0;
    each([&](int, const uint32_t* k) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) here += __popcll(ballot(k[e] == tau));
    });
    if (lane == 0) sh.count[2][wave] = here;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < W; ++v) tie0 += v < wave ? (uint32_t)sh.count[2][v] : 0u;
  }
  // f(first row of the group, which of this lane's four stay) over this wave's rows
  auto stays_of = [&](auto&& f) __attribute__((always_inline)) {
    uint32_t before = tie0;
    each([&](int j, const uint32_t* k) __attribute__((always_inline)) {
      bool stay[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) stay[e] = k[e] > t_sure;
      if (need > 0u) {  // uniform
        uint64_t eq[4];
        uint32_t mine = before;  // ties before this lane's
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          eq[e] = ballot(k[e] == tau);
          mine += (uint32_t)lanes_below(eq[e]);
          before += (uint32_t)__popcll(eq[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool tie = k[e] == tau;
          stay[e] = stay[e] || (tie && mine < need);
          mine += tie ? 1u : 0u;
        }
      }
      f(j, stay);
    });
  };
  int frees = 0, goes = 0;
  stays_of([&](int j, const bool* stay) __attribute__((always_inline)) {
    int n_stay = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) n_stay += __popcll(ballot(stay[e]));
    int df = j + kGroup <= keep ? kGroup - n_stay : 0, dg = j >= keep ? n_stay : 0;
    if (j < keep && j + kGroup > keep) {  // uniform: both
      df = dg = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool low = j + 4 * lane + e < keep;
        df += __popcll(ballot(low && !stay[e]));
        dg += __popcll(ballot(!low && stay[e]));
      }
    }
    frees += df;
    goes += dg;
  });
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
  // The moves: the i-th row to be freed and the i-th token that moves. Rows of one
  // group below `keep` (tokens that leave are listed) or not (those that stay are).
  int2* const moves = a.moves + (size_t)lh * (c.rows / 2) + row0 / 2;
  char* const list = reinterpret_cast<char*>(moves);
  auto emit = [&](int j, const bool* on, int& base, uint32_t half) __attribute__((always_inline)) {
    int mine = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) mine += on[e];
    if (ballot(mine > 0) == 0ull) return;
    const int incl = wave_scan(mine);
    // 32-bit byte offsets: there are less than 2^29 moves
    uint32_t at = 8u * (uint32_t)(base + incl - mine) + half;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (on[e]) {
        *reinterpret_cast<int*>(list + at) = j + 4 * lane + e;
        at += 8u;
      }
    }
    base += wave_total(incl);
  };
  if (frees + goes > 0)  // uniform over the wave
    stays_of([&](int j, const bool* stay) __attribute__((always_inline)) {
      bool on[4];
      if (j < keep) {  // uniform
#pragma unroll
        for (int e = 0; e < 4; ++e) on[e] = j + 4 * lane + e < keep && !stay[e];
        emit(j, on, fb, 0u);
      }
      if (j + kGroup > keep) {
#pragma unroll
        for (int e = 0; e < 4; ++e) on[e] = j + 4 * lane + e >= keep && stay[e];
        emit(j, on, gb, 4u);
      }
    });
  if (tid == 0) *head = Evict8Head{all, keep, k_edge, v_edge};
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
  constexpr int RP = kWave / PR;  // rows of a load
  constexpr int kRows = 16 / RP > 0 ? 16 / RP : 1;  // loads in flight, of each tensor
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
    const int before = moves[max(c0 - 1, 0)].x / kBlock8, last = moves[c1 - 1].x / kBlock8;
    const int prev = c0 > 0 ? before : -1;
    for (int i = c0;;) {  // lanes: moves i .. i + 63
      int2 m = make_int2(-1, -1);
      if (i + lane < head.moves) m = moves[i + lane];
      if (prev == last) break;  // all of them another chunk's
      const int b = m.x < 0 ? -1 : m.x / kBlock8;
      // of these, the moves into the chunk's blocks, but for a block that goes on after
      // the 64th (it is taken up again from its first move; no block has more than 64)
      const int b0 = uniform(b), b63 = __builtin_amdgcn_readlane(b, kWave - 1);
      const bool mine = b > prev && b <= last && (b != b63 || b63 == b0 || i + kWave >= head.moves);
      const uint64_t mask = ballot(mine);
      const int step = __popcll(ballot(b >= 0 && (b <= prev || mine)));  // the first `step` lanes are done with
      if (mask != 0ull) {
        const int i0 = __builtin_ctzll(mask), count = __popcll(mask);  // consecutive lanes
        u32x4_t kw[kRows], vw[kRows];  // 16 bytes of kRows rows, of the moves from i0 + j0 on
        auto load_rows = [&](int j0) __attribute__((always_inline)) {
#pragma unroll
          for (int u = 0; u < kRows; ++u) {
            const int from = __shfl(m.y, i0 + min(j0 + u * RP + sub, count - 1), kWave);
            kw[u] = reinterpret_cast<const u32x4_t*>(c.k_codes + (base + from) * D)[piece];
            vw[u] = reinterpret_cast<const u32x4_t*>(c.v_codes + (base + from) * D)[piece];
          }
        };
        load_rows(0);
        // what moves along, and scales as they were: of the blocks moved into, and of
        // those moved out of
        float kd = 1.f, vd = 1.f, ks = 1.f, vs = 1.f, weight = 0.f;
        int position = 0;
        if (mine) {
          const int f = m.y / kBlock8;
          kd = c.k_scales[scales + b];
          vd = c.v_scales[scales + b];
          ks = c.k_scales[scales + f];
          vs = c.v_scales[scales + f];
          weight = c.weights[base + m.y];
          position = c.positions[base + m.y];
          if (f == edge) ks = head.k_scale, vs = head.v_scale;
        }
        // what the rows need, and whether a block's scale is less
        int ek = kLeast8, ev = kLeast8;
        auto look = [&](int j0) __attribute__((always_inline)) {
#pragma unroll
          for (int u = 0; u < kRows; ++u) {
            uint32_t kt = top_of16(kw[u]), vt = top_of16(vw[u]);
#pragma unroll
            for (int off = PR / 2; off > 0; off >>= 1) {
              kt = max(kt, (uint32_t)__shfl_xor((int)kt, off, kWave));
              vt = max(vt, (uint32_t)__shfl_xor((int)vt, off, kWave));
            }
            // to the lane of the move: its row is the (lane - i0 - j0 - u RP)-th of these
            const int back = (lane - i0 - j0 - u * RP) * PR;
            const uint32_t kb = (uint32_t)__shfl((int)kt, back & 63, kWave);
            const uint32_t vb = (uint32_t)__shfl((int)vt, back & 63, kWave);
            if (back >= 0 && back < kWave && mine) {
              ek = need_of_code(kb, exponent_of(ks));
              ev = need_of_code(vb, exponent_of(vs));
            }
          }
        };
        look(0);
        for (int j0 = kRows * RP; j0 < count; j0 += kRows * RP) {
          load_rows(j0);
          look(j0);
        }
        const bool grows = mine && (ek > exponent_of(kd) || ev > exponent_of(vd));
        for (uint64_t left = ballot(grows); left != 0ull;) {  // blocks that grow: rare
          const int lead = __builtin_ctzll(left);
          const int at_b = __builtin_amdgcn_readlane(b, lead);
          const bool here = mine && b == at_b;
          left &= ~ballot(here);
          int nk = here ? ek : kLeast8, nv = here ? ev : kLeast8;
          uint64_t taken = here ? 1ull << (m.x % kBlock8) : 0ull;  // rows that are replaced
#pragma unroll
          for (int off = 32; off > 0; off >>= 1) {
            nk = max(nk, __shfl_xor(nk, off, kWave));
            nv = max(nv, __shfl_xor(nv, off, kWave));
            taken |= (uint64_t)__shfl_xor((unsigned long long)taken, off, kWave);
          }
          const float k_old = __shfl(kd, lead, kWave), v_old = __shfl(vd, lead, kWave);
          const int ok = uniform(exponent_of(k_old)), ov = uniform(exponent_of(v_old));
          nk = uniform(min(max(nk, ok), kMost8));
          nv = uniform(min(max(nv, ov), kMost8));
          const float kn = nk > ok ? pow2_of(nk) : k_old, vn = nv > ov ? pow2_of(nv) : v_old;
#pragma nounroll
          for (int j0 = 0; j0 < kBlock8; j0 += RP) {  // the block's other tokens
            const int j = j0 + sub;
            if (at_b * kBlock8 + j >= head.keep || (taken >> j & 1ull)) continue;
            const size_t r = base + (size_t)at_b * kBlock8 + j;
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
            c.k_scales[scales + at_b] = kn;
            c.v_scales[scales + at_b] = vn;
          }
          if (here) {
            kd = kn;
            vd = vn;
          }
        }
        auto store_rows = [&](int j0) __attribute__((always_inline)) {
#pragma unroll
          for (int u = 0; u < kRows; ++u) {
            const int at_j = j0 + u * RP + sub, j = i0 + min(at_j, count - 1);
            const int to = __shfl(m.x, j, kWave);
            const float fk = __shfl(ks, j, kWave), fv = __shfl(vs, j, kWave);
            const float tk = __shfl(kd, j, kWave), tv = __shfl(vd, j, kWave);
            if (at_j < count) {
              reinterpret_cast<u32x4_t*>(c.k_codes + (base + to) * D)[piece] = regrid16(kw[u], fk, tk);
              reinterpret_cast<u32x4_t*>(c.v_codes + (base + to) * D)[piece] = regrid16(vw[u], fv, tv);
            }
          }
        };
        if (count <= kRows * RP) {  // the rows are still there
          store_rows(0);
        } else {
          for (int j0 = 0; j0 < count; j0 += kRows * RP) {
            load_rows(j0);
            store_rows(j0);
          }
        }
        if (mine) {
          c.weights[base + m.x] = weight;
          c.positions[base + m.x] = position;
        }
      }
      if (step == 0 || b63 < 0 || b63 > last) break;  // the chunk's last move is among these
      i += step;
      if (i >= head.moves) break;
    }
  }
}

int64_t move_workgroups(const Evict8Args& a) {
  return ((int64_t)a.c.L * a.c.H * a.c.S * a.workers + kMoveThreads / kWave - 1) / (kMoveThreads / kWave);
}

}  // namespace

// Waves that move rows: as many as the chip holds, but no more than there can be
// chunks of moves (with keeps on the device, half as many: most find none).
void plan_evict8(Evict8Args& a, const int32_t* cu_rows_host) {
  a.longest = 0;
  for (int s = 0; s < a.c.S; ++s) a.longest = std::max(a.longest, cu_rows_host[s + 1] - cu_rows_host[s]);
  const int64_t heads = (int64_t)a.c.L * a.c.H * a.c.S, want = a.keeps ? 4096 : 8192;
  int64_t most = a.longest / 2;
  if (!a.keeps) most = std::min<int64_t>(most, std::max(a.longest - a.keep, 1));
  a.workers = (int)std::max<int64_t>(
      1, std::min<int64_t>((want + heads - 1) / heads, (most + kMoveChunk - 1) / kMoveChunk));
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
  // Waves and groups of 256 rows for the longest room: few keys a lane leave room for
  // more workgroups (28 layers x 4 heads x 16 sequences of 700 to 8192 rows: 4 waves
  // of 10 groups 32 us, 8 of 5 30).
  if (a.longest <= 4 * 256 * 2) run(integral_constant<int, 4>{}, integral_constant<int, 2>{}, once);
  else if (a.longest <= 8 * 256 * 5) run(integral_constant<int, 8>{}, integral_constant<int, 5>{}, once);
  else if (a.longest <= 16 * 256 * 8) run(integral_constant<int, 16>{}, integral_constant<int, 8>{}, once);
  else if (a.longest <= 16 * 256 * 20) run(integral_constant<int, 16>{}, integral_constant<int, 20>{}, once);
  else run(integral_constant<int, 16>{}, integral_constant<int, 4>{}, integral_constant<bool, true>{});
  const dim3 grid((unsigned)move_workgroups(a));
  if (a.c.d == 128)
    hipLaunchKernelGGL(move8_kernel<128>, grid, dim3(kMoveThreads), 0, st, a);
  else
    hipLaunchKernelGGL(move8_kernel<64>, grid, dim3(kMoveThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace stepkv
