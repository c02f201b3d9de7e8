// One decode step's attention over the 8-bit cache: out = softmax(scale *
// q . K^T) V per (layer, sequence, query head), and the weight that every token
// has in it.
//
// The cache's 2 d bytes a token and KV head bound it. One conversion instruction
// gives two exact bf16 values, the block's scale included, and both products run
// on MFMA.
//
// attend8_kernel: one workgroup per (layer, KV head, 16 query heads, split of
// a sequence's tokens), its waves on consecutive runs of 32-token tiles, each
// with its own online softmax. Per tile and wave:
//  - K: lane (g, r) = (l / 16, l % 16) holds 16 channels of row r at a time (those
//    from 64 j + 16 g, j < d / 64) as the A operand of v_mfma_f32_16x16x32_bf16, 8
//    channels a step; the query heads are the B operand in the same channel
//    order. Lane (g, r) then holds head r's logits of rows 4 g .. 4 g + 3 of each
//    16-row half.
//  - softmax per head in that layout, in the log2 domain, with a reference
//    that moves only when a logit exceeds it by kSlack.
//  - V: the codes go into the wave's LDS tile as they are; ds_read_b64_tr_b8 gives
//    a column's 8 rows per lane, in the order in which the lane holds P, and the
//    conversion makes them the B operand. P is the A operand, as three bf16 parts
//    that are it exactly (in one operand for narrow groups); the same parts times
//    ones give the softmax's sum.
// combine8_kernel merges the splits. To gather weights, which need the row's maximum
// and sum, the logits are kept (4 bytes a query head and token), and the same launch,
// or the workgroup that has the whole sequence, turns them into weights; or, for wide
// groups, that launch computes them from the keys again.
//
// 8 layers x 8 heads x 131071 tokens of d 128 (4 query heads each): 327 to 335 us, 6.4 to
// 6.6 TB/s, 489 with the weights; 28 layers x 4 heads x 16 sequences of 700 to 8192 tokens
// (7 each): 350 us, 5.8 TB/s, 522 with the weights. One layer of these a call, the layers
// in turn: 56 us (74 with the weights) and 30 (35). What the weights cost is memory:
// stores among loads slow these down by far more than their bytes (134 MB written
// beside 2.1 GB read: 80 us in a kernel that does only that).
#include "cache8_device.h"

#include <math.h>

#include <algorithm>
#include <type_traits>

namespace stepkv {
namespace {

typedef int i32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2_t lds_i32x2;

constexpr int kTile = 32;  // tokens a wave computes at a time
constexpr int kWaves = 4;  // waves of a workgroup
constexpr int kWavesFew = 8;  // where a whole sequence is one, and there are few
constexpr int kMostLds = 32768;  // bytes of logits kept in LDS
constexpr int kMergeThreads = 256;  // of a merge of many rows
constexpr int kMergeOne = 512;      // and of a merge of one query head
constexpr int kMostBlocks = 16;     // that a wave sweeps
constexpr int kMostLogits = 9;      // heads of a group whose logits are kept for the merge
constexpr float kSlack = 16.f;
constexpr float kLog2e = 1.44269504088896341f;

// Rows of a split, from the tokens there are when the kernel runs: as many as
// give at most a.splits splits in all, sum_s ceil(n_s / rows) <= total / rows +
// nonempty sequences. A multiple of a tile for each of the waves.
__device__ __forceinline__ int rows_per_split(const Attend8Args& a) {
  const int lane = threadIdx.x & 63;
  int64_t total = 0;
  int some = 0, most = 0;  // most: splits of min_rows
  for (int s0 = 0; s0 < a.c.S; s0 += kWave) {
    const int n = s0 + lane < a.c.S ? held_tokens(a.c, s0 + lane) : 0;
    total += (uint32_t)wave_total(wave_scan(n));  // the rooms add up to less than 2^31
    some += __popcll(ballot(n > 0));
    most += wave_total(wave_scan((n + a.min_rows - 1) / a.min_rows));
  }
  if (most <= a.splits) return a.min_rows;
  const int slots = max(a.splits - some, 1);
  const int64_t rows = (total + slots - 1) / slots;
  return (int)((max(rows, (int64_t)a.min_rows) + a.min_rows - 1) / a.min_rows * a.min_rows);
}

// The rank-th split in order of length, of at most 64 sequences: whole splits, then
// the sequences' last ones, the longest first. Its sequence, that one's first split,
// and (in rank) its number in the order of the sequences; false past the last.
__device__ __forceinline__ bool longest_first(const Attend8Args& a, int split, int& rank, int& s,
                                              int& first) {
  const int lane = threadIdx.x & 63;
  const int n = lane < a.c.S ? held_tokens(a.c, lane) : 0;
  const int whole = n / split, rest = n - whole * split;
  const int wholes = wave_scan(whole), all = wave_total(wholes);
  const int incl = wave_scan(whole + (rest > 0));
  int at;  // the split's number in its sequence
  if (rank < all) {
    s = __builtin_ctzll(ballot(wholes > rank));
    at = rank - __builtin_amdgcn_readlane(wholes - whole, s);
  } else {
    int before = 0;  // sequences whose last split is longer, or as long and of a lower index
    for (int j = 0; j < a.c.S; ++j) {
      const int other = __builtin_amdgcn_readlane(rest, j);
      before += other > rest || (other == rest && j < lane);
    }
    const uint64_t found = ballot(rest > 0 && before == rank - all);
    if (found == 0ull) return false;
    s = __builtin_ctzll(found);
    at = __builtin_amdgcn_readlane(whole, s);
  }
  first = __builtin_amdgcn_readlane(incl - whole - (rest > 0), s);
  rank = first + at;
  return true;
}

// Byte offset of piece j (16 channels) of row r in a wave's V tile, row-major:
// with the XORs the writes (whole rows) and the transposing reads (16 bytes of
// each of the 16 rows that two groups of 16 lanes take) touch every bank once.
template <int D>
__device__ __forceinline__ int v_at(int r, int j) {
  const int b12 = (r >> 1) & 3, b4 = (r >> 4) & 1;
  return D == 128 ? r * 128 + 16 * (j ^ (b12 | b4 << 2))
                  : r * 64 + 16 * (j ^ (((r >> 2) & 1) | b4 << 1));
}

// The reference of a wave that saw tokens, whose logits are all -inf: below every
// logit, but not that of a wave without tokens.
constexpr float kNoWeight = -3.40282347e38f;

// The result of a query head from its sums (row: (layer, sequence, query head)).
// Without a token zeros; where every logit is -inf (an overflow) the softmax of
// such logits, 0 / 0.
__device__ __forceinline__ void finish(const Attend8Args& a, size_t row, int ch, int D, float M,
                                       float Z, float O) {
  a.out[row * D + ch] = M == -INFINITY && Z == 0.f ? 0.f : O / Z;
  if (a.lse && ch == 0) a.lse[row] = Z == 0.f ? -INFINITY : (M + log2f(Z)) * 0.693147180559945309f;
}

// The logits are kept by tiles of 32 tokens, [L*H*tiles][rows / 32 + S][min(G, 16)][32]:
// a wave writes a tile in one piece. Offset of those of a unit and a sequence.
__device__ __forceinline__ size_t logits_at(const Attend8Args& a, int unit, int seq_row, int s) {
  const size_t tiles = a.c.rows / kTile + a.c.S;
  return ((size_t)unit * tiles + seq_row / kTile + s) * min(a.G, 16) * kTile;
}
// Of token j, head 0, from there; those of the next heads follow at kTile.
__device__ __forceinline__ size_t token_at(const Attend8Args& a, int j) {
  return (size_t)(j / kTile) * min(a.G, 16) * kTile + j % kTile;
}

// The weight of a token whose unscaled logit is y; NaN where M or 1 / Z says so.
__device__ __forceinline__ float weight_of(float y, float cl2, float2 norm) {
  return fast_exp2(fmaf(y, cl2, -norm.x)) * norm.y;
}

// What weights are gathered from: the logits, kept in memory or LDS, or the keys again.
enum { kNone, kMemory, kLds, kSweep };

// 16 bytes of keys. Lanes of one load take 64 bytes of a row: all of it (d 64), or half
// a line, whose other half should still be in the cache when the next load asks for
// it: 8 layers x 8 heads x 131071 tokens 346 us non-temporal, 334 so (timed in turn, as
// the pairs at plan_attend8).
template <int D>
__device__ __forceinline__ u32x4_t load_k(const uint8_t* p) {
  const u32x4_t* const x = reinterpret_cast<const u32x4_t*>(p);
  return D == 64 ? __builtin_nontemporal_load(x) : *x;
}

// NW waves share a split (or, with a.single, a whole sequence); C copies (1 or 3)
// of the query heads in the operands' rows.
template <int D, int NW, int GATHER, int C>
__global__ __launch_bounds__(NW * kWave) __attribute__((amdgpu_waves_per_eu(3)))
void attend8_kernel(Attend8Args a) {
  constexpr int KP = D / 64;        // 16-byte K pieces of a row that a lane loads
  constexpr int NS = D / 32;        // MFMA steps of S
  constexpr int VL = D / 32;        // 16-byte V pieces a lane loads per tile
  constexpr int VP = D / 16;        // of a row
  constexpr int VR = kTile / VL;    // rows between them
  constexpr int NB = D / 16;        // 16-column blocks of O
  constexpr int ST = D + 2;
  constexpr int TB = kTile * D;     // bytes of a V tile
  constexpr int kStateBytes = NW * 16 * ST * 4;
  __shared__ __attribute__((aligned(16)))
  uint8_t smem[NW * TB > kStateBytes ? NW * TB : kStateBytes];
  __shared__ __attribute__((aligned(16))) float fscale[NW][16];
  __shared__ float2 norm_s[16];
  const Cache8View& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int g4 = lane >> 4, c16 = lane & 15;
  if (blockIdx.x == 0 && wave == 0) report_rooms(c);
  // Workgroups are dealt to the 8 XCDs in turn; each XCD takes a contiguous
  // eighth of the splits or, in batches, of the units, and their longest splits first.
  const int xcd = (int)(blockIdx.x & 7), nth = (int)(blockIdx.x >> 3);
  int unit, gs;  // (layer, KV head, 16 query heads); its split
  if (a.by_length) {
    const int units = (int)(gridDim.x >> 3) / a.splits;  // of an XCD
    gs = uniform(nth / units);
    unit = uniform(xcd * units + (nth - gs * units));
  } else {
    const int bid = xcd * (int)(gridDim.x >> 3) + nth;
    unit = uniform(bid / a.splits);
    gs = uniform(bid - unit * a.splits);
  }
  const int tiles = (a.G + 15) / 16;
  if (unit >= c.L * c.H * tiles) return;  // the grid is padded to a multiple of 8
  const int lh = uniform(unit / tiles), hd0 = 16 * (unit - lh * tiles);  // first head of the group
  const int l = uniform(lh / c.H), h = lh - l * c.H;
  int s = gs, w0, w1;  // this wave's rows [w0, w1) of those of its sequence
  if (a.single) {
    const int share = (held_const(c, s) + NW * kTile - 1) / (NW * kTile) * kTile;
    w0 = wave * share;
    w1 = w0 + share;
  } else {
    int first;
    const int split = rows_per_split(a);
    if (a.by_length) {
      if (!longest_first(a, split, gs, s, first)) return;
    } else {
      locate_item(c.S, gs, [&](int sq) { return (held_tokens(c, sq) + split - 1) / split; }, s,
                  first);
      if (s < 0) return;  // past the last split: uniform over the workgroup
    }
    w0 = (gs - first) * split + wave * (split / NW);
    w1 = w0 + split / NW;
  }
  s = uniform(s);
  const int held = held_const(c, s);
  const int t0 = uniform(w0 / kTile), t1 = uniform((min(held, w1) + kTile - 1) / kTile);  // its tiles
  const int heads = min(a.G - hd0, 16);
  constexpr int kCols = 16 / C;  // columns of a copy
  const int copy = c16 / kCols, hcol = c16 % kCols;
  bf16x8_t qb[NS];
#pragma unroll
  for (int ks = 0; ks < NS; ++ks) {
    qb[ks] = bf16x8_t{};
    if (hcol < heads && copy < C)
      qb[ks] = *reinterpret_cast<const bf16x8_t*>(
          a.q + (((size_t)l * c.S + s) * a.Hq + h * a.G + hd0 + hcol) * D + 64 * (ks / 2) +
          16 * g4 + 8 * (ks % 2));
  }
  const float cl2 = a.scale * kLog2e;
  float m_ref = -INFINITY;
  f32x4_t o[NB], z = f32x4_t{};
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) o[nb] = f32x4_t{};
  const int seq_row = read_const(c.cu_rows, s);
  const size_t row0 = (size_t)lh * c.rows + seq_row;
  const size_t blk0 = (size_t)lh * c.nblk + first_block(seq_row, s);
  uint8_t* const vt = smem + wave * TB;
  const int vrow = lane / VP, vpiece = lane % VP;  // this lane's V row and piece
  // the logits of this lane's head and rows, from the sequence's first tile
  extern __shared__ __attribute__((aligned(16))) float zlds[];
  float* const zt =
      (GATHER == kLds ? zlds : GATHER == kMemory ? a.logits + logits_at(a, unit, seq_row, s) : nullptr) +
      c16 * kTile + 4 * g4;

  struct Tile {
    u32x4_t k[2][KP], v[VL];
    float ks, vs;
  };
  // Loads tile t (or, past the end, again the last one, so that the count of
  // loads in flight is the same in every round).
  auto load = [&](Tile& x, int t) __attribute__((always_inline)) {
    const int b = min(t, t1 - 1) * kTile, last = held - 1 - b;
    const uint8_t* __restrict__ kc = c.k_codes + (row0 + b) * D;
    const uint8_t* __restrict__ vc = c.v_codes + (row0 + b) * D;
    x.ks = read_const(c.k_scales, blk0 + b / kBlock8);
    x.vs = read_const(c.v_scales, blk0 + b / kBlock8);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t r = min(16 * u + c16, last);  // rows past the end: the last one again
#pragma unroll
      for (int j = 0; j < KP; ++j)
        x.k[u][j] = load_k<D>(kc + (r * D + 64 * j + 16 * g4));
    }
#pragma unroll
    for (int u = 0; u < VL; ++u) {
      const uint32_t r = min(VR * u + vrow, last);
      x.v[u] = __builtin_nontemporal_load(
          reinterpret_cast<const u32x4_t*>(vc + (r * D + 16 * vpiece)));
    }
  };
  // The first half of a tile's work, after which its registers are free: the
  // logits on the matrix cores, V's codes in LDS.
  f32x4_t acc[2];
  auto consume = [&](const Tile& x) __attribute__((always_inline)) {
    acc[0] = acc[1] = f32x4_t{};
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int ks = 0; ks < NS; ++ks)
        acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            __builtin_bit_cast(bf16x8_t, spread8(x.k[u][ks / 2][2 * (ks % 2)],
                                                 x.k[u][ks / 2][2 * (ks % 2) + 1], x.ks)),
            qb[ks], acc[u], 0, 0, 0);
#pragma unroll
    for (int u = 0; u < VL; ++u)
      *reinterpret_cast<u32x4_t*>(vt + v_at<D>(VR * u + vrow, vpiece)) = x.v[u];
  };
  auto attend = [&](int tok, float vs) __attribute__((always_inline)) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = acc[i >> 2][i & 3];
    if (tok + kTile > held) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (tok + 16 * (i >> 2) + 4 * g4 + (i & 3) >= held) y[i] = -INFINITY;
    }
    float tmax = y[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) tmax = fmaxf(tmax, y[i]);
    tmax *= cl2;  // the scale is positive
    if (__builtin_amdgcn_ballot_w64(tmax > m_ref + kSlack) != 0) {  // wave-uniform, rare
      tmax = fmaxf(tmax, xor16(tmax));
      tmax = fmaxf(tmax, xor32(tmax));
      const float m_new = tmax > m_ref + kSlack ? tmax : m_ref;
      const float f = m_ref == -INFINITY ? 0.f : fast_exp2(m_ref - m_new);
      m_ref = m_new;
      if (g4 == 0) fscale[wave][c16] = f;
      __builtin_amdgcn_wave_barrier();
      const float4 f4 = *reinterpret_cast<const float4*>(&fscale[wave][4 * g4]);
      z[0] *= f4.x;
      z[1] *= f4.y;
      z[2] *= f4.z;
      z[3] *= f4.w;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        o[nb][0] *= f4.x;
        o[nb][1] *= f4.y;
        o[nb][2] *= f4.z;
        o[nb][3] *= f4.w;
      }
    }
    // a logit of -inf has no weight, also while the reference is still -inf
    const float m = m_ref == -INFINITY ? 0.f : m_ref;
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = fast_exp2(fmaf(y[i], cl2, -m));
    const Parts<C> pp = split_parts<C>(p, copy);
    const bf16x8_t one = __builtin_bit_cast(bf16x8_t, u32x4_t{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
#pragma unroll
    for (int k = 0; k < Parts<C>::N; ++k) z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pp.x[k], one, z, 0, 0, 0);
    // column block nb: lane (g, c) gets column c of rows 4 g .. 4 g + 3 of both halves
    const int vr = c16 < 8 ? 4 * g4 + (c16 >> 1) : 16 + 4 * g4 + (c16 >> 1) - 4;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const i32x2_t w =
          __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(vt + v_at<D>(vr, nb) + 8 * (c16 & 1)));
      const bf16x8_t vb = __builtin_bit_cast(bf16x8_t, spread8((uint32_t)w[0], (uint32_t)w[1], vs));
#pragma unroll
      for (int k = 0; k < Parts<C>::N; ++k)
        o[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pp.x[k], vb, o[nb], 0, 0, 0);
    }
  };
  if (t0 < t1) {
    Tile cur;
    load(cur, t0);
    for (int t = t0; t < t1; ++t) {  // wave-uniform
      const float vs = cur.vs;
      consume(cur);
      // before the loads, whose wait then is for nothing else
      if (GATHER != kNone && c16 < heads) {  // the first copy's lanes; a tile has room for all its rows
        f32x4_t* const z4 = reinterpret_cast<f32x4_t*>(zt + (size_t)t * min(a.G, 16) * kTile);
        z4[0] = acc[0];
        z4[4] = acc[1];
      }
      load(cur, t + 1);
      attend(t * kTile, vs);
    }
  }
  __syncthreads();  // the states overwrite the V tiles of every wave
  auto state = reinterpret_cast<float(*)[16][ST]>(smem);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((4 * g4 + i) % kCols < heads && (4 * g4 + i) / kCols < C) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) state[wave][4 * g4 + i][16 * nb + c16] = o[nb][i];
      if (c16 == 0) state[wave][4 * g4 + i][D + 1] = z[i];
    }
  }
  if (g4 == 0 && c16 < heads)  // the same in every copy
    state[wave][c16][D] = t0 < t1 ? fmaxf(m_ref, kNoWeight) : -INFINITY;
  __syncthreads();
  float* const part = a.partial + ((size_t)unit * a.splits + gs) * min(a.G, 16) * ST;
  const size_t row_out = ((size_t)l * c.S + s) * a.Hq + h * a.G + hd0;
  for (int e = tid; e < heads * D; e += NW * kWave) {
    const int hd = e / D, ch = e - hd * D;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, state[w][hd][D]);
    float Z = 0.f, O = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float m = state[w][hd][D];
      const float x = m == -INFINITY ? 0.f : fast_exp2(m - M);  // a NaN sum stays NaN
      float z1 = state[w][hd][D + 1], o1 = state[w][hd][ch];
#pragma unroll
      for (int k = 1; k < C; ++k) {
        z1 += state[w][k * kCols + hd][D + 1];
        o1 += state[w][k * kCols + hd][ch];
      }
      Z = fmaf(z1, x, Z);
      O = fmaf(o1, x, O);
    }
    if (a.single) {
      finish(a, row_out + hd, ch, D, M, Z, O);
      if (GATHER != kNone && ch == 0) norm_s[hd] = make_float2(M, 1.f / Z);
      continue;
    }
    part[hd * ST + ch] = O;
    if (ch == 0) {
      part[hd * ST + D] = M;
      part[hd * ST + D + 1] = Z;
    }
  }
  if constexpr (GATHER != kNone) {
    // All heads' logits of the whole sequence are this workgroup's: their weights.
    if (!a.single) return;
    __threadfence_block();
    __syncthreads();
    const float* const base = zt - (c16 * kTile + 4 * g4);
    for (int j = tid; j < held; j += NW * kWave) {
      float w = 0.f;
      for (int g = 0; g < heads; ++g)
        w += weight_of(__hip_atomic_load(base + token_at(a, j) + g * kTile, __ATOMIC_RELAXED,
                                         __HIP_MEMORY_SCOPE_WORKGROUP), cl2, norm_s[g]);
      c.weights[row0 + j] += w;
    }
  }
}

// The splits of sequence s in the partial states of a unit: its first, and how many.
__device__ __forceinline__ void splits_of(const Attend8Args& a, int s, int& first, int& n) {
  const int lane = threadIdx.x & 63;
  const int split = rows_per_split(a);
  first = 0;
  for (int s0 = 0; s0 < s; s0 += kWave)
    first += wave_total(
        wave_scan(s0 + lane < s ? (held_tokens(a.c, s0 + lane) + split - 1) / split : 0));
  first = min(first, a.splits);
  n = min((held_const(a.c, s) + split - 1) / split, a.splits - first);
}

// What the softmax of `heads` query heads is taken over, for all threads: (M, 1 / Z)
// of head g from the states of the splits, a wave for each; (0, 0) past them.
template <int D, int THREADS>
__device__ __forceinline__ void norms_of(const Attend8Args& a, int unit, int split0, int splits, int heads,
                                         float2* norm_s) {
  constexpr int ST = D + 2;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), wide = min(a.G, 16);
  const float* __restrict__ part = a.partial + ((size_t)unit * a.splits + split0) * wide * ST;
  for (int g = wave; g < 16; g += THREADS / kWave) {
    float M = -INFINITY, Z = 0.f;
    if (g < heads)
      for (int i = lane; i < splits; i += kWave) {
        const float* __restrict__ p = part + ((size_t)i * wide + g) * ST + D;
        const float m = p[0], z = p[1], top = fmaxf(M, m);
        Z = (M == -INFINITY ? 0.f : Z * fast_exp2(M - top)) + (m == -INFINITY ? 0.f : z * fast_exp2(m - top));
        M = top;
      }
    const float top = wave_max(M);
    const float sum = wave_sum(M == -INFINITY ? 0.f : Z * fast_exp2(M - top));
    if (lane == 0) norm_s[g] = g < heads ? make_float2(top, 1.f / sum) : make_float2(0.f, 0.f);
  }
  __syncthreads();
}

// weights += the weights of a run of tokens of a (layer, KV head, sequence): the sums over
// the group's heads, in one order.
// From the logits that were kept, of at most kMostLogits heads: THREADS * 4 tokens, four a
// thread.
// SWEEP, from the keys once more: a.sweep blocks of 64 tokens a wave, the heads in the
// products' rows, so that a lane has four heads' logits of a token and four lanes meet
// for the sum.
template <int D, int THREADS, bool SWEEP>
__device__ __forceinline__ void gather(const Attend8Args& a, int at) {
  const int kRows = SWEEP ? THREADS * a.sweep : 4 * THREADS;
  __shared__ float2 norm_s[16];
  const Cache8View& c = a.c;
  const int tid = threadIdx.x;
  const int per = c.rows / kRows + c.S;  // runs that a (layer, KV head) may have
  const int lh = uniform(at / per);
  at -= lh * per;
  int s = 0, first = 0;
  locate_item(c.S, at, [&](int sq) { return (held_tokens(c, sq) + kRows - 1) / kRows; }, s, first);
  if (s < 0) return;
  s = uniform(s);
  const int j0 = (at - first) * kRows, held = held_const(c, s);
  const int seq_row = read_const(c.cu_rows, s);
  const float cl2 = a.scale * kLog2e;
  if constexpr (SWEEP) {
    int split0, splits;
    splits_of(a, s, split0, splits);
    constexpr int KP = D / 64, NS = D / 32;
    const int tiles = (a.G + 15) / 16;
    const int lane = tid & 63, wave = uniform(tid >> 6), g4 = lane >> 4, c16 = lane & 15;
    const int l = uniform(lh / c.H), h = lh - l * c.H;
    const int b0 = uniform(j0 / kBlock8 + wave * a.sweep);  // the wave's blocks
    const int b1 = uniform(min(b0 + a.sweep, (held + kBlock8 - 1) / kBlock8));
    const size_t row0 = (size_t)lh * c.rows + seq_row, blk0 = (size_t)lh * c.nblk + first_block(seq_row, s);
    __shared__ float sums_s[THREADS / kWave][kMostBlocks * kBlock8];
    float* const sums = sums_s[wave];
    struct Block {
      u32x4_t k[4][KP];
      float scale;
    };
    auto load = [&](Block& x, int b) __attribute__((always_inline)) {
      const int last = held - 1 - b * kBlock8;
      const size_t row = row0 + (size_t)b * kBlock8;
      const uint8_t* __restrict__ kc = c.k_codes + row * D;
      x.scale = read_const(c.k_scales, blk0 + b);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t r = min(16 * u + c16, last);  // rows past the end: the last one again
#pragma unroll
        for (int j = 0; j < KP; ++j)
          x.k[u][j] = load_k<D>(kc + (r * D + 64 * j + 16 * g4));
      }
    };
    for (int t = 0; t < tiles; ++t) {
      const int heads = min(a.G - 16 * t, 16);
      if (t > 0) __syncthreads();  // norm_s is read
      Block cur;
      if (b0 < b1) load(cur, b0);
      norms_of<D, THREADS>(a, lh * tiles + t, split0, splits, heads, norm_s);
      bf16x8_t qa[NS];
#pragma unroll
      for (int ks = 0; ks < NS; ++ks) {
        qa[ks] = bf16x8_t{};
        if (c16 < heads)
          qa[ks] = *reinterpret_cast<const bf16x8_t*>(
              a.q + (((size_t)l * c.S + s) * a.Hq + h * a.G + 16 * t + c16) * D + 64 * (ks / 2) +
              16 * g4 + 8 * (ks % 2));
      }
      float2 norm[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) norm[i] = norm_s[4 * g4 + i];
#pragma nounroll
      for (int b = b0; b < b1; ++b) {  // wave-uniform
        f32x4_t y[4];  // logits of token c16 of the block's 16-row pieces
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          y[u] = f32x4_t{};
#pragma unroll
          for (int ks = 0; ks < NS; ++ks)
            y[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                qa[ks], __builtin_bit_cast(bf16x8_t, spread8(cur.k[u][ks / 2][2 * (ks % 2)],
                                                             cur.k[u][ks / 2][2 * (ks % 2) + 1], cur.scale)),
                y[u], 0, 0, 0);
        }
        load(cur, min(b + 1, b1 - 1));  // its registers are free
        float w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          w[u] = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[u] += weight_of(y[u][e], cl2, norm[e]);
          w[u] += xor16(w[u]);
          w[u] += xor32(w[u]);
        }
        const float mine = g4 < 2 ? (g4 & 1 ? w[1] : w[0]) : (g4 & 1 ? w[3] : w[2]);  // lane i: token i
        float* const to = sums + (b - b0) * kBlock8 + lane;
        *to = t > 0 ? *to + mine : mine;
      }
    }
    // written at the end: stores among the loads would be waited for with them
    for (int j = b0 * kBlock8 + lane; j < min(b1 * kBlock8, held); j += kWave)
      c.weights[row0 + j] += sums[j - b0 * kBlock8];
  } else {
    const int j = j0 + 4 * tid;
    float* const to = c.weights + (size_t)lh * c.rows + seq_row + j;
    float w[4] = {}, was[4];
    f32x4_t y[kMostLogits];  // in flight while the norms are found
    if (j < held) {
      const float* __restrict__ z = a.logits + logits_at(a, lh, seq_row, s) + token_at(a, j);
#pragma unroll
      for (int g = 0; g < kMostLogits; ++g)
        if (g < a.G) y[g] = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(z + g * kTile));
      if (j + 4 <= held) __builtin_memcpy(was, to, 16);
    }
    int split0, splits;
    splits_of(a, s, split0, splits);
    norms_of<D, THREADS>(a, lh, split0, splits, a.G, norm_s);
    if (j >= held) return;
#pragma unroll
    for (int g = 0; g < kMostLogits; ++g)
      if (g < a.G) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] += weight_of(y[g][e], cl2, norm_s[g]);
      }
    if (j + 4 <= held) {
#pragma unroll
      for (int e = 0; e < 4; ++e) was[e] += w[e];
      __builtin_memcpy(to, was, 16);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (j + e < held) to[e] += w[e];
    }
  }
}

// out and lse of a (layer, sequence, KV head, 16 query heads), or of one query
// head of them: the splits' states merged by a running maximum, four in flight
// per thread. A thread per (head, channel), or with one head a group of
// THREADS / D threads per channel over the splits, merged in order. The first
// `gathers` workgroups add up weights instead.
template <int D, int THREADS, bool ONE, int GATHER>
__global__ __launch_bounds__(THREADS) void combine8_kernel(Attend8Args a, int gathers) {
  constexpr int ST = D + 2;
  constexpr int J = ONE ? THREADS / D : 1;
  constexpr int kAhead = 4;
  __shared__ float om[J][D], mm[J], zm[J];
  const Cache8View& c = a.c;
  int at = blockIdx.x;
  if constexpr (GATHER != kNone) {
    if (at < gathers) {
      gather<D, THREADS, GATHER == kSweep>(a, at);
      return;
    }
    at -= gathers;
  }
  const int tid = threadIdx.x;
  const int tiles = (a.G + 15) / 16, per = min(a.G, 16);
  int g0 = 0;
  if (ONE) {
    g0 = uniform(at % per);
    at = uniform(at / per);
  }
  const int unit = uniform(at / c.S), s = uniform(at - unit * c.S);
  const int lh = unit / tiles, hd0 = 16 * (unit - lh * tiles) + g0;
  const int heads = ONE ? 1 : min(a.G - hd0, 16);
  if (hd0 >= a.G) return;  // the last tile may be narrower: uniform
  int first, n;
  splits_of(a, s, first, n);
  const size_t stride = (size_t)per * ST;
  const float* __restrict__ base =
      a.partial + ((size_t)unit * a.splits + first) * stride + (size_t)g0 * ST;
  const int l = lh / c.H, h = lh - l * c.H;
  const size_t row = ((size_t)l * c.S + s) * a.Hq + h * a.G + hd0;
  const int jg = ONE ? tid / D : 0;
  for (int e = ONE ? tid % D : tid; e < heads * D; e += THREADS) {
    const int hd = e / D, ch = e - hd * D;
    const float* __restrict__ p = base + (size_t)hd * ST;
    float M = -INFINITY, Z = 0.f, O = 0.f;
    for (int j0 = jg; j0 < n; j0 += J * kAhead) {
      float m[kAhead], z[kAhead], o[kAhead];
      float top = M;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int j = min(j0 + J * u, n - 1);
        m[u] = p[j * stride + D];
        z[u] = p[j * stride + D + 1];
        o[u] = p[j * stride + ch];
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (j0 + J * u >= n) m[u] = -INFINITY, z[u] = o[u] = 0.f;
        top = fmaxf(top, m[u]);
      }
      const float f = M == -INFINITY ? 0.f : fast_exp2(M - top);
      Z *= f;  // a NaN sum stays NaN
      O *= f;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const float x = m[u] == -INFINITY ? 0.f : fast_exp2(m[u] - top);
        Z = fmaf(z[u], x, Z);
        O = fmaf(o[u], x, O);
      }
      M = top;
    }
    if constexpr (ONE) {
      om[jg][ch] = O;
      if (ch == 0) {
        mm[jg] = M;
        zm[jg] = Z;
      }
    } else {
      finish(a, row + hd, ch, D, M, Z, O);
    }
  }
  if constexpr (ONE) {
    __syncthreads();
    if (tid >= D) return;
    float M = -INFINITY, Z = 0.f, O = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) M = fmaxf(M, mm[j]);
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const float x = mm[j] == -INFINITY ? 0.f : fast_exp2(mm[j] - M);
      Z = fmaf(zm[j], x, Z);
      O = fmaf(om[j][tid], x, O);
    }
    finish(a, row, tid, D, M, Z, O);
  }
}

int64_t units_of(const Attend8Args& a) { return (int64_t)a.c.L * a.c.H * ((a.G + 15) / 16); }
// Workgroups of the attention, as many for each of the 8 XCDs.
int64_t attend_workgroups(const Attend8Args& a) {
  return a.by_length ? (units_of(a) + 7) / 8 * 8 * a.splits : (units_of(a) * a.splits + 7) / 8 * 8;
}
bool few_workgroups(const Attend8Args& a) { return a.single && attend_workgroups(a) <= 256; }
// The merge: one query head a workgroup while there are few.
bool merges_heads(const Attend8Args& a) { return units_of(a) * a.c.S >= 512; }
int64_t gather_workgroups(const Attend8Args& a) {
  const int rows = (a.sweep ? a.sweep : 4) * (merges_heads(a) ? kMergeThreads : kMergeOne);
  return (int64_t)a.c.L * a.c.H * (a.c.rows / rows + a.c.S);
}

}  // namespace

// Splits for the rooms. Short sequences are one split each, which needs no merge (up
// to about the length at which the merge's launch costs less than the wait); 8 waves
// share it while there are at most 256. Otherwise about 4096 rows a split, or 8192 of
// long sequences (131071 tokens 339 against 334 us, 504 against 489 with weights: fewer
// states to write and merge; of 700 to 8192 it would leave too few workgroups), but
// enough splits for four workgroups on each of the 256 compute units while those have
// a tile per wave. Batches take their longest splits first: 16 sequences of 700 to 8192
// 366 against 350 us.
void plan_attend8(Attend8Args& a, const int32_t* cu_rows_host) {
  const int64_t units = units_of(a);
  a.min_rows = kTile * kWaves;
  int64_t total = 0, most = 0, longest = 0;
  for (int s = 0; s < a.c.S; ++s) {
    const int64_t n = cu_rows_host[s + 1] - cu_rows_host[s];
    total += n;
    longest = std::max(longest, n);
    most += (n + a.min_rows - 1) / a.min_rows;
  }
  const int64_t rows = units * a.c.S;  // workgroups of one split a sequence
  const int64_t most_single = rows > 256 ? 1024 : std::min<int64_t>(2048, 640 + 12 * rows);
  a.single = longest * (a.c.d + 64) / 192 <= most_single && a.G <= 16;
  a.by_length = a.lds_bytes = a.sweep = 0;
  if (a.single) {
    a.splits = a.c.S;
    // few workgroups: a CU's LDS has room for the logits of a short sequence (300
    // tokens, 4 heads: a call 10.6 us with logits in memory, 8.2 so)
    const int64_t bytes = (longest + kTile - 1) / kTile * a.G * kTile * (int64_t)sizeof(float);
    if (few_workgroups(a) && bytes <= kMostLds) a.lds_bytes = (int)bytes;
    return;
  }
  const int64_t split_rows = longest >= 32768 ? 8192 : 4096;
  const int64_t want = std::max<int64_t>((1024 + units - 1) / units, total / split_rows);
  a.splits = (int)std::max<int64_t>(std::min<int64_t>(most, want + a.c.S), 1);
  a.by_length = a.c.S > 1 && a.c.S <= kWave && units >= 64;
  // Logits are 4 bytes a head written and read, keys d bytes read. us with logits and with
  // keys, of 28 layers x 4 heads x 16 sequences of 700 to 8192 and of 8 layers x 8 heads x
  // 131071 tokens:
  //   d 128  G 8 538, 570 and 549, 572   G 9 551, 576 and 562, 571   G 10 563, 580 and 572, 577
  //          G 12 585, 583 and 593, 579
  //   d 64   G 4 290, 312 and 302, 321   G 5 289, 303 and 312, 317   G 7 309, 306 and 333, 318
  //          G 8 322, 308 and 344, 319
  // so G 5 at d 64 is up to 5% faster with logits. One layer of them a call is faster with
  // logits up to G 10: d 128, G 10 37, 48 and 87, 97; d 64, G 8 25, 30 and 53, 57; G 12 at d 64
  // 30, 32 and 60, 60. (kMostLogits is the widest group that this leaves to the logits.)
  if (a.G * 14 > a.c.d || a.G > kMostLogits)
    a.sweep = (int)std::min<int64_t>(std::max<int64_t>((int64_t)a.c.L * a.c.H * total / (kBlock8 * 8192), 1), kMostBlocks);
}

size_t attend8_partial_floats(const Attend8Args& a) {
  if (a.single) return 0;
  return (size_t)units_of(a) * a.splits * std::min(a.G, 16) * (a.c.d + 2);
}

size_t attend8_logits(const Attend8Args& a) {
  if (a.lds_bytes > 0 || a.sweep) return 0;
  return (size_t)units_of(a) * (a.c.rows / kTile + a.c.S) * std::min(a.G, 16) * kTile;
}

bool attend8_fits(const Attend8Args& a) {
  // 8 waves a workgroup only where there are few; the merge's where there are many
  return grid_fits(attend_workgroups(a), kWaves * kWave) &&
         (a.single || grid_fits(units_of(a) * a.c.S * (merges_heads(a) ? 1 : std::min(a.G, 16)) +
                                    (a.gather ? gather_workgroups(a) : 0),
                                merges_heads(a) ? kMergeThreads : kMergeOne));
}

namespace {

template <int D>
void launch_attend(const Attend8Args& a, hipStream_t st) {
  const unsigned units = (unsigned)units_of(a);
  const dim3 grid((unsigned)attend_workgroups(a));
  auto copies = [&](auto nw, auto cc) {
    constexpr int NW = decltype(nw)::value, C = decltype(cc)::value;
    if (!a.gather || a.sweep)
      hipLaunchKernelGGL((attend8_kernel<D, NW, kNone, C>), grid, dim3(NW * kWave), 0, st, a);
    else if (a.lds_bytes == 0)
      hipLaunchKernelGGL((attend8_kernel<D, NW, kMemory, C>), grid, dim3(NW * kWave), 0, st, a);
    else if constexpr (NW == kWavesFew)
      hipLaunchKernelGGL((attend8_kernel<D, NW, kLds, C>), grid, dim3(NW * kWave), a.lds_bytes, st, a);
  };
  auto run = [&](auto nw) {
    if (a.G <= 5) copies(nw, std::integral_constant<int, 3>{});
    else copies(nw, std::integral_constant<int, 1>{});
  };
  if (few_workgroups(a)) run(std::integral_constant<int, kWavesFew>{});
  else run(std::integral_constant<int, kWaves>{});
  if (a.single) return;
  const unsigned rows = units * (unsigned)a.c.S, gathers = a.gather ? (unsigned)gather_workgroups(a) : 0u;
  auto merge = [&](auto gather) {
    constexpr int GATHER = decltype(gather)::value;
    if (merges_heads(a))
      hipLaunchKernelGGL((combine8_kernel<D, kMergeThreads, false, GATHER>), dim3(gathers + rows),
                         dim3(kMergeThreads), 0, st, a, (int)gathers);
    else
      hipLaunchKernelGGL((combine8_kernel<D, kMergeOne, true, GATHER>),
                         dim3(gathers + rows * std::min(a.G, 16)), dim3(kMergeOne), 0, st, a, (int)gathers);
  };
  if (!a.gather) merge(std::integral_constant<int, kNone>{});
  else if (a.sweep) merge(std::integral_constant<int, kSweep>{});
  else merge(std::integral_constant<int, kMemory>{});
}

}  // namespace

hipError_t launch_attend8(const Attend8Args& a, hipStream_t st) {
  if (a.c.d == 128) launch_attend<128>(a, st);
  else launch_attend<64>(a, st);
  return hipGetLastError();
}

}  // namespace stepkv
