// One decode step's attention over the 4-bit cache: out = softmax(scale *
// q . K^T) V per (layer, sequence, query head), over all tokens or over the
// listed blocks of 64.
//
// The cache's 17/16 d bytes a token and KV head bound it. A chip that streams
// them at full rate has about four vector operations a value to spend, which
// rules out arithmetic dequantisation; the conversion instruction gives two
// exact bf16 values, scale included, and both products run on MFMA.
//
// attend4_kernel: one workgroup per (layer, KV head, 16 query heads, split of
// a sequence's tokens), its waves on consecutive runs of 32-token tiles, each
// with its own online softmax. Per tile and wave:
//  - K: lane (g, r) = (l / 16, l % 16) holds row r's channels D/4 g .. + D/4 - 1
//    (16 bytes of codes; one scale) as the A operand of
//    v_mfma_f32_16x16x32_bf16, 8 channels a step; the query heads are the B
//    operand in the same channel order. Lane (g, r) then holds head r's
//    logits of rows 4 g .. 4 g + 3 of each 16-row half.
//  - softmax per head in that layout, in the log2 domain, with a reference
//    that moves only when a logit exceeds it by kSlack.
//  - V: lane l converts 32 channels (one scale) of one row to bf16 and puts
//    them into the wave's LDS tile; ds_read_b64_tr_b16 gives them back as the
//    B operand, a column's 4 + 4 rows per lane in the order in which the lane
//    holds P. P is the A operand, as three bf16 parts that are it exactly (in
//    one operand for narrow groups); the same parts times ones give the
//    softmax's sum on the matrix cores, which have the time.
// The next tile is loaded where the registers of a tile are free, before its
// softmax and P V. A second set of registers, loaded a tile earlier, costs a
// wave per SIMD and is no faster (8 layers x 8 heads x 131071 rows, splits of
// 1024: 215 us against 207).
// combine4_kernel merges the splits.
#include "cache4_device.h"

#include <math.h>

#include <algorithm>
#include <type_traits>

namespace stepkv {
namespace {

typedef float f32x4_t __attribute__((__vector_size__(4 * sizeof(float))));
typedef short i16x4_t __attribute__((__vector_size__(4 * sizeof(short))));

constexpr int kTile = 32;  // tokens a wave computes at a time
constexpr int kWaves = 4;  // waves of a workgroup
constexpr int kMergeThreads = 256;  // of a merge of many rows
constexpr float kSlack = 16.f;
constexpr float kLog2e = 1.44269504088896341f;

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

// Rows that sequence s gives to the splits: its tokens, or 64 per list entry.
// No more entries are looked at than the sequence has blocks.
__device__ __forceinline__ int split_rows_of(const Attend4Args& a, int s) {
  const int n = held_tokens(a.c, s);
  return a.blocks ? kBlock4 * min(a.nlist, (n + kBlock4 - 1) / kBlock4) : n;
}

__device__ __forceinline__ int split_rows_const(const Attend4Args& a, int held) {
  return a.blocks ? kBlock4 * min(a.nlist, (held + kBlock4 - 1) / kBlock4) : held;
}

// Rows of a split, from the tokens there are when the kernel runs: as many as
// give at most a.splits splits in all, sum_s ceil(n_s / rows) <= total / rows +
// nonempty sequences. A multiple of a tile for each of the waves.
__device__ __forceinline__ int rows_per_split(const Attend4Args& a) {
  const int lane = threadIdx.x & 63;
  int64_t total = 0;
  int some = 0, most = 0;  // most: splits of min_rows
  for (int s0 = 0; s0 < a.c.S; s0 += kWave) {
    const int n = s0 + lane < a.c.S ? split_rows_of(a, s0 + lane) : 0;
    total += (uint32_t)wave_total(wave_scan(n));  // the rooms add up to less than 2^31
    some += __popcll(ballot(n > 0));
    most += wave_total(wave_scan((n + a.min_rows - 1) / a.min_rows));
  }
  if (most <= a.splits) return a.min_rows;
  const int slots = max(a.splits - some, 1);
  const int64_t rows = (total + slots - 1) / slots;
  return (int)((max(rows, (int64_t)a.min_rows) + a.min_rows - 1) / a.min_rows * a.min_rows);
}

// Byte offset of piece j (8 channels) of group g of row r in a wave's V tile,
// row-major: with the XORs the writes of 16 lanes (whole rows) and the
// transposing reads of 32 lanes (32 bytes of each of 8 rows) touch every bank
// once.
template <int D>
__device__ __forceinline__ int v_write(int r, int j, int g) {
  return D == 128 ? r * 256 + 64 * (j ^ (r & 3)) + 32 * ((g >> 1) ^ ((r >> 2) & 1)) + 16 * (g & 1)
                  : r * 128 + 32 * (j ^ ((r >> 1) & 3)) + 16 * g;
}
// Column block (j, gp): pieces j of groups 2 gp and 2 gp + 1, row r, part c of 4.
template <int D>
__device__ __forceinline__ int v_read(int r, int j, int gp, int c) {
  return D == 128 ? r * 256 + 64 * (j ^ (r & 3)) + 32 * (gp ^ ((r >> 2) & 1)) + 8 * c
                  : r * 128 + 32 * (j ^ ((r >> 1) & 3)) + 8 * c;
}

typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;

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

// The reference of a wave that saw tokens, whose logits are all -inf: below every
// logit, but not that of a wave without tokens.
constexpr float kNoWeight = -3.40282347e38f;

// The result of a query head from its sums (row: (layer, sequence, query head)).
// Without a token zeros; where every logit is -inf (an overflow) the softmax of
// such logits, 0 / 0.
__device__ __forceinline__ void finish(const Attend4Args& a, size_t row, int ch, int D, float M,
                                       float Z, float O) {
  a.out[row * D + ch] = M == -INFINITY && Z == 0.f ? 0.f : O / Z;
  if (a.lse && ch == 0) a.lse[row] = Z == 0.f ? -INFINITY : (M + log2f(Z)) * 0.693147180559945309f;
}

// NW waves share a split (or, with a.single, a whole sequence); C copies (1 or 3)
// of the query heads in the operands' rows.
template <int D, int NW, bool LIST, int C>
__global__ __launch_bounds__(NW * kWave) __attribute__((amdgpu_waves_per_eu(LIST && D == 128 ? 3 : 4)))
void attend4_kernel(Attend4Args a) {
  constexpr int NS = D / kGroup4;    // scales a row; MFMA steps of S
  constexpr int VL = D / 64;         // 16-byte V pieces a lane loads per tile: 2 or 1
  constexpr int VR = kTile / VL;     // rows between them
  constexpr int GPN = D / 64;        // column blocks per piece index j
  constexpr int NB = 4 * GPN;        // 16-column blocks of O
  constexpr int ST = D + 2;
  constexpr int TB = kTile * D * 2;  // bytes of a V tile
  constexpr int kStateBytes = NW * 16 * ST * 4;
  __shared__ __attribute__((aligned(16)))
  uint8_t smem[NW * TB > kStateBytes ? NW * TB : kStateBytes];
  __shared__ __attribute__((aligned(16))) float fscale[NW][16];
  const Cache4View& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int g4 = lane >> 4, c16 = lane & 15;
  if (blockIdx.x == 0 && wave == 0) report_rooms(c);
  // Workgroups are dealt to the 8 XCDs in turn; each XCD takes a contiguous
  // eighth of the splits (8 layers x 8 heads x 131071 rows: 184 -> 179 us; with
  // the heads within a split instead 204).
  const int bid = (int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3);
  const int unit = uniform(bid / a.splits);  // (layer, KV head, 16 query heads)
  const int gs = uniform(bid - unit * a.splits);
  const int tiles = (a.G + 15) / 16;
  if (unit >= c.L * c.H * tiles) return;  // the grid is padded to a multiple of 8
  const int lh = uniform(unit / tiles), hd0 = 16 * (unit - lh * tiles);  // first head of the group
  const int l = uniform(lh / c.H), h = lh - l * c.H;
  int s = gs, w0, w1;  // this wave's rows [w0, w1) of those of its sequence
  if (a.single) {
    const int share = (split_rows_const(a, held_const(c, s)) + NW * kTile - 1) / (NW * kTile) * kTile;
    w0 = wave * share;
    w1 = w0 + share;
  } else {
    int first;
    const int split = rows_per_split(a);
    locate_item(c.S, gs, [&](int sq) { return (split_rows_of(a, sq) + split - 1) / split; }, s,
                first);
    if (s < 0) return;  // past the last split: uniform over the workgroup
    w0 = (gs - first) * split + wave * (split / NW);
    w1 = w0 + split / NW;
  }
  s = uniform(s);
  const int held = held_const(c, s), n = split_rows_const(a, held);
  const int t0 = uniform(w0 / kTile), t1 = uniform((min(n, w1) + kTile - 1) / kTile);  // its tiles
  const int heads = min(a.G - hd0, 16);
  constexpr int kCols = 16 / C;  // columns of a copy
  const int copy = c16 / kCols, hcol = c16 % kCols;
  bf16x8_t qb[NS];
#pragma unroll
  for (int ks = 0; ks < NS; ++ks) {
    qb[ks] = bf16x8_t{};
    if (hcol < heads && copy < C)
      qb[ks] = *reinterpret_cast<const bf16x8_t*>(
          a.q + (((size_t)l * c.S + s) * a.Hq + h * a.G + hd0 + hcol) * D + D / 4 * g4 + 8 * ks);
  }
  const float cl2 = a.scale * kLog2e;
  float m_ref = -INFINITY;
  f32x4_t o[NB], z = f32x4_t{};
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) o[nb] = f32x4_t{};
  const size_t row0 = (size_t)lh * c.rows + read_const(c.cu_rows, s);
  const int32_t* __restrict__ list =
      LIST ? a.blocks + (((size_t)l * c.S + s) * c.H + h) * a.nlist : nullptr;
  uint8_t* const vt = smem + wave * TB;
  const int vrow = lane / NS, vgrp = lane % NS;  // this lane's V row and group

  // The first token of tile t (held: none).
  const int nlist = LIST ? n / kBlock4 : 0;
  int entry = -1, ebase = -1, above = -1;  // lane i: entry ebase + i; all entries before: <= above
  if (LIST && t0 < t1) {
    for (int e = lane; e < t0 / 2; e += kWave) above = max(above, list[e]);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) above = max(above, __shfl_xor(above, off, kWave));
  }
  auto tile_token = [&](int t) -> int {
    if constexpr (!LIST) {
      return t * kTile;
    } else {
      const int e = t >> 1;
      if (ebase < 0 || e >= ebase + kWave) {  // the next 64 entries (t only grows)
        ebase = e;
        int v = e + lane < nlist ? list[e + lane] : -1;
        int before = v;  // maximum of the entries up to this lane's
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
          const int x = __shfl_up(before, off, kWave);
          if (lane >= off) before = max(before, x);
        }
        const int top = __shfl(before, kWave - 1, kWave);
        int prev = __shfl_up(before, 1, kWave);
        prev = lane == 0 ? above : max(prev, above);
        entry = v > prev && v < (held + kBlock4 - 1) / kBlock4 ? v : -1;
        above = max(above, top);
      }
      const int b = __builtin_amdgcn_readlane(entry, e - ebase);
      return b < 0 ? held : b * kBlock4 + (t & 1) * kTile;
    }
  };

  // A row's scales are loaded whole, as a word of their own type: a byte would
  // be extended where it arrives, which waits for the next tile's loads there.
  using Scales = typename std::conditional<D == 128, uint32_t, uint16_t>::type;
  struct Tile {
    uint32_t k[2][NS];
    u32x4_t v[VL];
    Scales ks[2], vs[VL];
    int base;
  };
  // The scale of group g as the conversions take it, which look at bits 23 .. 30 alone.
  auto scale = [](Scales w, int g) {
    if constexpr (D == 128) return __uint_as_float(__builtin_amdgcn_alignbit(w, w, 8 * g - 23));
    else return __uint_as_float((uint32_t)w << (23 - 8 * g));
  };
  // Loads tile t (or, past the end, again the last one, so that the count of
  // loads in flight is the same in every round).
  auto load = [&](Tile& x, int t) __attribute__((always_inline)) {
    x.base = uniform(tile_token(min(t, t1 - 1)));
    const int b = min(x.base, held - 1), last = held - 1 - b;
    const size_t row = row0 + b;
    const uint8_t* __restrict__ kc = c.k_codes + row * (D / 2);
    const uint8_t* __restrict__ vc = c.v_codes + row * (D / 2);
    const Scales* __restrict__ ksc = reinterpret_cast<const Scales*>(c.k_scales) + row;
    const Scales* __restrict__ vsc = reinterpret_cast<const Scales*>(c.v_scales) + row;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t r = min(16 * u + c16, last);  // rows past the end: the last one again
      if constexpr (D == 128) {
        const u32x4_t w = __builtin_nontemporal_load(
            reinterpret_cast<const u32x4_t*>(kc + (r * (D / 2) + 16 * g4)));
#pragma unroll
        for (int i = 0; i < 4; ++i) x.k[u][i] = w[i];
      } else {
        const u32x2_t w = __builtin_nontemporal_load(
            reinterpret_cast<const u32x2_t*>(kc + (r * (D / 2) + 8 * g4)));
        x.k[u][0] = w[0];
        x.k[u][1] = w[1];
      }
      x.ks[u] = ksc[r];
    }
#pragma unroll
    for (int u = 0; u < VL; ++u) {
      const uint32_t r = min(VR * u + vrow, last);
      x.v[u] = __builtin_nontemporal_load(
          reinterpret_cast<const u32x4_t*>(vc + (r * (D / 2) + 16 * vgrp)));
      x.vs[u] = vsc[r];
    }
  };
  // The first half of a tile's work, after which its registers are free: the
  // logits on the matrix cores, V as bf16 in LDS.
  f32x4_t acc[2];
  auto consume = [&](const Tile& x) __attribute__((always_inline)) {
    acc[0] = acc[1] = f32x4_t{};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float sk = scale(x.ks[u], g4 * NS / 4);
#pragma unroll
      for (int ks = 0; ks < NS; ++ks)
        acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            __builtin_bit_cast(bf16x8_t, spread8(x.k[u][ks], sk)), qb[ks], acc[u], 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < VL; ++u) {
      const float sv = scale(x.vs[u], vgrp);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t w = x.v[u][j];
        *reinterpret_cast<u32x4_t*>(vt + v_write<D>(VR * u + vrow, j, vgrp)) = spread8(w, sv);
      }
    }
  };
  auto attend = [&](int tok) __attribute__((always_inline)) {
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
    constexpr int kOps = 2;  // column blocks at a time (4: as fast, but 6 registers more)
#pragma unroll
    for (int nb0 = 0; nb0 < NB; nb0 += kOps) {
      bf16x8_t vb[kOps];
#pragma unroll
      for (int i = 0; i < kOps; ++i) {
        const int j = (nb0 + i) / GPN, gp = (nb0 + i) % GPN;
        i16x4_t b[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
          b[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds_i16x4*)(vt + v_read<D>(4 * g4 + (c16 >> 2), j, gp, c16 & 3) + u * 16 * 2 * D));
        vb[i] = __builtin_bit_cast(bf16x8_t,
                                   __builtin_shufflevector(b[0], b[1], 0, 1, 2, 3, 4, 5, 6, 7));
      }
#pragma unroll
      for (int k = 0; k < Parts<C>::N; ++k)
#pragma unroll
        for (int i = 0; i < kOps; ++i)
          o[nb0 + i] =
              __builtin_amdgcn_mfma_f32_16x16x32_bf16(pp.x[k], vb[i], o[nb0 + i], 0, 0, 0);
    }
  };
  bool any = false;  // a tile with tokens
  if (t0 < t1) {
    Tile cur;
    load(cur, t0);
    for (int t = t0; t < t1; ++t) {  // wave-uniform
      const int tok = cur.base;
      const bool some = !LIST || tok < held;
      if (some) consume(cur);
      load(cur, t + 1);
      if (some) attend(tok);
      any |= some;
    }
  }
  __syncthreads();  // the states overwrite the V tiles of every wave
  auto state = reinterpret_cast<float(*)[16][ST]>(smem);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((4 * g4 + i) % kCols < heads && (4 * g4 + i) / kCols < C) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int gp = 0; gp < GPN; ++gp)
          state[wave][4 * g4 + i][32 * (2 * gp + (c16 >> 3)) + 8 * j + (c16 & 7)] =
              o[j * GPN + gp][i];
      if (c16 == 0) state[wave][4 * g4 + i][D + 1] = z[i];
    }
  }
  if (g4 == 0 && c16 < heads)  // the same in every copy
    state[wave][c16][D] = any ? fmaxf(m_ref, kNoWeight) : -INFINITY;
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
      continue;
    }
    part[hd * ST + ch] = O;
    if (ch == 0) {
      part[hd * ST + D] = M;
      part[hd * ST + D + 1] = Z;
    }
  }
}

// out and lse of a (layer, sequence, KV head, 16 query heads), or of one query
// head of them: the splits' states merged by a running maximum, four in flight
// per thread. A thread per (head, channel), or with one head a group of
// THREADS / D threads per channel over the splits, merged in order. Two waits for
// memory bound it: 4 us for 64 heads of 33 splits each, 11 for 1792 x 7 heads of
// one or two.
template <int D, int THREADS, bool ONE>
__global__ __launch_bounds__(THREADS) void combine4_kernel(Attend4Args a) {
  constexpr int ST = D + 2;
  constexpr int J = ONE ? THREADS / D : 1;
  constexpr int kAhead = 4;
  __shared__ float om[J][D], mm[J], zm[J];
  const Cache4View& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63;
  const int tiles = (a.G + 15) / 16, per = min(a.G, 16);
  int at = blockIdx.x, g0 = 0;
  if (ONE) {
    g0 = uniform(at % per);
    at = uniform(at / per);
  }
  const int unit = uniform(at / c.S), s = at - unit * c.S;
  const int lh = unit / tiles, hd0 = 16 * (unit - lh * tiles) + g0;
  const int heads = ONE ? 1 : min(a.G - hd0, 16);
  if (hd0 >= a.G) return;  // the last tile may be narrower: uniform
  const int split = rows_per_split(a);
  int first = 0;  // splits of the sequences before s
  for (int s0 = 0; s0 < s; s0 += kWave)
    first += wave_total(
        wave_scan(s0 + lane < s ? (split_rows_of(a, s0 + lane) + split - 1) / split : 0));
  first = min(first, a.splits);
  const int n =
      min((split_rows_const(a, held_const(c, s)) + split - 1) / split, a.splits - first);
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

}  // namespace

// Splits for the rooms. Short sequences are one split each, which needs no merge;
// 8 waves share it while there are at most 256. Such a step takes about 5.5 us and
// 4.2 ns a row of the longest sequence (d 64: 2.5 ns), splits and their merge 8.5
// us and more for more sequences (8 heads, d 128, one sequence of 600 rows: 7.6 us
// in one split, 8.6 in many; of 1536 11.3, 8.5; 16 sequences of 600: 8.5, 13.1; of
// 2048 14.9, 19.0; 28 layers x 4 heads x 16 sequences x 1024: 57, 94). Otherwise about 4096 rows a split (a wave's
// start and merge cost about three tiles; 8 layers x 8 heads x 131071 rows: 1024
// rows 226 us, 2048 197, 4096 193, 8192 197), but enough splits for four
// workgroups on each of the 256 compute units while those have a tile per wave.
void plan_attend4(Attend4Args& a, const int32_t* cu_rows_host) {
  const int64_t units = (int64_t)a.c.L * a.c.H * ((a.G + 15) / 16);
  a.min_rows = kTile * kWaves;
  int64_t total = 0, most = 0, longest = 0;
  for (int s = 0; s < a.c.S; ++s) {
    int64_t n = cu_rows_host[s + 1] - cu_rows_host[s];
    if (a.nlist > 0) n = kBlock4 * std::min<int64_t>(a.nlist, (n + kBlock4 - 1) / kBlock4);
    total += n;
    longest = std::max(longest, n);
    most += (n + a.min_rows - 1) / a.min_rows;
  }
  const int64_t rows = units * a.c.S;  // workgroups of one split a sequence
  const int64_t most_single = rows > 256 ? 1024 : std::min<int64_t>(2048, 640 + 12 * rows);
  a.single = longest * (a.c.d + 64) / 192 <= most_single;
  if (a.single) {
    a.splits = a.c.S;
    return;
  }
  const int64_t want = std::max<int64_t>((1024 + units - 1) / units, total / 4096);
  a.splits = (int)std::max<int64_t>(std::min<int64_t>(most, want + a.c.S), 1);
}

size_t attend4_partial_floats(const Attend4Args& a) {
  if (a.single) return 0;
  return (size_t)a.c.L * a.c.H * ((a.G + 15) / 16) * a.splits * std::min(a.G, 16) * (a.c.d + 2);
}

bool attend4_fits(const Attend4Args& a) {
  const int64_t units = (int64_t)a.c.L * a.c.H * ((a.G + 15) / 16);
  // 8 waves a workgroup only where there are few; the merge's where there are many
  return grid_fits((units * a.splits + 7) / 8 * 8, kWaves * kWave) &&
         (a.single || grid_fits(units * a.c.S, kMergeThreads));
}

namespace {

template <int D>
void launch_attend(const Attend4Args& a, hipStream_t st) {
  const unsigned units = (unsigned)(a.c.L * a.c.H) * (unsigned)((a.G + 15) / 16);
  const dim3 grid((units * (unsigned)a.splits + 7u) / 8u * 8u);
  auto copies = [&](auto nw, auto cc) {
    constexpr int NW = decltype(nw)::value, C = decltype(cc)::value;
    if (a.blocks)
      hipLaunchKernelGGL((attend4_kernel<D, NW, true, C>), grid, dim3(NW * kWave), 0, st, a);
    else
      hipLaunchKernelGGL((attend4_kernel<D, NW, false, C>), grid, dim3(NW * kWave), 0, st, a);
  };
  auto run = [&](auto nw) {
    if (a.G <= 5) copies(nw, std::integral_constant<int, 3>{});
    else copies(nw, std::integral_constant<int, 1>{});
  };
  if (a.single && grid.x <= 256) run(std::integral_constant<int, 8>{});
  else run(std::integral_constant<int, kWaves>{});
  if (a.single) return;
  const unsigned rows = units * (unsigned)a.c.S;
  if (rows >= 512)
    hipLaunchKernelGGL((combine4_kernel<D, kMergeThreads, false>), dim3(rows), dim3(kMergeThreads),
                       0, st, a);
  else
    hipLaunchKernelGGL((combine4_kernel<D, 512, true>), dim3(rows * std::min(a.G, 16)), dim3(512),
                       0, st, a);
}

}  // namespace

hipError_t launch_attend4(const Attend4Args& a, hipStream_t st) {
  if (a.c.d == 128) launch_attend<128>(a, st);
  else launch_attend<64>(a, st);
  return hipGetLastError();
}

}  // namespace stepkv
