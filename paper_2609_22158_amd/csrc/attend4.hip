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
//    holds P. P is the A operand, as bf16 hi + lo parts (P to 2^-16).
// The next tile's codes and scales are loaded before a tile is computed.
// combine4_kernel merges the splits.
#include "cache4_device.h"

#include <math.h>

#include <algorithm>

namespace stepkv {
namespace {

typedef float f32x4_t __attribute__((__vector_size__(4 * sizeof(float))));
typedef short i16x4_t __attribute__((__vector_size__(4 * sizeof(short))));

constexpr int kTile = 32;  // tokens a wave computes at a time
constexpr int kWaves = 4;  // waves of a workgroup
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

// Rows of a split, from the tokens there are when the kernel runs: as many as
// give at most a.splits splits in all, sum_s ceil(n_s / rows) <= total / rows +
// nonempty sequences. A multiple of a tile for each wave.
__device__ __forceinline__ int rows_per_split(const Attend4Args& a) {
  const int lane = threadIdx.x & 63;
  int64_t total = 0;
  int some = 0, most = 0;  // most: splits of min_rows
  for (int s0 = 0; s0 < a.c.S; s0 += kWave) {
    const int n = s0 + lane < a.c.S ? split_rows_of(a, s0 + lane) : 0;
    total += n;
    some += n > 0;
    most += (n + a.min_rows - 1) / a.min_rows;
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    total += __shfl_xor(total, off, kWave);
    some += __shfl_xor(some, off, kWave);
    most += __shfl_xor(most, off, kWave);
  }
  if (most <= a.splits) return a.min_rows;
  const int slots = max(a.splits - some, 1);
  const int64_t rows = (total + slots - 1) / slots;
  constexpr int kUnit = kTile * kWaves;
  return (int)((max(rows, (int64_t)a.min_rows) + kUnit - 1) / kUnit * kUnit);
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

template <int D, bool LIST>
__global__ __launch_bounds__(kWaves * kWave) void attend4_kernel(Attend4Args a) {
  constexpr int NS = D / kGroup4;    // scales a row; MFMA steps of S
  constexpr int KW = D / 32;         // code words of a lane's K row: 4 or 2
  constexpr int VL = D / 64;         // 16-byte V pieces a lane loads per tile: 2 or 1
  constexpr int VR = kTile / VL;     // rows between them
  constexpr int GPN = D / 64;        // column blocks per piece index j
  constexpr int NB = 4 * GPN;        // 16-column blocks of O
  constexpr int ST = D + 2;
  constexpr int TB = kTile * D * 2;  // bytes of a V tile
  constexpr int kStateBytes = kWaves * 16 * ST * 4;
  __shared__ __attribute__((aligned(16)))
  uint8_t smem[kWaves * TB > kStateBytes ? kWaves * TB : kStateBytes];
  __shared__ __attribute__((aligned(16))) float fscale[kWaves][16];
  const Cache4View& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int g4 = lane >> 4, c16 = lane & 15;
  if (blockIdx.x == 0 && tid == 0) report_rooms(c);
  const int unit = blockIdx.x / a.splits;  // (layer, KV head, 16 query heads)
  const int gs = blockIdx.x - unit * a.splits;
  const int tiles = (a.G + 15) / 16;
  const int lh = unit / tiles, hd0 = 16 * (unit - lh * tiles);  // first head of the group
  const int l = lh / c.H, h = lh - l * c.H;
  const int split = uniform(rows_per_split(a));
  int s, first;
  locate_item(c.S, gs, [&](int sq) { return (split_rows_of(a, sq) + split - 1) / split; }, s, first);
  if (s < 0) return;  // past the last split: uniform over the workgroup
  const int held = uniform(held_tokens(c, s));
  const int n = uniform(split_rows_of(a, s));
  // this wave's 32-row tiles [t0, t1)
  const int w0 = (gs - first) * split + wave * (split / kWaves);
  const int t0 = w0 / kTile, t1 = (min(n, w0 + split / kWaves) + kTile - 1) / kTile;
  const int heads = min(a.G - hd0, 16);
  bf16x8_t qb[NS];
#pragma unroll
  for (int ks = 0; ks < NS; ++ks) {
    qb[ks] = bf16x8_t{};
    if (c16 < heads)
      qb[ks] = *reinterpret_cast<const bf16x8_t*>(
          a.q + (((size_t)l * c.S + s) * a.Hq + h * a.G + hd0 + c16) * D + D / 4 * g4 + 8 * ks);
  }
  const float cl2 = a.scale * kLog2e;
  float m_ref = -INFINITY, zp = 0.f;
  f32x4_t o[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) o[nb] = f32x4_t{};
  const size_t row0 = (size_t)lh * c.rows + c.cu_rows[s];
  const uint8_t* __restrict__ kc = c.k_codes + row0 * (D / 2);
  const uint8_t* __restrict__ vc = c.v_codes + row0 * (D / 2);
  const uint8_t* __restrict__ ksc = c.k_scales + row0 * NS;
  const uint8_t* __restrict__ vsc = c.v_scales + row0 * NS;
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

  struct Tile {
    uint32_t k[2][KW];
    u32x4_t v[VL];
    uint32_t ks[2], vs[VL];
  };
  auto load = [&](Tile& x, int base) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const size_t r = min(base + 16 * u + c16, held - 1);
      if constexpr (D == 128) {
        const u32x4_t w = __builtin_nontemporal_load(
            reinterpret_cast<const u32x4_t*>(kc + r * (D / 2) + 16 * g4));
#pragma unroll
        for (int i = 0; i < 4; ++i) x.k[u][i] = w[i];
      } else {
        const u32x2_t w = __builtin_nontemporal_load(
            reinterpret_cast<const u32x2_t*>(kc + r * (D / 2) + 8 * g4));
        x.k[u][0] = w[0];
        x.k[u][1] = w[1];
      }
      x.ks[u] = ksc[r * NS + g4 * NS / 4];
    }
#pragma unroll
    for (int u = 0; u < VL; ++u) {
      const size_t r = min(base + VR * u + vrow, held - 1);
      x.v[u] = __builtin_nontemporal_load(
          reinterpret_cast<const u32x4_t*>(vc + r * (D / 2) + 16 * vgrp));
      x.vs[u] = vsc[r * NS + vgrp];
    }
  };
  auto compute = [&](const Tile& x, int base) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < VL; ++u) {
      const float sv = scale_of(x.vs[u]);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<u32x4_t*>(vt + v_write<D>(VR * u + vrow, j, vgrp)) =
            spread8(x.v[u][j], sv);
    }
    f32x4_t acc[2] = {f32x4_t{}, f32x4_t{}};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float sk = scale_of(x.ks[u]);
#pragma unroll
      for (int ks = 0; ks < NS; ++ks)
        acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            __builtin_bit_cast(bf16x8_t, spread8(x.k[u][ks], sk)), qb[ks], acc[u], 0, 0, 0);
    }
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = acc[i >> 2][i & 3] * cl2;
    if (base + kTile > held) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (base + 16 * (i >> 2) + 4 * g4 + (i & 3) >= held) y[i] = -INFINITY;
    }
    float tmax = y[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) tmax = fmaxf(tmax, y[i]);
    if (__builtin_amdgcn_ballot_w64(tmax > m_ref + kSlack) != 0) {  // wave-uniform, rare
      tmax = fmaxf(tmax, xor16(tmax));
      tmax = fmaxf(tmax, xor32(tmax));
      const float m_new = tmax > m_ref + kSlack ? tmax : m_ref;
      const float f = m_ref == -INFINITY ? 0.f : fast_exp2(m_ref - m_new);
      zp *= f;
      m_ref = m_new;
      if (g4 == 0) fscale[wave][c16] = f;
      __builtin_amdgcn_wave_barrier();
      const float4 f4 = *reinterpret_cast<const float4*>(&fscale[wave][4 * g4]);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        o[nb][0] *= f4.x;
        o[nb][1] *= f4.y;
        o[nb][2] *= f4.z;
        o[nb][3] *= f4.w;
      }
    }
    bf16x8_t ph, pl;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // -inf has no weight, also while the reference is still -inf
      const float p = y[i] == -INFINITY ? 0.f : fast_exp2(y[i] - m_ref);
      zp += p;
      ph[i] = (__bf16)p;
      pl[i] = (__bf16)(p - (float)ph[i]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int gp = 0; gp < GPN; ++gp) {
        const int r = 4 * g4 + (c16 >> 2);
        i16x4_t b[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
          b[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds_i16x4*)(vt + v_read<D>(r, j, gp, c16 & 3) + u * 16 * 2 * D));
        const bf16x8_t vb = __builtin_bit_cast(
            bf16x8_t, __builtin_shufflevector(b[0], b[1], 0, 1, 2, 3, 4, 5, 6, 7));
        const int nb = j * GPN + gp;
        o[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ph, vb, o[nb], 0, 0, 0);
        o[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pl, vb, o[nb], 0, 0, 0);
      }
  };
  if (t0 < t1) {
    Tile cur, nxt;
    int base = tile_token(t0);
    load(cur, base);
    for (int t = t0; t < t1; ++t) {  // wave-uniform
      int ahead = held;
      if (t + 1 < t1) {
        ahead = tile_token(t + 1);
        load(nxt, ahead);
      }
      if (base < held) compute(cur, base);
      cur = nxt;
      base = ahead;
    }
  }
  zp += xor16(zp);
  zp += xor32(zp);
  __syncthreads();  // the states overwrite the V tiles of every wave
  auto state = reinterpret_cast<float(*)[16][ST]>(smem);
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int gp = 0; gp < GPN; ++gp)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int ch = 32 * (2 * gp + (c16 >> 3)) + 8 * j + (c16 & 7);
        if (4 * g4 + i < heads) state[wave][4 * g4 + i][ch] = o[j * GPN + gp][i];
      }
  if (g4 == 0 && c16 < heads) {
    state[wave][c16][D] = m_ref;
    state[wave][c16][D + 1] = zp;
  }
  __syncthreads();
  float* const part = a.partial + ((size_t)unit * a.splits + gs) * min(a.G, 16) * ST;
  for (int e = tid; e < heads * D; e += kWaves * kWave) {
    const int hd = e / D, ch = e - hd * D;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, state[w][hd][D]);
    float Z = 0.f, O = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float m = state[w][hd][D];
      const float x = m == -INFINITY ? 0.f : fast_exp2(m - M);  // a NaN sum stays NaN
      Z = fmaf(state[w][hd][D + 1], x, Z);
      O = fmaf(state[w][hd][ch], x, O);
    }
    part[hd * ST + ch] = O;
    if (ch == 0) {
      part[hd * ST + D] = M;
      part[hd * ST + D + 1] = Z;
    }
  }
}

// out and lse of one (layer, sequence, query head): the splits' states merged.
// Thread groups of D share the splits; their sums are added in group order.
template <int D>
__global__ __launch_bounds__(256) void combine4_kernel(Attend4Args a) {
  constexpr int ST = D + 2;
  constexpr int J = 256 / D;
  __shared__ float osum[J][D], zsum[J];
  const Cache4View& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63;
  const int hq = blockIdx.x % a.Hq;
  const int s = (blockIdx.x / a.Hq) % c.S;
  const int l = blockIdx.x / (a.Hq * c.S);
  const int h = hq / a.G, g = hq - h * a.G;
  const int tiles = (a.G + 15) / 16, per = min(a.G, 16);
  const int unit = (l * c.H + h) * tiles + g / 16;
  const int split = uniform(rows_per_split(a));
  int first = 0;  // splits of the sequences before s
  for (int s0 = 0; s0 < s; s0 += kWave) {
    int cnt = s0 + lane < s ? (split_rows_of(a, s0 + lane) + split - 1) / split : 0;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) cnt += __shfl_xor(cnt, off, kWave);
    first += cnt;
  }
  first = min(uniform(first), a.splits);
  const int n = min(uniform((split_rows_of(a, s) + split - 1) / split), a.splits - first);
  const size_t stride = (size_t)per * ST;
  const float* __restrict__ base =
      a.partial + ((size_t)unit * a.splits + first) * stride + (size_t)(g % 16) * ST;
  float M = -INFINITY;
  for (int j = lane; j < n; j += kWave) M = fmaxf(M, base[j * stride + D]);
  M = wave_max(M);
  const int jg = tid / D, ch = tid % D;
  float Z = 0.f, O = 0.f;
  for (int j = jg; j < n; j += J) {
    const float m = base[j * stride + D];
    const float x = m == -INFINITY ? 0.f : fast_exp2(m - M);
    Z = fmaf(base[j * stride + D + 1], x, Z);
    O = fmaf(base[j * stride + ch], x, O);
  }
  osum[jg][ch] = O;
  if (ch == 0) zsum[jg] = Z;
  __syncthreads();
  if (tid >= D) return;
  Z = zsum[0];
  O = osum[0][ch];
#pragma unroll
  for (int j = 1; j < J; ++j) {
    Z += zsum[j];
    O += osum[j][ch];
  }
  const size_t row = ((size_t)l * c.S + s) * a.Hq + hq;
  a.out[row * D + ch] = Z == 0.f ? 0.f : O / Z;  // no token: zeros
  if (a.lse && ch == 0) a.lse[row] = Z == 0.f ? -INFINITY : (M + log2f(Z)) * 0.693147180559945309f;
}

}  // namespace

// Splits for the rooms: about 1024 rows each, but enough for four workgroups
// on each of the 256 compute units while those have a tile per wave.
void plan_attend4(Attend4Args& a, const int32_t* cu_rows_host) {
  const int64_t units = (int64_t)a.c.L * a.c.H * ((a.G + 15) / 16);
  a.min_rows = kTile * kWaves;
  int64_t total = 0, most = 0;
  for (int s = 0; s < a.c.S; ++s) {
    int64_t n = cu_rows_host[s + 1] - cu_rows_host[s];
    if (a.nlist > 0) n = kBlock4 * std::min<int64_t>(a.nlist, (n + kBlock4 - 1) / kBlock4);
    total += n;
    most += (n + a.min_rows - 1) / a.min_rows;
  }
  const int64_t want = std::max<int64_t>((1024 + units - 1) / units, total / 1024);
  a.splits = (int)std::max<int64_t>(std::min<int64_t>(most, want + a.c.S), 1);
}

size_t attend4_partial_floats(const Attend4Args& a) {
  return (size_t)a.c.L * a.c.H * ((a.G + 15) / 16) * a.splits * std::min(a.G, 16) * (a.c.d + 2);
}

hipError_t launch_attend4(const Attend4Args& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.c.L * a.c.H) * (unsigned)((a.G + 15) / 16) * (unsigned)a.splits);
  const dim3 block(kWaves * kWave);
  if (a.c.d == 128) {
    if (a.blocks) hipLaunchKernelGGL((attend4_kernel<128, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((attend4_kernel<128, false>), grid, block, 0, st, a);
  } else {
    if (a.blocks) hipLaunchKernelGGL((attend4_kernel<64, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((attend4_kernel<64, false>), grid, block, 0, st, a);
  }
  const dim3 rows((unsigned)(a.c.L * a.c.S) * (unsigned)a.Hq);
  if (a.c.d == 128) hipLaunchKernelGGL(combine4_kernel<128>, rows, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(combine4_kernel<64>, rows, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace stepkv
