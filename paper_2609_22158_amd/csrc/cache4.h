// Kernel launch interface of the 4-bit cache (include/stepkv_cache4.h) between
// its C ABI layer (cache4_api.cpp) and the HIP kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "launch.h"

namespace stepkv {

constexpr int kBlock4 = 64;  // tokens of a block (STEPKV_CACHE4_BLOCK)
constexpr int kGroup4 = 32;  // channels of a scale (STEPKV_CACHE4_GROUP)

// The cache as the kernels see it.
struct Cache4View {
  uint8_t* k_codes;          // [L*H][rows][d/2]
  uint8_t* v_codes;
  uint8_t* k_scales;         // [L*H][rows][d/32]
  uint8_t* v_scales;
  uint16_t* k_bounds;        // bf16 [L*H][nblk][2][d], or null
  const int32_t* cu_rows;    // [S+1]
  int32_t* lens;             // [S]
  uint32_t* status;          // device status word (STEPKV_FLAG_*) or null
  int L, H, S, d, rows, nblk;
};

// ---------------------------------------------------------------- write, read
struct Write4Args {
  Cache4View c;
  const uint16_t* k;         // bf16, element strides below
  const uint16_t* v;
  int64_t k_layer, k_row, k_head, v_layer, v_row, v_head;
  const int32_t* cu_src;     // compact: cu_seqlens; append: cu_new
  const int32_t* cu_retained;// compact; append: null
  const int32_t* idx;        // compact: [L*H][nsrc] or [nsrc]
  int nsrc;                  // source rows (Ntot, num_new)
  int shared_idx;
  int nblocks;               // (sequence, block) pairs a (layer, head) can touch
};
bool write4_fits(const Write4Args& a);
hipError_t launch_write4(const Write4Args& a, hipStream_t st);
hipError_t launch_advance4(const Cache4View& c, const int32_t* cu_new, hipStream_t st);

struct Read4Args {
  Cache4View c;
  const int32_t* cu_out;     // [S+1]
  uint16_t* k_out;           // bf16 [L*H][out_rows][d], or null
  uint16_t* v_out;
  int out_rows;
};
bool read4_fits(const Read4Args& a);
hipError_t launch_read4(const Read4Args& a, hipStream_t st);

// ---------------------------------------------------------------- attention
struct Attend4Args {
  Cache4View c;
  const uint16_t* q;         // bf16 [L][S][Hq][d]
  const int32_t* blocks;     // [L][S][H][nlist] or null
  float* out;                // [L][S][Hq][d]
  float* lse;                // [L][S][Hq] or null
  float* partial;            // [L*H*tiles][splits][min(G, 16)][d+2]: o, m (log2), z
  int Hq, G, nlist;
  int splits;                // split slots of a (layer, KV head)
  int min_rows;              // least rows of a split
  int single;                // nonzero: a sequence is one split, written without a merge
  float scale;
};
// Fills splits, min_rows and single from the shape and the rooms of the sequences.
void plan_attend4(Attend4Args& a, const int32_t* cu_rows_host);
size_t attend4_partial_floats(const Attend4Args& a);
bool attend4_fits(const Attend4Args& a);
hipError_t launch_attend4(const Attend4Args& a, hipStream_t st);

// ---------------------------------------------------------------- block selection
struct Select4Args {
  Cache4View c;
  const uint16_t* q;         // bf16 [L][S][Hq][d]
  uint64_t* keys;            // workspace [L*H][nblk]: ordered scores
  int32_t* blocks;           // [L][S][H][n]
  int Hq, G, n, first, last;
  int chunks;                // score chunks of a (layer, KV head); 0: scored where selected
  int most;                  // blocks that the longest sequence has room for
};
// Fills chunks and most from the shape and the rooms of the sequences.
void plan_select4(Select4Args& a, const int32_t* cu_rows_host);
bool select4_fits(const Select4Args& a);
hipError_t launch_select4(const Select4Args& a, hipStream_t st);

}  // namespace stepkv
