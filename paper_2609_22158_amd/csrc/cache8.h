// Kernel launch interface of the 8-bit cache (include/stepkv_cache8.h) between
// its C ABI layer (cache8_api.cpp) and the HIP kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "launch.h"

namespace stepkv {

constexpr int kBlock8 = 64;  // tokens of a scale (STEPKV_CACHE8_BLOCK)

// The cache as the kernels see it.
struct Cache8View {
  uint8_t* k_codes;          // [L*H][rows][d]
  uint8_t* v_codes;
  float* k_scales;           // [L*H][nblk]
  float* v_scales;
  float* weights;            // [L*H][rows], or null
  int32_t* positions;        // [L*H][rows], or null
  const int32_t* cu_rows;    // [S+1]
  int32_t* lens;             // [S]
  int32_t* seen;             // [S]
  uint32_t* status;          // device status word (STEPKV_FLAG_*) or null
  int L, H, S, d, rows, nblk;
};

// ---------------------------------------------------------------- write, read
struct Write8Args {
  Cache8View c;
  const uint16_t* k;         // bf16, element strides below
  const uint16_t* v;
  int64_t k_layer, k_row, k_head, v_layer, v_row, v_head;
  const int32_t* cu_src;     // compact: cu_seqlens; append: cu_new
  const int32_t* cu_retained;// compact; append: null
  const int32_t* idx;        // compact: [L*H][nsrc] or [nsrc]
  const float* gathered;     // compact: source weights [L*H][nsrc], or null
  int nsrc;                  // source rows (Ntot, num_new)
  int shared_idx;
  int nblocks;               // (sequence, block) pairs a (layer, head) can touch
};
bool write8_fits(const Write8Args& a);
hipError_t launch_write8(const Write8Args& a, hipStream_t st);
hipError_t launch_advance8(const Cache8View& c, const int32_t* cu_new, hipStream_t st);

struct Read8Args {
  Cache8View c;
  const int32_t* cu_out;     // [S+1]
  uint16_t* k_out;           // bf16 [L*H][out_rows][d], or null
  uint16_t* v_out;
  int out_rows;
};
bool read8_fits(const Read8Args& a);
hipError_t launch_read8(const Read8Args& a, hipStream_t st);

// ---------------------------------------------------------------- attention
struct Attend8Args {
  Cache8View c;
  const uint16_t* q;         // bf16 [L][S][Hq][d]
  float* out;                // [L][S][Hq][d]
  float* lse;                // [L][S][Hq] or null
  float* partial;            // [L*H*tiles][splits][min(G, 16)][d+2]: o, m (log2), z
  float* logits;             // gather: the logits, unscaled, by tiles of tokens
  int Hq, G;
  int splits;                // split slots of a (layer, KV head)
  int min_rows;              // least rows of a split
  int single;                // nonzero: a sequence is one split, written without a merge
  int by_length;             // nonzero: the longest splits are taken first
  int gather;                // nonzero: weights are added up
  int sweep;                 // nonzero: from the keys, read again, this many blocks a wave (then logits is null)
  int lds_bytes;             // of the logits, where LDS holds them (then logits is null)
  float scale;
};
// Fills splits, min_rows, single, by_length, sweep and lds_bytes from the shape and the rooms of the sequences.
void plan_attend8(Attend8Args& a, const int32_t* cu_rows_host);
size_t attend8_partial_floats(const Attend8Args& a);
size_t attend8_logits(const Attend8Args& a);  // floats of them
bool attend8_fits(const Attend8Args& a);
hipError_t launch_attend8(const Attend8Args& a, hipStream_t st);

// ---------------------------------------------------------------- eviction
// What the selection leaves for the moves of one (layer, KV head, sequence).
struct Evict8Head {
  int moves;                 // rows that move
  int keep;                  // tokens that stay, or -1: the sequence is not touched
  float k_scale, v_scale;    // of the block that holds row `keep`, before any move
};
struct Evict8Args {
  Cache8View c;
  const int32_t* keeps;      // [S] or null
  Evict8Head* heads;         // workspace [L*H][S]
  int2* moves;               // workspace [L*H][rows / 2]: (to, from), ascending; sequence s
                             // from cu_rows[s] / 2 (it moves no more than half of its room)
  int keep, first, recent;
  int workers;               // waves that move rows of a (layer, KV head, sequence)
  int longest;               // rows of the longest room
};
void plan_evict8(Evict8Args& a, const int32_t* cu_rows_host);
bool evict8_fits(const Evict8Args& a);
hipError_t launch_evict8(const Evict8Args& a, hipStream_t st);

}  // namespace stepkv
