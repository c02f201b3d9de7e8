/*
 * stepkv_cache4.h - a KV cache held in 4 bits, and what reads it (gfx950).
 *
 * The compacted cache of a trajectory (stepkv.h) serves the decoding steps
 * until the next pruning boundary and grows by their tokens. Here its rows
 * are held in 4 bits a channel with one scale byte per 32 channels, 17/64 of
 * the bytes of bf16:
 *
 *   stepkv_cache4_compact   the retained rows of a boundary, quantised as they
 *                           are gathered (eq. problem, like stepkv_compact)
 *   stepkv_cache4_advance   a step's new tokens get their rows ...
 *   stepkv_cache4_append    ... and are quantised into them, layer by layer
 *   stepkv_cache4_read      rows back in bf16 (the next boundary's scoring)
 *   stepkv_cache4_decode    one decode step's attention over the cache, or
 *                           over a list of its blocks
 *   stepkv_cache4_select_blocks   the blocks of 64 rows that score best for a
 *                           decode step's queries
 *   stepkv_cache4_decode_sparse   that selection and attention over it
 *
 * Conventions (ownership, streams, errors, validation) are those of stepkv.h.
 * Calls allocate nothing and may be captured into HIP graphs: a replay uses
 * the values that lens, cu_new, ... hold when it runs.
 *
 * The format. A group is 32 channels of one row (channels 32 g .. 32 g + 31).
 *   e     = the smallest integer with max|x| <= 7 * 2^e over the group,
 *           clamped to [-124, 125]; its scale byte is e + 127
 *   code  = x / 2^e rounded to the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 (codes
 *           0 .. 7; ties to the even code; 6 above 6), plus 8 where x has its
 *           sign bit set
 *   value = element * 2^(byte - 127), exact in bf16. Byte 255: the group held
 *           a NaN or an infinity, and all its values are NaN.
 * Quantising values that were read back gives the same codes and scales, so a
 * cache that is read back, pruned and written again loses nothing more.
 * Channel 2 i is the low half of byte i of a row's codes.
 *
 * Layouts (L layers, H KV heads, d head dim, R = cu_rows[S] rows, S sequences):
 *   k_codes, v_codes    uint8 [L][H][R][d/2]   16-byte aligned
 *   k_scales, v_scales  uint8 [L][H][R][d/32]  aligned to d/32 bytes
 *   k_bounds            bf16  [L][H][floor(R/64) + S][2][d]  16-byte aligned
 *   lens                int32 [S]
 * Sequence s owns rows cu_rows[s] .. cu_rows[s+1] - 1 (its room) and holds
 * lens[s] tokens, token j in row cu_rows[s] + j. lens[s] may exceed the room:
 * tokens past it are neither stored nor read, and calls that write or attend
 * set STEPKV_FLAG_OUT_ROWS. So does a writing call for a token of its span that
 * has no source (a compacted position outside its sequence, a new token at or
 * past num_new): such a token keeps what its row holds, and counts as that.
 * Rows that hold no token are never read or written.
 * Block b of sequence s is its tokens 64 b .. 64 b + 63; k_bounds holds the
 * least (0) and greatest (1) key value per channel over the tokens that the
 * block holds (NaN where one is NaN), at block floor(cu_rows[s]/64) + s + b. They
 * are kept by the calls that write; where lens[s] was lowered by the caller, the
 * last block's are those of its earlier tokens too (wider, and bounds still).
 */
#ifndef STEPKV_CACHE4_H_
#define STEPKV_CACHE4_H_

#include "stepkv.h"

#ifdef __cplusplus
extern "C" {
#endif

#define STEPKV_CACHE4_BLOCK 64 /* tokens of a block */
#define STEPKV_CACHE4_GROUP 32 /* channels of a scale */
/* Rows of a (layer, KV head), cu_rows[S], and of a read (EUNSUPPORTED beyond):
 * sums of rows and of a split's length stay within 31 bits. A call whose launch
 * would have 2^32 threads or more (2^24 workgroups of 256: as many blocks of 64
 * rows written, or sequences attended to, over all layers and heads) is
 * EUNSUPPORTED too. */
#define STEPKV_CACHE4_MAX_ROWS ((1 << 30) - (1 << 20))

/* A cache: its shape, the rows of its sequences, and its device buffers (all
 * owned by the caller). The layers l0 .. l0 + n - 1 of a cache are a cache of
 * n layers whose buffer pointers are offset (a model's own layer); they share
 * cu_rows and lens. */
typedef struct stepkv_cache4 {
  int32_t num_layers;   /* L >= 1 */
  int32_t num_kv_heads; /* H >= 1 */
  int32_t head_dim;     /* d: 64 or 128 */
  int32_t num_seqs;     /* S >= 1 */
  const int32_t* cu_rows_host; /* [S+1] host: 0 = cu_rows[0] <= cu_rows[1] <= ... (read at
                                  every call: it sizes the launches) */
  const int32_t* cu_rows;      /* [S+1] device copy of the same values */
  int32_t* lens;               /* [S] device: tokens of every sequence */
  void* k_codes;
  void* v_codes;
  void* k_scales;
  void* v_scales;
  void* k_bounds;   /* NULL: none are kept (no block selection) */
  uint32_t* status; /* device status word as stepkv_problem.status, or NULL */
} stepkv_cache4;

/* eq. problem into 4 bits: for every (l, h) and sequence s, token
 * j < R_s = cu_retained[s+1] - cu_retained[s] of the cache becomes
 * k[l][h][cu_seqlens[s] + idx[l][h][cu_seqlens[s] + j]], and likewise v;
 * lens[s] = R_s. (An R_s past the sequence's source tokens counts as these, and
 * sets STEPKV_FLAG_OUT_ROWS.) pb gives the source (num_layers, num_kv_heads, head_dim and
 * num_seqs as the cache's); k, v, idx and cu_retained are as stepkv_compact's,
 * and idx is int32 [Ntot], one set for every layer and head, if shared_idx is
 * nonzero. A position outside its sequence leaves its row as it was
 * (STEPKV_FLAG_OUT_ROWS). k_bounds of the R_s tokens' blocks are set.
 * STEPKV_FLAG_NONFINITE: a group held a NaN or an infinity. Errors: EINVAL (null
 * or misaligned pointers, a bad problem or cache, shapes that differ),
 * EUNSUPPORTED (d, rows), EHIP. */
int stepkv_cache4_compact(const stepkv_problem* pb, const stepkv_cache4* c, const void* k,
                          const void* v, const int32_t* idx, int32_t shared_idx,
                          const int32_t* cu_retained, void* stream);

/* lens[s] += cu_new[s+1] - cu_new[s] for every sequence: rows for a step's new
 * tokens, once for all layers, before they are appended (cu_new: device int32
 * [S+1], non-decreasing). Errors: EINVAL, EHIP. */
int stepkv_cache4_advance(const stepkv_cache4* c, const int32_t* cu_new, void* stream);

/* Quantises new tokens into the last rows of their sequences: tokens
 * cu_new[s] .. cu_new[s+1] - 1 of k_new and v_new become the last
 * n_s = cu_new[s+1] - cu_new[s] tokens of sequence s, lens[s] - n_s ..
 * lens[s] - 1. num_new is the number of tokens that k_new and v_new hold (host;
 * tokens at or past it are not read: their rows stay as they were, and
 * STEPKV_FLAG_OUT_ROWS is set; with num_new 0 nothing is done at all); n_s may
 * be zero. Token t of layer l and head h is the d contiguous bf16 values at
 *   k_new + l * k_strides[0] + t * k_strides[1] + h * k_strides[2]
 * (strides in elements, multiples of 8, host int64 [3]; k_new 16-byte
 * aligned), so token-major and head-major tensors and slices of them serve
 * alike; v_new likewise. k_bounds: a block whose first token is among the new
 * ones starts anew, others widen (appending the same tokens again changes
 * nothing; other values in their place leave bounds that still hold).
 * STEPKV_FLAG_NONFINITE as compact. Errors: EINVAL, EUNSUPPORTED (d, rows), EHIP. */
int stepkv_cache4_append(const stepkv_cache4* c, const void* k_new, const int64_t* k_strides,
                         const void* v_new, const int64_t* v_strides, const int32_t* cu_new,
                         int32_t num_new, void* stream);

/* The last n_s = cu_out[s+1] - cu_out[s] tokens of every sequence in bf16:
 * row cu_out[s] + i of k_out and v_out, bf16 [L][H][out_rows][d], is token
 * lens[s] - n_s + i. With cu_out the prefix sums of lens these are the whole
 * sequences, in the layout that stepkv_score takes. Rows at or past out_rows
 * and rows without a token are left as they were. k_out or v_out may be NULL:
 * it is not read back. Errors: EINVAL (both NULL with out_rows > 0, negative
 * out_rows, misaligned pointers), EUNSUPPORTED (d, rows, out_rows), EHIP. */
int stepkv_cache4_read(const stepkv_cache4* c, const int32_t* cu_out, int32_t out_rows,
                       void* k_out, void* v_out, void* stream);

/* Bytes of device workspace stepkv_cache4_decode needs for num_q_heads query
 * heads (0 when invalid); num_blocks as the call's, 0 without a list. 256: the
 * call needs none, and takes NULL (short sequences, which are not split). */
size_t stepkv_cache4_decode_workspace_bytes(const stepkv_cache4* c, int32_t num_q_heads,
                                            int32_t num_blocks);

/* One decode step: for every layer, sequence and query head hq (KV head
 * hq / (num_q_heads / H)),
 *   out = softmax(scale * q . K^T) V
 * over the tokens of the sequence. q_dec bf16 [L][S][Hq][d], 16-byte aligned;
 * out fp32 [L][S][Hq][d]; lse fp32 [L][S][Hq] or NULL: the natural-log
 * log-sum-exp of the row's logits, with which results over several caches can
 * be joined. A sequence without tokens gives zeros, and -inf. scale <= 0
 * selects 1/sqrt(d). A logit that overflows fp32 to -inf has no weight; where
 * every one does, the result is NaN, and the log-sum-exp -inf.
 * blocks (int32 [L][S][H][num_blocks], or NULL with num_blocks 0): attention
 * over the tokens of the listed blocks only, an ascending list per (layer,
 * sequence, KV head); an entry that is no block of the sequence (-1), or is
 * not above every entry before it, is passed over, and so are the entries past
 * as many as the sequence has blocks.
 * A NaN in an attended key, value or query makes its results NaN, and so does a
 * logit that overflows to +inf. fp32 sums of exact products; the probabilities, in
 * fp32 and up to 2^16, are divided by their sum after the products of the n tokens
 * attended to with the values were added up: of values past 2^111 / n these may
 * overflow. Results are the same from call to call. What other sequences hold does
 * not enter them; how many tokens they hold may move the borders of the splits, and
 * so change the last bits.
 * Errors: EINVAL (also a scale whose product with log2(e) overflows),
 * EUNSUPPORTED (d, rows), EWORKSPACE (below stepkv_cache4_decode_workspace_bytes,
 * or not 256-byte aligned), EHIP. */
int stepkv_cache4_decode(const stepkv_cache4* c, int32_t num_q_heads, const void* q_dec,
                         const int32_t* blocks, int32_t num_blocks, float scale, float* out,
                         float* lse, void* workspace, size_t ws_bytes, void* stream);

/* Bytes of device workspace stepkv_cache4_select_blocks needs (0 when invalid). */
size_t stepkv_cache4_select_workspace_bytes(const stepkv_cache4* c);

/* The num_blocks blocks of every (layer, sequence, KV head) that a decode step
 * attends to: the first first_blocks and the last last_blocks of the sequence,
 * and those others with the greatest score
 *   score(b) = sum over the heads g of the KV head and the channels i of
 *              max(q_gi kmin_bi, q_gi kmax_bi),
 * (q kmax where q > 0, q kmin where q < 0), an upper bound of the group's summed
 * logits in the block, computed in 64 bits; a NaN score ranks as -inf, equal
 * scores the lower block first. So a NaN in any of the group's queries, which
 * makes every score NaN, lists the lowest blocks. Written ascending to blocks
 * int32 [L][S][H][num_blocks], -1 past the last; all the blocks of a sequence
 * that has no more than num_blocks.
 * Errors: EINVAL (also a cache without k_bounds, num_blocks < 1, negative
 * counts, first_blocks + last_blocks > num_blocks), EUNSUPPORTED (d, rows),
 * EWORKSPACE, EHIP. */
int stepkv_cache4_select_blocks(const stepkv_cache4* c, int32_t num_q_heads, const void* q_dec,
                                int32_t num_blocks, int32_t first_blocks, int32_t last_blocks,
                                int32_t* blocks, void* workspace, size_t ws_bytes, void* stream);

/* Bytes of device workspace stepkv_cache4_decode_sparse needs (0 when invalid). */
size_t stepkv_cache4_sparse_workspace_bytes(const stepkv_cache4* c, int32_t num_q_heads,
                                            int32_t num_blocks);

/* stepkv_cache4_select_blocks, then stepkv_cache4_decode over the selected
 * blocks, with the same arguments, results and errors. blocks (required) is
 * written. */
int stepkv_cache4_decode_sparse(const stepkv_cache4* c, int32_t num_q_heads, const void* q_dec,
                                int32_t num_blocks, int32_t first_blocks, int32_t last_blocks,
                                float scale, int32_t* blocks, float* out, float* lse,
                                void* workspace, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* STEPKV_CACHE4_H_ */
