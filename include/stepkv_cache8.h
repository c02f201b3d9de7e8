/*
 * stepkv_cache8.h - a KV cache held in 8 bits, the attention that reads it and
 * gathers each token's weight, and eviction by those weights (gfx950).
 *
 * Like the 4-bit cache (stepkv_cache4.h) it serves the decoding steps between
 * two pruning boundaries (stepkv.h), in half the bytes of bf16:
 *
 *   stepkv_cache8_compact   the retained rows of a boundary, quantised as they
 *                           are gathered (eq. problem, like stepkv_compact)
 *   stepkv_cache8_advance   a step's new tokens get their rows ...
 *   stepkv_cache8_append    ... and are quantised into them, layer by layer
 *   stepkv_cache8_read      rows back in bf16 (the next boundary's scoring)
 *   stepkv_cache8_decode    one decode step's attention over the cache; it can
 *                           add every token's attention weight to what the
 *                           token has gathered
 *   stepkv_cache8_evict     the tokens of least gathered weight are given up
 *
 * With the last two the cache keeps its size between boundaries: an H2O-style
 * policy (tokens by accumulated attention, and the recent ones) where the pass
 * of stepkv.h prunes once per reasoning step.
 *
 * Conventions (ownership, streams, errors, validation) are those of stepkv.h.
 * Calls allocate nothing and may be captured into HIP graphs: a replay uses
 * the values that lens, cu_new, ... hold when it runs.
 *
 * The format. An element is an e4m3 number (OCP: bias 7, 448 the greatest,
 * 2^-9 the least, no infinities), times a power of two 2^e that the 64 tokens
 * of a block share: one for the keys and one for the values of each (layer, KV
 * head, block). Block b of sequence s is its tokens 64 b .. 64 b + 63.
 *   need  of some rows: the smallest e with max|x| <= 464 * 2^e over their
 *         finite elements, clamped to [-117, 119] (464: what still rounds to 448)
 *   e     of a block: when its first token is written, the need of the rows that
 *         the call writes into it; afterwards it grows to the need of every row
 *         written or moved into it. It does not shrink. Where it grows, the
 *         block's other tokens are rounded to the new power.
 *   code  = x / 2^e rounded to the nearest e4m3 number, ties to even, at most
 *         448; a NaN or an infinity is held as NaN.
 *   value = element * 2^e, exact in bf16.
 * An element of magnitude up to 464 * 2^119 is off by at most 2^-4 of it, or by
 * 2^-9 * 2^E if that is more, where E is the greatest exponent that a block had
 * while it held the element: its block's e, however often that grew (powers of
 * two move e4m3 numbers without a rounding above 2^-6), and, of a row that
 * eviction moved, those of the blocks that it was in before too. Finite elements
 * of greater magnitude are held as 448 * 2^119, the greatest bf16 value 12.2% low.
 * Quantising rows that were read back, block by block, gives the same values.
 *
 * Layouts (L layers, H KV heads, d head dim, R = cu_rows[S] rows, S sequences):
 *   k_codes, v_codes    uint8 [L][H][R][d]  16-byte aligned
 *   k_scales, v_scales  fp32  [L][H][floor(R/64) + S], 2^e of block b of sequence s
 *                       at floor(cu_rows[s]/64) + s + b; 4-byte aligned
 *   weights             fp32  [L][H][R]  attention weight that a token gathered
 *   positions           int32 [L][H][R]  its position in its sequence
 *   lens, seen          int32 [S]
 * Sequence s owns rows cu_rows[s] .. cu_rows[s+1] - 1 (its room) and holds
 * lens[s] tokens, token j in row cu_rows[s] + j; seen[s] tokens came so far,
 * those that were pruned or evicted included, and the next one's position is
 * seen[s]. Eviction moves tokens, each head its own: their order is that of
 * positions, which attention does not depend on. lens[s] may exceed the room:
 * tokens past it are neither stored nor read, and calls that write, attend or
 * evict set STEPKV_FLAG_OUT_ROWS. So does a writing call for a token of its span
 * that has no source (a compacted position outside its sequence, a new token at
 * or past num_new): such a token's row keeps its bytes (but for the rounding to
 * a scale that grows), and counts as a token. Rows that hold no token are never
 * read or written, and scales are read as powers of two (their exponent bits).
 */
#ifndef STEPKV_CACHE8_H_
#define STEPKV_CACHE8_H_

#include "stepkv.h"

#ifdef __cplusplus
extern "C" {
#endif

#define STEPKV_CACHE8_BLOCK 64 /* tokens of a scale */
/* Rows of a (layer, KV head), cu_rows[S], and of a read (EUNSUPPORTED beyond):
 * sums of rows and of a split's length stay within 31 bits. A call whose launch
 * would have 2^32 threads or more is EUNSUPPORTED too. */
#define STEPKV_CACHE8_MAX_ROWS ((1 << 30) - (1 << 20))

/* A cache: its shape, the rows of its sequences, and its device buffers (all
 * owned by the caller). The layers l0 .. l0 + n - 1 of a cache are a cache of
 * n layers whose buffer pointers are offset (a model's own layer); they share
 * cu_rows, lens and seen. */
typedef struct stepkv_cache8 {
  int32_t num_layers;   /* L >= 1 */
  int32_t num_kv_heads; /* H >= 1 */
  int32_t head_dim;     /* d: 64 or 128 */
  int32_t num_seqs;     /* S >= 1 */
  const int32_t* cu_rows_host; /* [S+1] host: 0 = cu_rows[0] <= cu_rows[1] <= ... (read at
                                  every call: it sizes the launches) */
  const int32_t* cu_rows;      /* [S+1] device copy of the same values */
  int32_t* lens;               /* [S] device: tokens of every sequence */
  int32_t* seen;               /* [S] device: tokens that came so far */
  void* k_codes;
  void* v_codes;
  float* k_scales;
  float* v_scales;
  float* weights;      /* NULL, and positions too: nothing is gathered or evicted */
  int32_t* positions;
  uint32_t* status;    /* device status word as stepkv_problem.status, or NULL */
} stepkv_cache8;

/* eq. problem into 8 bits: for every (l, h) and sequence s, token
 * j < R_s = cu_retained[s+1] - cu_retained[s] of the cache becomes
 * k[l][h][cu_seqlens[s] + i] with i = idx[l][h][cu_seqlens[s] + j], and likewise
 * v; lens[s] = R_s, and seen[s] = the sequence's source tokens. (An R_s past those
 * counts as them, and sets STEPKV_FLAG_OUT_ROWS.) The token's position is i, and
 * its weight weights[l][h][cu_seqlens[s] + i] (fp32 [L][H][Ntot], for instance the
 * window's saliency; NULL: 0). pb gives the source (num_layers, num_kv_heads,
 * head_dim and num_seqs as the cache's); k, v, idx and cu_retained are as
 * stepkv_compact's, and idx is int32 [Ntot], one set for every layer and head, if
 * shared_idx is nonzero. A position outside its sequence leaves its row as it was
 * (STEPKV_FLAG_OUT_ROWS). STEPKV_FLAG_NONFINITE: a row held a NaN or an infinity.
 * Errors: EINVAL (null or misaligned pointers, a bad problem or cache, shapes that
 * differ, weights for a cache without), EUNSUPPORTED (d, rows), EHIP. */
int stepkv_cache8_compact(const stepkv_problem* pb, const stepkv_cache8* c, const void* k,
                          const void* v, const int32_t* idx, int32_t shared_idx,
                          const int32_t* cu_retained, const float* weights, void* stream);

/* lens[s] and seen[s] += cu_new[s+1] - cu_new[s] for every sequence: rows for a
 * step's new tokens, once for all layers, before they are appended (cu_new:
 * device int32 [S+1], non-decreasing). Errors: EINVAL, EHIP. */
int stepkv_cache8_advance(const stepkv_cache8* c, const int32_t* cu_new, void* stream);

/* Quantises new tokens into the last rows of their sequences: tokens
 * cu_new[s] .. cu_new[s+1] - 1 of k_new and v_new become the last
 * n_s = cu_new[s+1] - cu_new[s] tokens of sequence s, lens[s] - n_s ..
 * lens[s] - 1, at positions seen[s] - n_s .. seen[s] - 1, with weight 0. num_new
 * is the number of tokens that k_new and v_new hold (host; tokens at or past it
 * are not read: their rows keep their bytes, and STEPKV_FLAG_OUT_ROWS is set;
 * with num_new 0 nothing is done at all); n_s may be zero. Token t of layer l and
 * head h is the d contiguous bf16 values at
 *   k_new + l * k_strides[0] + t * k_strides[1] + h * k_strides[2]
 * (strides in elements, multiples of 8, host int64 [3]; k_new 16-byte
 * aligned), so token-major and head-major tensors and slices of them serve
 * alike; v_new likewise. Appending the same tokens again changes nothing but the
 * weights, which are 0 again. STEPKV_FLAG_NONFINITE as compact. Errors: EINVAL,
 * EUNSUPPORTED (d, rows), EHIP. */
int stepkv_cache8_append(const stepkv_cache8* c, const void* k_new, const int64_t* k_strides,
                         const void* v_new, const int64_t* v_strides, const int32_t* cu_new,
                         int32_t num_new, void* stream);

/* The last n_s = cu_out[s+1] - cu_out[s] tokens of every sequence in bf16:
 * row cu_out[s] + i of k_out and v_out, bf16 [L][H][out_rows][d], is token
 * lens[s] - n_s + i. With cu_out the prefix sums of lens these are the whole
 * sequences, in the layout that stepkv_score takes. Rows at or past out_rows
 * and rows without a token are left as they were. k_out or v_out may be NULL:
 * it is not read back. Errors: EINVAL (both NULL with out_rows > 0, negative
 * out_rows, misaligned pointers), EUNSUPPORTED (d, rows, out_rows), EHIP. */
int stepkv_cache8_read(const stepkv_cache8* c, const int32_t* cu_out, int32_t out_rows,
                       void* k_out, void* v_out, void* stream);

/* Bytes of device workspace stepkv_cache8_decode needs for num_q_heads query
 * heads (0 when invalid). 256: the call needs none, and takes NULL (short
 * sequences, which are not split, without gathering or a few of them). */
size_t stepkv_cache8_decode_workspace_bytes(const stepkv_cache8* c, int32_t num_q_heads,
                                            int32_t gather);

/* One decode step: for every layer, sequence and query head hq (KV head
 * hq / (num_q_heads / H)),
 *   out = sum_j p_j v_j,  p = softmax(scale * q . K^T)
 * over the tokens of the sequence. q_dec bf16 [L][S][Hq][d], 16-byte aligned;
 * out fp32 [L][S][Hq][d]; lse fp32 [L][S][Hq] or NULL: the natural-log
 * log-sum-exp of the row's logits, with which results over several caches can
 * be joined. If gather is nonzero, every token's weight in the cache becomes
 *   weights[l][h][j] + sum over the query heads of KV head h of p_j.
 * A sequence without tokens gives zeros, and -inf. scale <= 0 selects 1/sqrt(d).
 * A logit that overflows fp32 to -inf has no weight; where every one does, the
 * result is NaN, the log-sum-exp -inf and the tokens' weights NaN. A NaN in an
 * attended key, value or query makes its results NaN (in a key or query also the
 * weights of the KV head's tokens), and so does a logit that overflows to +inf.
 * fp32 sums of exact products; the probabilities, in fp32 and up to 2^16, are
 * divided by their sum after the n tokens' products with the values were added up:
 * of values past 2^111 / n these may overflow. Results are the same from call to
 * call. What other sequences hold does not enter them; how many tokens they hold
 * may move the borders of the splits, and so change the last bits.
 * Errors: EINVAL (also a scale whose product with log2(e) overflows, gather on a
 * cache without weights), EUNSUPPORTED (d, rows), EWORKSPACE (below
 * stepkv_cache8_decode_workspace_bytes, or not 256-byte aligned), EHIP. */
int stepkv_cache8_decode(const stepkv_cache8* c, int32_t num_q_heads, const void* q_dec,
                         float scale, int32_t gather, float* out, float* lse, void* workspace,
                         size_t ws_bytes, void* stream);

/* Bytes of device workspace stepkv_cache8_evict needs (0 when invalid). */
size_t stepkv_cache8_evict_workspace_bytes(const stepkv_cache8* c);

/* Every sequence that holds more than K_s tokens gives up the others, in every
 * (layer, KV head) its own: the K_s that stay are the first in this order:
 *   tokens with position < first or >= seen[s] - recent, the lower rows first;
 *   then by gathered weight, the greatest first, of equal ones the lower rows
 *   (a NaN weight ranks as -inf, -0 as +0).
 * K_s is `keep`, or max(1, keeps[s]) when keeps (device int32 [S]) is non-NULL.
 * Tokens that stay in rows K_s and above move, with their weights and positions,
 * into the rows below K_s that became free: in the order of the rows, the i-th
 * into the i-th. Other tokens are not touched, but for the rounding to a block's
 * scale that grows with a row moved into it. lens[s] becomes K_s. The rows that
 * no longer hold a token are left as they were.
 * lens is shared by all layers: the cache has to be the whole one, with every
 * layer appended to.
 * Errors: EINVAL (also keep < 1 without keeps, negative first or recent, a cache
 * without weights and positions), EUNSUPPORTED (d, rows), EWORKSPACE, EHIP.
 * Deterministic. */
int stepkv_cache8_evict(const stepkv_cache8* c, int32_t keep, const int32_t* keeps, int32_t first,
                        int32_t recent, void* workspace, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* STEPKV_CACHE8_H_ */
