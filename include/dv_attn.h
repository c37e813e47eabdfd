/* dv_attn.h -- operators over a KV cache held in 8 bits, for one MI355X (gfx950):
 *
 *   dv_quant_in   rounds a 16-bit contiguous buffer (the "wire" of dv.h) into an
 *                 8-bit cache: whole prompts, or a decode step's tokens;
 *   dv_attend     one layer's attention of the newest tokens over such a cache,
 *                 which also accumulates the weight each cached token received;
 *   dv_evict      keeps, of each head's tokens, the most recent and those with
 *                 the most accumulated weight, and compacts the cache.
 *
 * The conventions of dv.h hold: every argument is checked on the host before
 * anything is enqueued, the caller owns every buffer, nothing is allocated,
 * work is enqueued on `stream`, host arrays are read during the call only.
 * DV_ERR_HIP: the runtime refused a launch; earlier ones of the same call may
 * have been enqueued, so what the call writes is unspecified.  A call whose
 * every sequence is empty enqueues nothing and returns DV_OK.
 */
#ifndef DV_ATTN_H
#define DV_ATTN_H

#include "dv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* An 8-bit cache.  Its codes lie in a dv_cache with elem_bytes 1, DV_DENSE or
 * DV_PAGED, in device memory, so everything of dv.h streams and swaps the codes.
 * A code is an e4m3 number (sign, 4 exponent bits with bias 7, 3 fraction bits;
 * magnitudes 0 to 448, 0x7f and 0xff are NaN) and stands for code * scale; the
 * `scale_block` tokens of a block share one scale in each head, a power of two,
 * separately for keys and values:
 *   DV_DENSE  scale[layer][K|V][batch][head][ceil(max_seq / scale_block)],
 *             token s in block s / scale_block
 *   DV_PAGED  scale[layer][K|V][num_blocks][head]; scale_block == block_size
 * A scale that is not a power of two of [2^-64, 2^120] gives unspecified results
 * where a token of its block is used; blocks that no table names may hold anything.
 * Two optional companions go by slots (a token's place in its sequence):
 *   weight    [layer][batch][head][capacity]: accumulated attention weight;
 *   position  [layer][batch][head][capacity]: the tokens' positions, where they
 *             are not their slots (after an eviction).
 * capacity is max_seq, or max_blocks * block_size.  Each is a host array
 * [num_mb] of device addresses, or NULL; entries of the companions may be NULL
 * too.  Scales, weights and positions are 4-byte aligned.
 * A replica needs the scales as well as the codes.  Where they divide by 4 they
 * are a dv_cache of their own with elem_bytes 4, which streams and swaps them
 * (16-byte aligned then):
 *   DV_PAGED  num_heads a multiple of 4: one head, head_dim num_heads, block_size
 *             1, the same table; block j of a sequence is its token j
 *   DV_DENSE  ceil(max_seq / scale_block) a multiple of 4: head_dim 4, max_seq a
 *             quarter of it; blocks 4 j to 4 j + 3 are token j
 * Weights and positions, without K|V halves, are not: copy them as arrays. */
typedef struct dv_quant {
  const dv_cache* cache;
  int32_t scale_block;
  float* const* scale;
  float* const* weight;
  int32_t* const* position;
} dv_quant;

/* Types of the 16-bit numbers that go in and come out. */
typedef enum { DV_F16 = 0, DV_BF16 = 1 } dv_type;

/* Bytes of one microbatch's scale array.  Host-only. */
DV_API int dv_quant_scale_bytes(const dv_quant* c, uint64_t* out_bytes);

/* Append tokens [t0[b], t1[b]) of every sequence, layers [l0, l1), to microbatch
 * `mb` of `dst` (t0 may be NULL: all zero).  `src` is the wire of these ranges
 * with 2-byte elements of `type` (twice dv_packed_bytes(dst->cache, ...) bytes;
 * `src_bytes` is at least that), 16-byte aligned.  Per block of tokens and head:
 *   need  = the smallest power of two, 2^-64 or more, with 448 * need >= |x| for
 *           the block's new elements x
 *   scale = need where the block holds no token before t0[b], else the larger
 *           of need and the scale it has; where that grows, the codes of the
 *           tokens before t0[b] are rounded to it (exact, down to the smallest
 *           magnitudes)
 *   code  = x / scale, to the nearest, ties to the even code.
 * |x| above 240/256 of the type's 2^16 or 2^128 (infinities among them) counts
 * as that: the largest number of the format that the type still holds.  NaN
 * becomes NaN and counts for no scale.  A sequence ends at t1[b] afterwards:
 * slots of its last block past that hold nothing.  Weights of the new tokens
 * become zero; their positions go on from the token before t0[b] (from 0 where
 * t0[b] is 0), where those arrays are given.  Tokens whose table entry is
 * outside [0, num_blocks) are skipped.  `src` must not overlap the cache, its
 * table, scales or companions.
 * DV_OK, DV_ERR_INVALID, DV_ERR_RANGE, DV_ERR_SPACE, DV_ERR_UNSUPPORTED, DV_ERR_HIP. */
DV_API int dv_quant_in(const dv_quant* dst, int32_t mb, int32_t l0, int32_t l1, const int32_t* t0,
                       const int32_t* t1, const void* src, uint64_t src_bytes, int32_t type,
                       void* stream);

/* Queries and results of dv_attend.  Token i of sequence b is row
 * sum_{b' < b} q_len[b'] + i of q and out; element d of its head g lies at
 * row * token stride + g * head stride + d (strides in elements, multiples of 8
 * below 2^31; bases 16-byte aligned).  No two rows of out share an element. */
typedef struct dv_attend_args {
  int32_t type;     /* dv_type of q and out */
  int32_t q_heads;  /* a multiple of the cache's heads: query heads [k*G, (k+1)*G) share
                       cache head k, G = q_heads / num_heads */
  float scale;      /* the scores' factor, e.g. 1/sqrt(head_dim) */
  float decay;      /* with `weigh`: factor of the weights from before */
  int32_t weigh;    /* nonzero: accumulate into the cache's weight array */
  int32_t rows;     /* rows that q, out and lse have: at least the sum of q_len */
  const void* q;
  void* out;
  int64_t q_token, q_head, out_token, out_head; /* strides */
  const float* slopes; /* device [q_heads], or NULL: bias slope * (key's - query's position) */
  float* lse;          /* device [rows][q_heads], or NULL: log of the sum of exp of the scores */
  void* workspace;     /* device, 16-byte aligned, dv_attend_bytes of it (may be NULL if 0) */
  uint64_t workspace_bytes;
} dv_attend_args;

/* Workspace bytes of a dv_attend with these lengths; goes by a->type, q_heads
 * and weigh only.  Host-only. */
DV_API int dv_attend_bytes(const dv_quant* c, const int32_t* q_len, const int32_t* kv_len,
                           const dv_attend_args* a, uint64_t* out_bytes);

/* Attention over layer `layer` of microbatch `mb`.  Sequence b holds kv_len[b]
 * tokens, of which the last q_len[b] are the queries' own: query i stands in
 * slot a = kv_len[b] - q_len[b] + i and sees slots [0, a] (none where a < 0).
 *   score(t) = scale * q.k(t) + slope * (position(t) - position(a))
 *   p = softmax of the scores,   out = sum over t of p(t) v(t)
 * position(t) is the companion array's, or t where there is none.  A query that
 * sees nothing (also: whose slots are all unmapped) gets zeros and lse -infinity.
 * With `weigh`, for every slot t below kv_len[b] of every cache head
 *   weight(t) = decay * weight(t) + sum of p(t) over the queries and heads of its
 *   group
 * (with decay 0 the old weight is not read); sequences without queries keep
 * their weights.  Codes past a query's slot do not enter its result, NaN or
 * not; slots in unmapped blocks are not seen.  Scores, sums and weights are kept
 * in 32 bits (a weight errs by as much as a score and its row's log-sum do, 2^-23 of
 * them).
 * The most rows of a sequence (q_len times G) decide for the call how
 * probabilities and cached numbers enter the products.  Up to 64 (32 for head_dim
 * above 128) probabilities keep 16 bits, and cached numbers all of theirs whatever
 * the queries' type.  Beyond, both are rounded to the queries' type: half a step of
 * it for a probability; f16 takes numbers beyond it (of a cache rounded from bf16)
 * as its largest and the smallest as multiples of 2^-24.
 * head_dim at most 256 (DV_ERR_UNSUPPORTED); one layer's keys at most 64 GB.
 * Results do not depend on the order in which workgroups run.  q, the cache and
 * its table are not written; out, lse, workspace and weights must not overlap
 * them nor each other (q and out, lse, workspace are checked as one contiguous
 * range each only where the strides make them one).
 * DV_OK, DV_ERR_INVALID, DV_ERR_RANGE, DV_ERR_SPACE (workspace or rows too few),
 * DV_ERR_UNSUPPORTED, DV_ERR_HIP. */
DV_API int dv_attend(const dv_quant* c, int32_t mb, int32_t layer, const int32_t* q_len,
                     const int32_t* kv_len, const dv_attend_args* a, void* stream);

/* Keep min(len[b], keep[b]) of each head's len[b] tokens: the last `recent` of
 * them, and of the others those with the largest weight (ties: the lower slot;
 * NaN counts as less than any number), in slot order, in slots 0, 1, ... of
 * microbatch `dst_mb` of `dst`.  Each block of the result gets the scale that
 * dv_quant_in would give its tokens.  Weights and positions move along where
 * `dst` has those arrays (positions: the slots, where `src` has none).
 * kept: device int32 [l1 - l0][batch][head][kept_stride], the slots kept,
 * ascending; entries past a sequence's count are left as they are.
 * `src` needs its weight array.  `dst` may be `src` itself (the same microbatch
 * of the same arrays and layout: compaction in place) or another cache of the
 * same layers, heads, head_dim and batch, disjoint from it (one block table may
 * serve both).  Slots that an unmapped block leaves without codes count as zeros;
 * blocks that `dst` does not map are skipped.
 * DV_OK, DV_ERR_INVALID, DV_ERR_RANGE, DV_ERR_UNSUPPORTED, DV_ERR_HIP. */
DV_API int dv_evict(const dv_quant* src, int32_t src_mb, const dv_quant* dst, int32_t dst_mb,
                    int32_t l0, int32_t l1, const int32_t* len, const int32_t* keep,
                    int32_t recent, int32_t* kept, int32_t kept_stride, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* DV_ATTN_H */
