/* dv_draft.h -- a decode step with drafted tokens over an 8-bit KV cache, for one
 * MI355X (gfx950):
 *
 *   dv_attend_tree  one layer's attention of drafted tokens that branch;
 *   dv_verify       which of them the target model accepts, and what follows;
 *   dv_keep_path    the accepted ones' keys and values move together;
 *   dv_quant_out    cached tokens come back as a 16-bit stream.
 *
 * The conventions of dv.h and dv_attn.h hold: arguments are checked on the host
 * before anything is enqueued, the caller owns every buffer, nothing is allocated,
 * work is enqueued on `stream`, host arrays are read during the call only.
 *
 * Drafts.  Sequence b holds kv_len[b] tokens, of which the last q_len[b], at most
 * DV_MAX_DRAFTS, are its drafts: draft i stands in slot base + i, base =
 * kv_len[b] - q_len[b] >= 0 (appended there by dv_quant_in).  Arrays over drafts
 * have a row for each, those of sequence b from row sum_{b' < b} q_len[b'] on.
 * parent[row of draft i] (device int32) is the draft that draft i follows, below i;
 * -1 where it follows the tokens before the drafts.  Any other value, on the way up
 * too, takes a draft out: it is not there.  A draft's line is itself and all drafts that
 * it follows; its depth is how many it follows, 0 of draft 0.
 * A step: draft 0 is the last token that was sampled, not yet in the cache before,
 * and the others guess on from it.
 */
#ifndef DV_DRAFT_H
#define DV_DRAFT_H

#include "dv_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define DV_MAX_DRAFTS 128 /* of a sequence */

/* dv_attend with drafts in place of consecutive queries.  Draft i sees the slots
 * before base and those of its line; one that is not there sees nothing (zeros and
 * lse -infinity).  Its position is that of slot base - 1 (the companion array's, or
 * the slot; -1 where base is 0) + 1 + its depth, as a query's and as a key's:
 *   score(t) = scale * q.k(t) + slope * (position(t) - position(i))
 * The companion's entries for the drafts' own slots are not read.  Everything else
 * is as in dv_attend, its workspace (dv_attend_bytes of the same lengths) and the
 * rounding of probabilities among it, but `weigh` has to be 0: drafts that are not
 * accepted would count.  parent: 4-byte aligned, [rows]; it must not overlap out,
 * lse or workspace.
 * DV_OK, DV_ERR_INVALID, DV_ERR_RANGE, DV_ERR_SPACE, DV_ERR_UNSUPPORTED (`weigh`,
 * too many drafts), DV_ERR_HIP. */
DV_API int dv_attend_tree(const dv_quant* c, int32_t mb, int32_t layer, const int32_t* q_len,
                          const int32_t* kv_len, const int32_t* parent, const dv_attend_args* a,
                          void* stream);

/* Type of 32-bit logits, beside dv_type's. */
#define DV_F32 2

typedef struct dv_verify_args {
  int32_t type;          /* of the logits: DV_F16, DV_BF16 or DV_F32 */
  int32_t batch;         /* sequences */
  int32_t vocab;         /* tokens, at most 2^24 */
  int32_t rows;          /* that the arrays over drafts have: at least the sum of q_len */
  const void* logits;    /* device [rows][logits_row]: the target's, of what follows each draft */
  int64_t logits_row;    /* elements from row to row, at least vocab, at most 2^33 */
  const float* drawn;    /* device [rows][drawn_row], or NULL: the distribution that the drafts
                            which follow this one were drawn from */
  int64_t drawn_row;
  const int32_t* parent; /* device [rows] */
  const int32_t* token;  /* device [rows]: each draft's token (draft 0's is not read) */
  const float* uniform;  /* device [rows]: random numbers of [0, 1) */
  int32_t* path;         /* device [rows]: the drafts accepted, ascending, from the sequence's
                            first row on; entries past their count are left as they are */
  int32_t* count;        /* device [batch]: how many */
  int32_t* next;         /* device [batch]: the token that follows the last of them */
  void* workspace;       /* device, 16-byte aligned, dv_verify_bytes of it */
  uint64_t workspace_bytes;
} dv_verify_args;

/* Workspace bytes of a dv_verify with these lengths; goes by a->type, batch, vocab and
 * whether a->drawn is NULL only.  Host-only. */
DV_API int dv_verify_bytes(const int32_t* q_len, const dv_verify_args* a, uint64_t* out_bytes);

/* Accept drafts so that what is accepted, and the token after it, are distributed as
 * the target's own samples.  With p(i) the target's distribution after draft i,
 *   p(i)(x) = exp(logits[i][x] / temperature[b]) / their sum,
 * or where the temperature is 0, 1 for the largest logit (ties: the lowest token):
 * accept draft 0; r = p(0).  Then each draft i in order that follows the draft
 * accepted last (a), x = token[i]:
 *   drawn:     accept it where uniform[i] * drawn[a][x] < r(x);
 *              else r becomes max(r - drawn[a], 0) over its sum
 *   not drawn: accept it where uniform[i] < r(x);
 *              else r(x) becomes 0, and r is divided by its sum, however little that is
 * (r stays as it is where that leaves nothing), and where it was accepted r = p(i).
 * At the end next is the lowest token y with r(0) + ... + r(y) above uniform[0].
 * Drafts that follow one draft have to be drawn from drawn[a] independently, the same
 * token twice if it comes so: of siblings drawn without replacement what is accepted is
 * not distributed as the target's samples.  Drafts that were not drawn may be any tokens
 * that do not depend on `uniform`.  A sibling that is tried after a drawn one was refused
 * takes a pass over the row, the longer the more were refused.
 * All of it is decided as by sums in 64 bits.  A logit that is NaN counts as -infinity;
 * infinite ones share all probability.  Draft 0 is there whatever its parent; any other
 * with a token outside [0, vocab), or that is not there, is passed over.  drawn[i][x]
 * counts as 0 where it is negative or NaN.  A row whose logits are all -infinity accepts
 * nothing; next is then -1.  A probability below 2^-1020 of the row's largest counts as 0.
 * A number outside [0, 1) counts as the nearest end (1: the last token that r holds), NaN
 * as 1.
 * A sequence without drafts gets count 0 and its next is left as it is.
 * temperature: host [batch], finite, 0 or more; NULL: all 1.  What the call writes
 * must not overlap what it reads nor each other.
 * DV_OK, DV_ERR_INVALID, DV_ERR_RANGE (q_len, rows or batch below 0),
 * DV_ERR_SPACE (workspace or rows too few), DV_ERR_UNSUPPORTED (more than
 * DV_MAX_DRAFTS, 2^24 tokens, or 2^31 bytes of workspace), DV_ERR_HIP. */
DV_API int dv_verify(const int32_t* q_len, const float* temperature, const dv_verify_args* a,
                     void* stream);

/* Keep of every sequence's drafts those that `path` names (as dv_verify gives them)
 * and move them to slots base, base + 1, ... of microbatch `mb` of `c`, layers
 * [l0, l1): what dv_quant_in does with the numbers that they stand for, in place.
 * Blocks that hold tokens from before base keep the larger of their scale and the
 * kept ones' need (also where only the append of rejected drafts had raised it), others
 * get what their kept tokens need.  path: device int32 [rows], count: device int32
 * [batch].  A path ends before its first entry that is not above the one before it, not
 * below q_len[b] or negative, or after count[b].
 * Weights move along; positions stay, since a slot's is that of the token which
 * dv_quant_in would append there.  Slots past the kept ones hold nothing.  Tokens
 * of an unmapped block count as zeros; blocks that are not mapped are skipped.
 * path and count must not overlap the cache.
 * DV_OK, DV_ERR_INVALID, DV_ERR_RANGE, DV_ERR_UNSUPPORTED (more than
 * DV_MAX_DRAFTS), DV_ERR_HIP. */
DV_API int dv_keep_path(const dv_quant* c, int32_t mb, int32_t l0, int32_t l1,
                        const int32_t* q_len, const int32_t* kv_len, const int32_t* path,
                        const int32_t* count, void* stream);

/* dv_quant_in's way back: tokens [t0[b], t1[b]) of every sequence, layers [l0, l1), of
 * microbatch `mb` of `src` as the wire of these ranges with 2-byte elements of
 * `type` (t0 may be NULL: all zero), into `dst` (device, 16-byte aligned) of `dst_cap`
 * bytes.
 * Each element is its code times its scale, to the nearest (ties to even; exact but
 * for f16's multiples of 2^-24); beyond the type's largest number it is that, NaN is
 * NaN.  On return *out_bytes (if not NULL) holds the wire's size, also on
 * DV_ERR_SPACE.  Wire bytes of tokens without a block are left unwritten.  `dst` must
 * not overlap the cache, its table, scales or companions.
 * DV_OK, DV_ERR_INVALID, DV_ERR_RANGE, DV_ERR_SPACE, DV_ERR_UNSUPPORTED, DV_ERR_HIP. */
DV_API int dv_quant_out(const dv_quant* src, int32_t mb, int32_t l0, int32_t l1,
                        const int32_t* t0, const int32_t* t1, void* dst, uint64_t dst_cap,
                        int32_t type, uint64_t* out_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* DV_DRAFT_H */
