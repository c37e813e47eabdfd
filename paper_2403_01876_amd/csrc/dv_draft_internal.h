// Launch descriptors shared by the host side (dv_draft.cpp) and the kernels
// (dv_verify.hip, dv_draft.hip) of the operators over drafted tokens.
#pragma once

#include "dv_attn_internal.h"

namespace dv {

// ---- dv_verify ----
// A piece is kPiece logits of a row, counted from the 16-byte boundary at or below
// the row's start, so that every lane's 16-byte loads are aligned.
constexpr int kPiece = 4096;
// What one piece of a row adds to its distribution.
struct PieceSum {
  double sum;   // of exp((x - top) / temperature), or 1 for a piece of a greedy row
  float top;    // largest logit, -infinity for none
  int32_t arg;  // the lowest token that has it
};
// What the walk leaves of a sequence for its last token to be sampled from.
struct Final {
  double total;     // the row's sum relative to top
  float top;        // the row's largest logit
  int32_t arg;      // and its lowest token
  int32_t row;      // in the call
  int32_t rejected; // drafts that were not accepted there; -1: nothing to sample
  int32_t arrived;  // pieces whose sums are written
  int32_t pad;
};
struct VerifyArgs {
  const void* logits;
  const float* drawn;
  const int32_t* parent;
  const int32_t* token;
  const float* uniform;
  int32_t* path;
  int32_t* count;
  int32_t* next;
  PieceSum* sums;   // [rows][pieces]
  Final* finals;    // [batch]
  double* turns;    // [rows]: not drawn: a sequence's rejected tokens (as numbers); drawn: the
                    // sums that its residuals were divided by
  double* left;     // [batch][pieces][2]: what the last row's pieces hold, and held before the
                    // last rejection
  int64_t logits_row, drawn_row;  // elements
  int32_t vocab, pieces, type;
  int32_t b0, nseq, row0;         // sequences and rows before this launch's
  int32_t tok[kQSeqs + 1];        // rows of earlier sequences
  double scale2[kQSeqs];          // log2(e) / temperature; 0: greedy
};
static_assert(sizeof(VerifyArgs) <= 3584, "arguments stay under 4 KB");
hipError_t launch_verify_sums(const VerifyArgs& a, hipStream_t s);
hipError_t launch_verify_walk(const VerifyArgs& a, hipStream_t s);
hipError_t launch_verify_next(const VerifyArgs& a, hipStream_t s);

// ---- dv_keep_path ----
// A wave takes one head of one sequence in one slab.
struct KeepArgs {
  QLayout q;
  const int32_t* path;   // advanced to this launch's first row
  const int32_t* count;  // and sequence
  int32_t slab0, b0, nseq;
  FastDiv d_du, d_heads;
  int32_t base[kQSeqs];
  int32_t tok[kQSeqs + 1];  // rows of earlier sequences
};
static_assert(sizeof(KeepArgs) <= 3584, "arguments stay under 4 KB");
hipError_t launch_keep(const KeepArgs& a, uint32_t nslabs, hipStream_t s);

// ---- dv_quant_out ----
// Work items as of dv_quant_in; `held` 8-code units to a lane at a time.
hipError_t launch_quant_out(const QuantArgs& a, uint32_t nslabs, hipStream_t s);

}  // namespace dv
