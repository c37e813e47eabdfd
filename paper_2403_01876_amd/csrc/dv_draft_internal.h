// Launch descriptors shared by the host side (dv_draft.cpp) and the kernels
// (dv_verify.hip, dv_draft.hip) of the operators over drafted tokens.
#pragma once

#include "dv_attn_internal.h"

namespace dv {

// ---- dv_verify ----
// A piece is kPiece logits of a row, counted from the 16-byte boundary at or below
// the row's start, so that all 16-byte loads are aligned.
constexpr int kPiece = 2048;
// What one piece of a row adds to its distribution.
struct PieceSum {
  double sum;   // of exp((x - top) / temperature); 1 for a piece of a greedy row
  float top;    // largest logit, -infinity for none
  int32_t arg;  // greedy: the lowest token that has it
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
  PieceSum* sums;    // [rows][pieces]
  double* left;      // [batch][pieces][2]: what the last row's pieces hold, and held before the
                     // last rejection
  int32_t* arrived;  // [batch]: workgroups that are done with their part of the last row
  int64_t logits_row, drawn_row;  // elements
  int32_t vocab, pieces, parts;   // parts: workgroups to a sequence
  int32_t type;
  int32_t b0, nseq, row0;         // sequences and rows before this launch's
  int32_t tok[kQSeqs + 1];        // rows of earlier sequences
  double scale2[kQSeqs];          // log2(e) / temperature; 0: greedy
};
static_assert(sizeof(VerifyArgs) <= 3584, "arguments stay under 4 KB");
hipError_t launch_verify_sums(const VerifyArgs& a, hipStream_t s);
hipError_t launch_verify_walk(const VerifyArgs& a, hipStream_t s);

// ---- dv_keep_path ----
// A wave takes one head of one sequence in one layer.
struct KeepArgs {
  QLayout q;
  const int32_t* path;   // advanced to this launch's first row
  const int32_t* count;  // and sequence
  int32_t l0, b0, nseq;
  FastDiv d_du, d_heads;
  int32_t base[kQSeqs];
  int32_t tok[kQSeqs + 1];  // rows of earlier sequences
};
static_assert(sizeof(KeepArgs) <= 3584, "arguments stay under 4 KB");
hipError_t launch_keep(const KeepArgs& a, uint32_t layers, hipStream_t s);

// ---- dv_quant_out ----
// Work items as of dv_quant_in; `held` 8-code units to a lane at a time.
hipError_t launch_quant_out(const QuantArgs& a, uint32_t nslabs, hipStream_t s);

}  // namespace dv
