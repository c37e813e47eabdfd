// Launch descriptors shared by the host side (dv_attn.cpp) and the kernels
// (dv_quant.hip, dv_attend.hip, dv_evict.hip) of the 8-bit cache operators.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dv_internal.h"

namespace dv {

// Sequences of one launch: their tables travel in the kernel arguments (four
// int32 each, 3 KB in all).
constexpr int kQSeqs = 192;

// Where an 8-bit cache's codes (bytes) and scales (floats) lie.  Token t of
// (sequence b, head h) in slab = 2 * layer + half: block j = t / bs, blk = table
// entry j of b (paged) or j itself (dense);
//   code  slab * s_slab + b * s_b + blk * s_blk + h * s_h + (t % bs) * D
//   scale slab * c_slab + b * c_b + blk * c_blk + h * c_h
struct QLayout {
  uint8_t* codes;
  float* scale;
  const int32_t* bt;  // paged: [batch][max_blocks], else null
  float* weight;      // [layer][batch][head][cap] or null
  int32_t* position;
  int64_t s_slab, s_b, s_blk, s_h;
  int64_t c_slab, c_b, c_blk, c_h;
  int32_t bs, D, heads, batch;
  int32_t num_blocks, max_blocks;
  int32_t cap;
  FastDiv d_bs;
};

// ---- dv_quant_in ----
// A work item is one block of one head of one sequence; item[] counts those of
// earlier sequences.  A group of 1 << lanes_log2 lanes takes an item, and each of
// them holds `held` (2 or 4) units of 16 elements in registers.
struct QuantArgs {
  QLayout q;
  const uint8_t* wire;  // advanced to this launch's first sequence
  int64_t w_slab;       // wire bytes per slab (layer, half)
  int32_t slab0, b0, nseq, items;
  int32_t lanes_log2, held, bf16;
  int32_t item[kQSeqs];     // INT32_MAX past the last
  int32_t tok[kQSeqs + 1];  // tokens of earlier sequences
  int32_t t0[kQSeqs];
};
static_assert(sizeof(QuantArgs) <= 3584, "arguments stay under 4 KB");
hipError_t launch_quant(const QuantArgs& a, uint32_t nslabs, hipStream_t s);

// ---- dv_attend ----
// Queries of a sequence and the heads of a group are rows r = i * G + g.
struct AttendArgs {
  QLayout q;
  const void* query;
  void* out;
  int64_t q_token, q_head, o_token, o_head;  // elements
  const float* slopes;
  float* lse;
  float* part;    // splits: [item][R rows][Dp], sums of a work item's rows
  float* ml;      // splits: [item][R rows][2], their reference and sum
  float* scores;  // weigh, split rows: [sequence][head][row][padded tokens], log2 units
  float* row_lse; // weigh, many rows: [row of the call][q_heads], log2 units
  float* sums;    // weigh, many rows in shares: [share][item][kWeighTokens]
  float scale2;   // scale * log2 e
  float decay;
  int32_t layer, b0, nseq, items;
  int32_t G, q_heads, chunk;  // chunk: tokens of a split
  int32_t weigh, bf16, row0;  // row0: rows of q before this launch's
  FastDiv d_G;
  int32_t nt;                 // whether the codes are read past the caches
  int32_t item[kQSeqs];       // work items of earlier sequences; INT32_MAX past the last
  int32_t tok[kQSeqs + 1];    // queries of earlier sequences
  int32_t len[kQSeqs];        // tokens in the cache
  int32_t soff[kQSeqs];       // scores of earlier sequences, in 32 floats
};
static_assert(sizeof(AttendArgs) <= 3800, "arguments stay under 4 KB");
// Few rows: RT tiles of 16 rows (1, 2, 4), the token axis split into chunks of
// a.chunk tokens; `direct`: one chunk a sequence, results go straight to out.
// head_dim as the kernels are built for it.
inline int padded(int64_t D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }
// Tokens of a wave's step over the cache, and of a workgroup's (four waves).
constexpr int kSplitStep = 32;
constexpr int kSplitRound = 4 * kSplitStep;
constexpr int kSplitChunkMax = 1792;  // its tables take 28 KB of LDS at most
// Bytes of LDS for the queries of the split kernel: those of four tiles leave no
// registers for two workgroups a CU.
constexpr int split_queries(int DP, int RT) { return RT == 4 ? RT * DP * 32 : 0; }
// Workgroups of the split kernel that the registers of RT tiles of results allow
// a CU, its bytes of LDS (the codes of a step of four waves and the tables of a
// chunk, or the waves' results) and those that both allow.
constexpr int split_waves(int DP, int RT) {
  return DP <= 64 ? (RT == 1 ? 4 : RT == 2 ? 3 : 2) : DP <= 128 ? (RT == 1 ? 3 : 2) : RT == 1 ? 2 : 1;
}
inline size_t split_lds(int DP, int rt, int chunk, bool slopes) {
  const size_t tables = (size_t)4 * 2 * kSplitStep * DP + split_queries(DP, rt) +
                        (size_t)chunk * (slopes ? 16 : 12) + rt * 256 + 16;
  const size_t join = (size_t)4 * 16 * DP * 4 + (size_t)4 * rt * 16 * 8 + 32;
  return tables > join ? tables : join;
}
inline int split_groups(int DP, int rt, int chunk, bool slopes) {
  const int by_lds = (int)(160 * 1024 / split_lds(DP, rt, chunk, slopes));
  return by_lds < split_waves(DP, rt) ? by_lds : split_waves(DP, rt);
}
hipError_t launch_attend_split(const AttendArgs& a, int rt, bool direct, hipStream_t s);
hipError_t launch_attend_join(const AttendArgs& a, int rows, hipStream_t s);
// Many rows: tiles of kTileRows rows.
constexpr int kTileRows = 128;
constexpr int tile_waves(int DP) { return DP <= 128 ? 2 : 1; }  // workgroups a CU
hipError_t launch_attend_tile(const AttendArgs& a, bool direct, hipStream_t s);
// Column sums of the probabilities, from the rows' lse.
constexpr int kWeighTokens = 128;
constexpr int weigh_waves(int DP) { return DP <= 128 ? 3 : 1; }  // workgroups a CU
hipError_t launch_attend_weigh(const AttendArgs& a, int shares, hipStream_t s);

// ---- dv_evict ----
// A work item is a group of `group` blocks of the result of one head of one
// sequence, or in place all of them; item[] counts those of earlier sequences.
struct EvictArgs {
  QLayout s, d;
  int32_t* kept;
  int32_t kept_stride, recent, l0, nl;
  int32_t b0, nseq, in_place, most;  // most: tokens of the longest sequence
  int32_t blocks, group, items;  // blocks: most result blocks of a sequence
  FastDiv d_du;                       // by 16-code units of a token
  int32_t len[kQSeqs];
  int32_t keep[kQSeqs];
  int32_t item[kQSeqs];  // INT32_MAX past the last
};
static_assert(sizeof(EvictArgs) <= 3584, "arguments stay under 4 KB");
// Lanes of a workgroup that selects (a head of a sequence): see the kernel.
inline int evict_select_lanes(int most) { return most > 16 * 256 ? 1024 : 256; }
hipError_t launch_evict_select(const EvictArgs& a, hipStream_t s);
hipError_t launch_evict_move(const EvictArgs& a, hipStream_t s);

}  // namespace dv
