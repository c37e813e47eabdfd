// The validated view of a cache descriptor that every entry point starts from,
// and the checks they share (host code, no kernels here).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "../../include/dv.h"

namespace dv {

// A validated view of one microbatch of a cache, sizes in 16-byte units.
struct View {
  int kind;
  int mem;
  int64_t L, H, D, B, E;
  int64_t du;        // units per token
  int64_t cap;       // token capacity per sequence
  int64_t S;         // dense kinds: max_seq
  int64_t bs, NB, max_blocks;
  char* base;
  const int32_t* bt;
  int32_t* owner;    // paged: optional owner-map workspace [NB]
  uint64_t bytes;    // storage bytes of the microbatch
};

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// The layout of a descriptor, without a microbatch (sizing calls).
inline int layout_of(const dv_cache* c, View* v) {
  if (!c || !c->mb_base) return DV_ERR_INVALID;
  if (c->elem_bytes <= 0 || c->num_layers <= 0 || c->num_heads <= 0 || c->head_dim <= 0 ||
      c->batch <= 0 || c->num_mb <= 0)
    return DV_ERR_INVALID;
  if (((int64_t)c->head_dim * c->elem_bytes) % 16 != 0) return DV_ERR_INVALID;
  if (c->mem != DV_MEM_DEVICE && c->mem != DV_MEM_HOST_PINNED) return DV_ERR_INVALID;
  v->kind = c->kind;
  v->mem = c->mem;
  v->L = c->num_layers;
  v->H = c->num_heads;
  v->D = c->head_dim;
  v->B = c->batch;
  v->E = c->elem_bytes;
  v->du = v->D * v->E / 16;
  v->S = v->bs = v->NB = v->max_blocks = 0;
  v->bt = nullptr;
  v->owner = nullptr;
  if (c->kind == DV_DENSE || c->kind == DV_DENSE_KSPLIT) {
    if (c->max_seq <= 0) return DV_ERR_INVALID;
    v->S = v->cap = c->max_seq;
    v->bytes = (uint64_t)v->L * 2 * v->B * v->H * v->S * v->du * 16;
  } else if (c->kind == DV_PAGED) {
    if (c->block_size <= 0 || c->num_blocks <= 0 || c->max_blocks <= 0 || !c->block_table)
      return DV_ERR_INVALID;
    v->bs = c->block_size;
    v->NB = c->num_blocks;
    v->max_blocks = c->max_blocks;
    v->cap = v->bs * v->max_blocks;
    v->bytes = (uint64_t)v->L * 2 * v->NB * v->H * v->bs * v->du * 16;
  } else {
    return DV_ERR_INVALID;
  }
  // Extents whose products the kernels take in 32-bit arithmetic (a launch's
  // first slab index, 2 * layer + 1, among them).
  if (v->L > (1 << 24) || v->cap > (1 << 24) || v->du > (1 << 16) || v->H * v->du > (1 << 20) ||
      v->cap * v->du > (1ll << 30))
    return DV_ERR_UNSUPPORTED;
  // A paged tile may reach past a sequence's last block, and a unit's place in
  // the head's run is counted from the sequence's first: capacity and one block
  // together must stay well inside int32.
  if (c->kind == DV_PAGED && v->bs * v->du > (1ll << 29)) return DV_ERR_UNSUPPORTED;
  // Every byte count derived from the descriptor stays far inside 64 bits:
  // its storage and the longest stream it can produce (all layers, every
  // sequence at full capacity) must be below 2^48 bytes.
  using u128 = unsigned __int128;
  const u128 per_token = (u128)v->L * 2 * v->H * v->du * 16;
  const u128 rows = c->kind == DV_PAGED ? (u128)v->NB * v->bs : (u128)v->B * v->S;
  const u128 limit = (u128)1 << 48;
  if (per_token * rows >= limit || per_token * v->B * v->cap >= limit) return DV_ERR_UNSUPPORTED;
  v->base = nullptr;
  return DV_OK;
}

// The layout plus microbatch mb's base address (and table, owner map).
inline int view_of(const dv_cache* c, int32_t mb, View* v) {
  const int rc = layout_of(c, v);
  if (rc != DV_OK) return rc;
  if (mb < 0 || mb >= c->num_mb) return DV_ERR_RANGE;
  v->base = static_cast<char*>(c->mb_base[mb]);
  if (!v->base || !aligned16(v->base)) return DV_ERR_INVALID;
  if (c->kind == DV_PAGED) {
    v->bt = c->block_table[mb];
    if (!v->bt) return DV_ERR_INVALID;
    v->owner = c->block_owner ? c->block_owner[mb] : nullptr;
    if ((reinterpret_cast<uintptr_t>(v->owner) & 3u) != 0) return DV_ERR_INVALID;
  }
  return DV_OK;
}

inline bool overlaps(const void* a, uint64_t na, const void* b, uint64_t nb) {
  if (na == 0 || nb == 0) return false;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

// DV_ERR_HIP for a failed runtime call; with DV_DEBUG set in the environment
// the runtime's error name is also printed to stderr.
inline int hip_fail(hipError_t e, const char* what) {
  if (e == hipSuccess) return DV_OK;
  static const bool debug = getenv("DV_DEBUG") != nullptr;
  if (debug) fprintf(stderr, "libdv: %s failed: %s\n", what, hipGetErrorName(e));
  return DV_ERR_HIP;
}

// Whether [p, p + n) overlaps a paged view's block table, which the kernels
// read while the call writes: the table must stay out of everything written.
inline bool overlaps_table(const View& v, const void* p, uint64_t n) {
  return v.bt && overlaps(p, n, v.bt, (uint64_t)v.B * v.max_blocks * 4);
}

}  // namespace dv
