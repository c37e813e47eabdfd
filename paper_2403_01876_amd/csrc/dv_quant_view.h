// The validated view of an 8-bit cache that every operator over one starts from,
// and the checks they share (host code, no kernels here).
#pragma once

#include <string.h>

#include <algorithm>

#include "../../include/dv_attn.h"
#include "dv_attn_internal.h"
#include "dv_view.h"

namespace dv {

// Layers of a launch that takes several (two rows of the grid each),
// and work items of any: a grid's lanes are counted in 32 bits.
constexpr int32_t kLayers = 16384;
constexpr int64_t kMaxItems = 1 << 23;

inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// A validated 8-bit cache; addresses only where a microbatch was named.
struct Quant {
  View v;
  int64_t sb, nb;  // tokens of a scale, scales of a dense head
  uint64_t scale_bytes, slot_bytes;
  float* scale;
  float* weight;
  int32_t* position;
};

inline int layout8(const dv_quant* c, Quant* q) {
  if (!c || !c->cache) return DV_ERR_INVALID;
  const int rc = layout_of(c->cache, &q->v);
  if (rc != DV_OK) return rc;
  const View& v = q->v;
  if (v.E != 1 || v.mem != DV_MEM_DEVICE || c->scale_block <= 0) return DV_ERR_INVALID;
  if (v.kind == DV_DENSE_KSPLIT) return DV_ERR_UNSUPPORTED;
  if (v.kind == DV_PAGED && c->scale_block != v.bs) return DV_ERR_INVALID;
  if (v.kind == DV_PAGED && (uint64_t)v.NB * v.H * v.bs * v.D >= (1ull << 36))
    return DV_ERR_UNSUPPORTED;  // a token's row is counted in 32 bits of 16 bytes
  q->sb = c->scale_block;
  q->nb = (v.cap + q->sb - 1) / q->sb;
  q->scale_bytes = (uint64_t)v.L * 2 * v.H * 4 * (v.kind == DV_PAGED ? v.NB : v.B * q->nb);
  q->slot_bytes = (uint64_t)v.L * v.B * v.H * v.cap * 4;
  q->scale = nullptr;
  q->weight = nullptr;
  q->position = nullptr;
  return DV_OK;
}

inline int quant_of(const dv_quant* c, int32_t mb, Quant* q) {
  int rc = layout8(c, q);
  if (rc != DV_OK) return rc;
  rc = view_of(c->cache, mb, &q->v);
  if (rc != DV_OK) return rc;
  if (!c->scale || !c->scale[mb]) return DV_ERR_INVALID;
  q->scale = c->scale[mb];
  q->weight = c->weight ? c->weight[mb] : nullptr;
  q->position = c->position ? c->position[mb] : nullptr;
  if (!aligned4(q->scale) || !aligned4(q->weight) || !aligned4(q->position))
    return DV_ERR_INVALID;
  return DV_OK;
}

inline uint64_t held(const void* p, uint64_t n) { return p ? n : 0; }

// Whether [p, p + n) overlaps anything of the cache but its table.
inline bool hits_arrays(const Quant& q, const void* p, uint64_t n) {
  return overlaps(p, n, q.v.base, q.v.bytes) || overlaps(p, n, q.scale, q.scale_bytes) ||
         overlaps(p, n, q.weight, held(q.weight, q.slot_bytes)) ||
         overlaps(p, n, q.position, held(q.position, q.slot_bytes));
}

// Whether [p, p + n) overlaps anything of the cache.
inline bool hits(const Quant& q, const void* p, uint64_t n) {
  return hits_arrays(q, p, n) || overlaps_table(q.v, p, n);
}

// Whether two caches overlap, other than by tables, which calls only read.
inline bool hits(const Quant& a, const Quant& b) {
  return hits(a, b.v.base, b.v.bytes) || hits(a, b.scale, b.scale_bytes) ||
         hits(a, b.weight, held(b.weight, b.slot_bytes)) ||
         hits(a, b.position, held(b.position, b.slot_bytes)) ||
         (b.v.bt && hits_arrays(a, b.v.bt, (uint64_t)b.v.B * b.v.max_blocks * 4));
}

// A cache whose own parts overlap.
inline bool tangled(const Quant& q) {
  const uint64_t w = held(q.weight, q.slot_bytes), p = held(q.position, q.slot_bytes);
  const View& v = q.v;
  return overlaps(q.scale, q.scale_bytes, v.base, v.bytes) ||
         overlaps(q.weight, w, v.base, v.bytes) || overlaps(q.position, p, v.base, v.bytes) ||
         overlaps(q.weight, w, q.scale, q.scale_bytes) ||
         overlaps(q.position, p, q.scale, q.scale_bytes) ||
         overlaps(q.weight, w, q.position, p) || overlaps_table(v, v.base, v.bytes) ||
         overlaps_table(v, q.scale, q.scale_bytes) || overlaps_table(v, q.weight, w) ||
         overlaps_table(v, q.position, p);
}

inline QLayout layout_args(const Quant& q) {
  const View& v = q.v;
  QLayout a;
  memset(&a, 0, sizeof a);
  a.codes = reinterpret_cast<uint8_t*>(v.base);
  a.scale = q.scale;
  a.weight = q.weight;
  a.position = q.position;
  a.bs = (int32_t)std::min<int64_t>(q.sb, v.cap);
  a.D = (int32_t)v.D;
  a.heads = (int32_t)v.H;
  a.batch = (int32_t)v.B;
  a.cap = (int32_t)v.cap;
  a.d_bs = fast_div((uint32_t)a.bs);
  a.s_blk = a.bs * v.D;
  if (v.kind == DV_PAGED) {
    a.bt = v.bt;
    a.num_blocks = (int32_t)v.NB;
    a.max_blocks = (int32_t)v.max_blocks;
    a.s_h = v.bs * v.D;
    a.s_blk = v.H * a.s_h;
    a.s_slab = v.NB * a.s_blk;
    a.c_h = 1;
    a.c_blk = v.H;
    a.c_slab = v.NB * v.H;
  } else {
    a.s_h = v.S * v.D;
    a.s_b = v.H * a.s_h;
    a.s_slab = v.B * a.s_b;
    a.c_blk = 1;
    a.c_h = q.nb;
    a.c_b = v.H * q.nb;
    a.c_slab = v.B * a.c_b;
  }
  return a;
}

inline int64_t blocks_of(const Quant& q, int64_t t0, int64_t t1) {
  return t1 > t0 ? (t1 + q.sb - 1) / q.sb - t0 / q.sb : 0;
}

// Tokens [t0, t1) of layers [l0, l1) of a wire at `wire`, as many layers and sequences
// to a launch as its table and grid hold: launch(layers, a) with a's tables filled.
template <typename Launch>
int by_launches(const Quant& q, int32_t l0, int32_t l1, const int32_t* t0, const int32_t* t1,
                const void* wire, QuantArgs a, Launch launch) {
  const View& v = q.v;
  for (int32_t l = l0; l < l1; l += kLayers) {
    const int32_t nl = std::min(kLayers, l1 - l);
    int64_t tok = 0;
    for (int64_t b = 0; b < v.B;) {
      const int64_t b0 = b, first = tok;
      int64_t items = 0;
      int n = 0;
      for (; b < v.B && n < kQSeqs; ++b, ++n) {
        const int64_t s = t0 ? t0[b] : 0, e = t1[b], more = v.H * blocks_of(q, s, e);
        if (items + more >= kMaxItems) break;
        a.item[n] = (int32_t)items;
        a.tok[n] = (int32_t)(tok - first);
        a.t0[n] = (int32_t)s;
        items += more;
        tok += e - s;
        if (tok - first >= (1ll << 30)) { ++b; ++n; break; }
      }
      a.tok[n] = (int32_t)(tok - first);
      a.nseq = n;
      a.b0 = (int32_t)b0;
      a.items = (int32_t)items;
      a.slab0 = 2 * l;
      a.wire = static_cast<const uint8_t*>(wire) + (uint64_t)(l - l0) * 2 * a.w_slab +
               (uint64_t)first * v.H * v.D * 2;
      if (items == 0) continue;
      const hipError_t e = launch(nl, a);
      if (e != hipSuccess) return hip_fail(e, "stream launch");
    }
  }
  return DV_OK;
}

}  // namespace dv
