// C-ABI entry points of the operators over drafted tokens, but for their attention:
// host-side validation and dispatch.  Everything is checked before the first launch.
#include <math.h>

#include "../../include/dv_draft.h"
#include "dv_draft_internal.h"
#include "dv_quant_view.h"

namespace {

using namespace dv;

// ---- dv_verify ------------------------------------------------------------------------------

struct VerifyPlan {
  int64_t rows, pieces;
  uint64_t sums, left, arrived, bytes;  // bytes of the workspace's parts
};

int plan_of(const int32_t* q_len, const dv_verify_args* a, VerifyPlan* p) {
  if (!q_len || !a) return DV_ERR_INVALID;
  if (a->type != DV_F16 && a->type != DV_BF16 && a->type != DV_F32) return DV_ERR_INVALID;
  if (a->vocab <= 0) return DV_ERR_INVALID;
  if (a->batch < 0) return DV_ERR_RANGE;
  if (a->vocab > 1 << 24) return DV_ERR_UNSUPPORTED;
  p->rows = 0;
  for (int32_t b = 0; b < a->batch; ++b) {
    if (q_len[b] < 0) return DV_ERR_RANGE;
    if (q_len[b] > kMaxDrafts) return DV_ERR_UNSUPPORTED;
    p->rows += q_len[b];
  }
  // (a row may begin up to seven numbers after the boundary that its pieces go by)
  p->pieces = ((int64_t)a->vocab + 7 + kPiece - 1) / kPiece;
  p->sums = (uint64_t)p->rows * p->pieces * sizeof(PieceSum);
  p->left = (uint64_t)a->batch * p->pieces * 16;
  p->arrived = (uint64_t)a->batch * 4;
  p->bytes = p->rows ? p->sums + p->left + p->arrived : 0;
  if (p->bytes >= 1ull << 31) return DV_ERR_UNSUPPORTED;
  return DV_OK;
}

int verify(const int32_t* q_len, const float* temperature, const dv_verify_args* u, void* stream) {
  VerifyPlan p;
  const int rc = plan_of(q_len, u, &p);
  if (rc != DV_OK) return rc;
  if (u->rows < 0) return DV_ERR_RANGE;
  for (int32_t b = 0; temperature && b < u->batch; ++b)
    if (!(temperature[b] >= 0.f) || isinf(temperature[b])) return DV_ERR_INVALID;
  if (u->rows < p.rows) return DV_ERR_SPACE;
  if (u->batch == 0) return DV_OK;
  const uint64_t n4 = (uint64_t)p.rows * 4, b4 = (uint64_t)u->batch * 4;
  if (!u->count || !aligned4(u->count)) return DV_ERR_INVALID;
  const int size = u->type == DV_F32 ? 4 : 2;
  uint64_t ln = 0, dn = 0;
  if (p.rows) {
    if (!u->logits || !u->parent || !u->token || !u->uniform || !u->path || !u->next ||
        !aligned4(u->parent) || !aligned4(u->token) || !aligned4(u->uniform) ||
        !aligned4(u->path) || !aligned4(u->next) || !aligned4(u->drawn) ||
        (reinterpret_cast<uintptr_t>(u->logits) & (size - 1)) || !aligned16(u->workspace))
      return DV_ERR_INVALID;
    // fewer than 2^27 rows (the workspace's limit): their bytes stay inside 64 bits
    const int64_t most = 1ll << 33;
    if (u->logits_row < u->vocab || u->logits_row > most) return DV_ERR_INVALID;
    if (u->drawn && (u->drawn_row < u->vocab || u->drawn_row > most)) return DV_ERR_INVALID;
    if (u->workspace_bytes < p.bytes) return DV_ERR_SPACE;
    if (!u->workspace) return DV_ERR_INVALID;
    ln = ((uint64_t)(p.rows - 1) * u->logits_row + u->vocab) * size;
    dn = u->drawn ? ((uint64_t)(p.rows - 1) * u->drawn_row + u->vocab) * 4 : 0;
    const void* const read[] = {u->logits, u->drawn, u->parent, u->token, u->uniform};
    const uint64_t read_bytes[] = {ln, dn, n4, n4, n4};
    const void* const written[] = {u->path, u->count, u->next, u->workspace};
    const uint64_t written_bytes[] = {n4, b4, b4, p.bytes};
    for (int i = 0; i < 4; ++i) {
      for (int j = 0; j < 5; ++j)
        if (overlaps(written[i], written_bytes[i], read[j], read_bytes[j])) return DV_ERR_INVALID;
      for (int j = 0; j < i; ++j)
        if (overlaps(written[i], written_bytes[i], written[j], written_bytes[j]))
          return DV_ERR_INVALID;
    }
  }

  hipStream_t st = static_cast<hipStream_t>(stream);
  char* w = static_cast<char*>(u->workspace);
  VerifyArgs a;
  memset(&a, 0, sizeof a);
  a.logits = u->logits;
  a.drawn = u->drawn;
  a.parent = u->parent;
  a.token = u->token;
  a.uniform = u->uniform;
  a.path = u->path;
  a.count = u->count;
  a.next = u->next;
  a.sums = reinterpret_cast<PieceSum*>(w);
  a.left = reinterpret_cast<double*>(w + p.sums);
  a.arrived = reinterpret_cast<int32_t*>(w + p.sums + p.left);
  a.logits_row = u->logits_row;
  a.drawn_row = u->drawn_row;
  a.vocab = u->vocab;
  a.pieces = (int32_t)p.pieces;
  a.type = u->type;
  int64_t row0 = 0;
  // as many sequences to a launch as its table and grids hold
  const int64_t seqs = std::min<int64_t>(kQSeqs, kMaxItems / (p.pieces * kMaxDrafts));
  for (int64_t b0 = 0; b0 < u->batch; b0 += seqs) {
    a.b0 = (int32_t)b0;
    a.nseq = (int32_t)std::min<int64_t>(seqs, u->batch - b0);
    a.row0 = (int32_t)row0;
    int32_t tok = 0;
    for (int i = 0; i <= kQSeqs; ++i) {
      a.tok[i] = tok;
      if (i >= a.nseq) continue;
      const float t = temperature ? temperature[b0 + i] : 1.f;
      a.scale2[i] = t == 0.f ? 0. : 1.4426950408889634074 / t;
      tok += q_len[b0 + i];
    }
    row0 += tok;
    // As many workgroups as there are CUs, as far as they have a piece each.  (32 sequences
    // of 16 pieces: chains 25.4 us in 8 parts, 26.3 in 16, 28.2 in 4.)
    a.parts = (int32_t)std::min<int64_t>(p.pieces, std::max<int64_t>(1, 256 / a.nseq));
    a.parts = (int32_t)((p.pieces + (p.pieces + a.parts - 1) / a.parts - 1) /
                        ((p.pieces + a.parts - 1) / a.parts));  // none without a piece
    hipError_t e = tok ? launch_verify_sums(a, st) : hipSuccess;
    if (e == hipSuccess) e = launch_verify_walk(a, st);
    if (e != hipSuccess) return hip_fail(e, "verification launch");
  }
  return DV_OK;
}

}  // namespace

extern "C" {

int dv_verify_bytes(const int32_t* q_len, const dv_verify_args* a, uint64_t* out_bytes) {
  VerifyPlan p;
  const int rc = plan_of(q_len, a, &p);
  if (rc != DV_OK) return rc;
  if (!out_bytes) return DV_ERR_INVALID;
  *out_bytes = p.bytes;
  return DV_OK;
}

int dv_verify(const int32_t* q_len, const float* temperature, const dv_verify_args* a,
              void* stream) {
  return verify(q_len, temperature, a, stream);
}

int dv_keep_path(const dv_quant* c, int32_t mb, int32_t l0, int32_t l1, const int32_t* q_len,
                 const int32_t* kv_len, const int32_t* path, const int32_t* count, void* stream) {
  Quant q;
  const int rc = quant_of(c, mb, &q);
  if (rc != DV_OK) return rc;
  const View& v = q.v;
  if (!q_len || !kv_len) return DV_ERR_INVALID;
  if (l0 < 0 || l1 < l0 || l1 > v.L) return DV_ERR_RANGE;
  int64_t rows = 0;
  for (int64_t b = 0; b < v.B; ++b) {
    if (q_len[b] < 0 || kv_len[b] < q_len[b] || kv_len[b] > v.cap) return DV_ERR_RANGE;
    if (q_len[b] > kMaxDrafts) return DV_ERR_UNSUPPORTED;
    rows += q_len[b];
  }
  if (rows == 0 || l1 == l0) return DV_OK;
  if (!path || !count || !aligned4(path) || !aligned4(count)) return DV_ERR_INVALID;
  if (tangled(q) || hits(q, path, rows * 4) || hits(q, count, (uint64_t)v.B * 4))
    return DV_ERR_INVALID;
  if (v.H >= kMaxItems) return DV_ERR_UNSUPPORTED;

  KeepArgs a;
  memset(&a, 0, sizeof a);
  a.q = layout_args(q);
  a.d_du = fast_div((uint32_t)(v.D / 16));
  a.d_heads = fast_div((uint32_t)v.H);
  const int64_t seqs = std::min<int64_t>(kQSeqs, kMaxItems / v.H);
  for (int32_t l = l0; l < l1; l += kLayers) {
    const int32_t nl = std::min(kLayers, l1 - l);
    a.l0 = l;
    int64_t row0 = 0;
    for (int64_t b0 = 0; b0 < v.B; b0 += seqs) {
      a.b0 = (int32_t)b0;
      a.nseq = (int32_t)std::min<int64_t>(seqs, v.B - b0);
      a.path = path + row0;
      a.count = count + b0;
      int32_t tok = 0;
      for (int i = 0; i < a.nseq; ++i) {
        a.base[i] = kv_len[b0 + i] - q_len[b0 + i];
        a.tok[i] = tok;
        tok += q_len[b0 + i];
      }
      a.tok[a.nseq] = tok;
      row0 += tok;
      if (tok == 0) continue;
      const hipError_t e = launch_keep(a, nl, static_cast<hipStream_t>(stream));
      if (e != hipSuccess) return hip_fail(e, "path launch");
    }
  }
  return DV_OK;
}

int dv_quant_out(const dv_quant* src, int32_t mb, int32_t l0, int32_t l1, const int32_t* t0,
                 const int32_t* t1, void* dst, uint64_t dst_cap, int32_t type,
                 uint64_t* out_bytes, void* stream) {
  Quant q;
  const int rc = quant_of(src, mb, &q);
  if (rc != DV_OK) return rc;
  const View& v = q.v;
  if (!t1 || (type != DV_F16 && type != DV_BF16)) return DV_ERR_INVALID;
  if (l0 < 0 || l1 < l0 || l1 > v.L) return DV_ERR_RANGE;
  int64_t N = 0, longest = 0;
  for (int64_t b = 0; b < v.B; ++b) {
    const int64_t a = t0 ? t0[b] : 0, e = t1[b];
    if (a < 0 || e < a || e > v.cap) return DV_ERR_RANGE;
    N += e - a;
    longest = std::max(longest, e - a);
    if (v.H * blocks_of(q, a, e) >= kMaxItems) return DV_ERR_UNSUPPORTED;
  }
  const uint64_t need = (uint64_t)(l1 - l0) * 2 * v.H * v.D * 2 * (uint64_t)N;
  if (out_bytes) *out_bytes = need;
  if (need > dst_cap) return DV_ERR_SPACE;
  if (need == 0) return DV_OK;
  if (!dst || !aligned16(dst) || hits(q, dst, need) || tangled(q)) return DV_ERR_INVALID;

  QuantArgs a;
  memset(&a, 0, sizeof a);
  a.q = layout_args(q);
  a.w_slab = v.H * v.D * 2 * N;
  a.bf16 = type == DV_BF16;
  // As few lanes to a block as read its 8-code units in one go of four each.
  const int64_t units = std::min<int64_t>(a.q.bs, longest) * v.D / 8;
  while (a.lanes_log2 < 6 && (4ll << a.lanes_log2) < units) ++a.lanes_log2;
  return by_launches(q, l0, l1, t0, t1, dst, a, [&](int32_t nl, const QuantArgs& x) {
    return launch_quant_out(x, 2 * nl, static_cast<hipStream_t>(stream));
  });
}

}  // extern "C"
