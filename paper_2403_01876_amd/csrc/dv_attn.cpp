// C-ABI entry points of the 8-bit cache operators: host-side validation and
// dispatch.  Everything is checked before the first launch.
#include "../../include/dv_draft.h"
#include "dv_quant_view.h"

namespace {

using namespace dv;

// ---- dv_attend ------------------------------------------------------------------------------

// Rows (queries and heads of a group) up to which the split kernel takes a call,
// the second for head_dim above 128: as many as its registers hold, since it is
// faster up to there.  16 sequences of 128 to 4096 tokens, 8 heads: 16 rows 24.5 us
// instead of 50.7, 64 rows 45 instead of 57; head_dim 256, 4 heads, 32 rows 35
// instead of 80.
constexpr int64_t kFewRows = 64, kFewRowsWide = 32;

// How a call's work is divided, and its workspace.
struct Plan {
  bool split;      // few rows: the split kernel, R = 16, 32 or 64 rows
  bool direct;     // no joining
  int R;
  int32_t chunk;   // tokens of a split
  int64_t Dp;
  int64_t most;    // rows of the longest sequence
  uint64_t part, ml, scores, lse, sums, bytes;  // bytes of the workspace's parts
};

uint64_t up256(uint64_t n) { return (n + 255) & ~255ull; }

// Shares of the rows that each of `items` work items of the weights is dealt in:
// as many as the card holds at once, with 256 rows or more.
int shares_of(const Plan& p, int64_t items) {
  const int64_t slots = 256 * dv::weigh_waves((int)p.Dp);
  return (int)std::max<int64_t>(1, std::min(slots / std::max<int64_t>(1, items), p.most / 256));
}

int64_t splits_of(const Plan& p, int64_t len) {
  return std::max<int64_t>(1, (len + p.chunk - 1) / p.chunk);
}

int plan_of(const Quant& q, const int32_t* q_len, const int32_t* kv_len, const dv_attend_args* a,
            Plan* p) {
  const View& v = q.v;
  if (!q_len || !kv_len || !a) return DV_ERR_INVALID;
  if (a->type != DV_F16 && a->type != DV_BF16) return DV_ERR_INVALID;
  if (a->q_heads <= 0 || a->q_heads % v.H != 0) return DV_ERR_INVALID;
  if (v.D > 256 || a->q_heads > (1 << 20)) return DV_ERR_UNSUPPORTED;
  const int64_t G = a->q_heads / v.H;
  int64_t most = 0, tokens = 0, total = 0, longest = 0;
  for (int64_t b = 0; b < v.B; ++b) {
    const int64_t n = q_len[b], len = kv_len[b];
    if (n < 0 || n > (1 << 24) || len < 0 || len > v.cap) return DV_ERR_RANGE;
    if (n == 0) continue;
    most = std::max(most, n * G);
    tokens += n;
    total += len * v.H;
    longest = std::max(longest, len);
  }
  // rows are counted in 32 bits
  if (most >= (1ll << 30) || tokens * a->q_heads >= (1ll << 31)) return DV_ERR_UNSUPPORTED;
  p->Dp = dv::padded(v.D);
  p->most = most;
  p->split = most <= (p->Dp == 256 ? kFewRowsWide : kFewRows);
  if (p->split) {
    p->R = most <= 16 ? 16 : most <= 32 ? 32 : 64;
    // The smallest chunk whose work items the card holds all at once: 32 sequences
    // of 128 to 4096 tokens, 8 heads 32 us; half as many items 38.8, 1.5, 2 and 3
    // times as many 39.4, 35.4 and 40.6.
    const int64_t round = dv::kSplitRound;
    uint32_t chunk = (uint32_t)(std::max<int64_t>(1, total / 1024 / round) * round);
    for (; chunk < dv::kSplitChunkMax; chunk += round) {
      uint32_t splits = 0;
      for (int64_t b = 0; b < v.B; ++b)
        if (q_len[b] > 0) splits += kv_len[b] ? ((uint32_t)kv_len[b] + chunk - 1) / chunk : 1;
      if (splits * v.H <=
          256 * dv::split_groups((int)p->Dp, p->R / 16, (int)chunk, a->slopes != nullptr))
        break;
    }
    // (Up to two rounds of four waves are not worth joining: 250 tokens 9.7 us,
    // joined 11.7; 400 tokens in one chunk 13.1, joined 12.4.)
    int64_t most_split = longest <= 2 * round ? (longest + round - 1) / round * round : 0;
    most_split = std::max<int64_t>(std::max<int64_t>(most_split, chunk), round);
    p->chunk = (int32_t)std::min<int64_t>(most_split, dv::kSplitChunkMax);
  } else {
    p->R = dv::kTileRows;
    // The longest sequence in as many parts, of 256 tokens or more, as leave all
    // work items at once on the card: 4000 tokens under 8 tiles of 8 heads 42.5 us
    // in eight parts, 75 in four, 127 in one; under 32 tiles 104 in two, 128 in
    // one; but under 50 tiles 166 in one, 187 in three and 276 in two uneven ones.
    // (Up to 512 tokens are not worth joining: 500 tokens 24 us, in two parts 29.)
    const int64_t slots = 256 * dv::tile_waves((int)p->Dp);
    const auto tiles = [&](int64_t b) { return (q_len[b] * G + p->R - 1) / p->R * v.H; };
    const auto chunk_of = [&](int64_t n) {
      return std::max<int64_t>(64, ((longest + n - 1) / n + 63) / 64 * 64);
    };
    const auto items = [&](int64_t chunk) {
      int64_t sum = 0;
      for (int64_t b = 0; b < v.B; ++b)
        sum += tiles(b) * std::max<int64_t>(1, (kv_len[b] + chunk - 1) / chunk);
      return sum;
    };
    int64_t work = 0;
    for (int64_t b = 0; b < v.B; ++b) work += tiles(b) * kv_len[b];
    int64_t n = longest <= 512 ? 1 : (longest + 255) / 256;
    n = std::min(n, longest * slots / std::max<int64_t>(1, work));
    while (n > 1 && items(chunk_of(n)) > slots) --n;
    p->chunk = (int32_t)chunk_of(std::max<int64_t>(1, n));
  }
  p->direct = longest <= p->chunk;
  // Workspace of the largest launch; they run one after another.
  p->part = p->ml = p->scores = p->lse = p->sums = 0;
  for (int64_t b0 = 0; b0 < v.B; b0 += kQSeqs) {
    uint64_t items = 0, scores = 0, rows = 0;
    int64_t weigh_items = 0;
    for (int64_t b = b0; b < std::min<int64_t>(b0 + kQSeqs, v.B); ++b) {
      if (q_len[b] == 0) continue;
      const int64_t r = q_len[b] * G, len = kv_len[b];
      items += (r + p->R - 1) / p->R * v.H * splits_of(*p, len);
      scores += (uint64_t)r * v.H * ((len + 31) / 32);
      rows += (uint64_t)r * v.H;
      weigh_items += v.H * ((len + dv::kWeighTokens - 1) / dv::kWeighTokens);
    }
    if (items >= (uint64_t)kMaxItems || weigh_items >= kMaxItems) return DV_ERR_UNSUPPORTED;
    if (p->split && a->weigh && scores >= (1ull << 31)) return DV_ERR_UNSUPPORTED;
    if (!p->direct) {
      p->part = std::max(p->part, up256(items * p->R * p->Dp * 4));
      p->ml = std::max(p->ml, up256(items * p->R * 8));
    }
    if (a->weigh && p->split) p->scores = std::max(p->scores, up256(scores * 128));
    if (a->weigh && !p->split) {
      p->lse = std::max(p->lse, up256(rows * 4));
      const int shares = shares_of(*p, weigh_items);
      if (shares > 1)
        p->sums = std::max(p->sums, up256((uint64_t)shares * weigh_items * dv::kWeighTokens * 4));
    }
  }
  p->bytes = p->part + p->ml + p->scores + p->lse + p->sums;
  return DV_OK;
}

// Whether two of n * m rows of D elements share one: row (i, j) starts at i * s + j * t.
bool collide(int64_t n, int64_t s, int64_t m, int64_t t, int64_t D) {
  if ((n > 1 && s < D) || (m > 1 && t < D)) return true;
  if (n == 1 || m == 1 || (m - 1) * t + D <= s || (n - 1) * s + D <= t) return false;
  // Two rows lie |i * s - j * t| apart, i below n and j below m: for each j the
  // nearest i on either side.
  for (int64_t j = 1; j < m; ++j) {
    const int64_t i = j * t / s, over = j * t - i * s;
    if (i < n && over < D) return true;
    if (i + 1 < n && s - over < D) return true;
    if (i >= n) return false;  // and farther for every later j
  }
  return false;
}

// Sequences [b0, b0 + nseq) of a launch, `items(b)` work items each.
template <typename Items>
void fill(dv::AttendArgs* a, const int32_t* q_len, const int32_t* kv_len, int64_t b0, int nseq,
          int64_t G, int64_t H, Items items) {
  int64_t item = 0, tok = 0, scores = 0;
  for (int i = 0; i < kQSeqs; ++i) {
    a->item[i] = i < nseq ? (int32_t)item : INT32_MAX;
    a->tok[i] = (int32_t)tok;
    a->len[i] = i < nseq ? kv_len[b0 + i] : 0;
    a->soff[i] = (int32_t)scores;
    if (i < nseq && q_len[b0 + i] > 0) {
      item += items(b0 + i);
      tok += q_len[b0 + i];
      scores += q_len[b0 + i] * G * H * (((int64_t)kv_len[b0 + i] + 31) / 32);
    }
  }
  a->tok[kQSeqs] = (int32_t)tok;
  a->items = (int32_t)item;
}

// The same for trees, under many rows the longest sequences first: where work items do
// not all fit the card at once, those that end last should not begin last.  (32 sequences
// of 128 to 4096 tokens under 40 to 64 drafts of 8 heads of 8: 198 us, in the batch's order
// 257.  Few rows' items do fit.)
template <typename Items>
void fill_tree(dv::AttendArgs* a, const int32_t* q_len, const int32_t* kv_len, int64_t b0,
               int nseq, bool sorted, Items items) {
  int32_t order[kQSeqs], first[kQSeqs], tok = 0;
  for (int i = 0; i < nseq; ++i) {
    order[i] = i;
    first[i] = tok;
    tok += q_len[b0 + i];
  }
  if (sorted)
    std::sort(order, order + nseq, [&](int32_t x, int32_t y) {  // equal ones in the batch's order
      return kv_len[b0 + x] != kv_len[b0 + y] ? kv_len[b0 + x] > kv_len[b0 + y] : x < y;
    });
  int64_t item = 0;
  for (int i = 0; i < kQSeqs; ++i) {
    const int64_t b = i < nseq ? b0 + order[i] : b0;
    a->item[i] = i < nseq ? (int32_t)item : INT32_MAX;
    a->tok[i] = i < nseq ? first[order[i]] : tok;
    a->len[i] = i < nseq ? kv_len[b] : 0;
    a->soff[i] = i < nseq ? order[i] << 8 | q_len[b] : 0;
    if (i < nseq && q_len[b] > 0) item += items(b);
  }
  a->tok[kQSeqs] = tok;
  a->items = (int32_t)item;
}

// `tree`: drafts that follow each other as `parent` says.
int attend(const dv_quant* c, int32_t mb, int32_t layer, const int32_t* q_len,
           const int32_t* kv_len, bool tree, const int32_t* parent, const dv_attend_args* u,
           void* stream) {
  Quant q;
  int rc = quant_of(c, mb, &q);
  if (rc != DV_OK) return rc;
  const View& v = q.v;
  if (layer < 0 || layer >= v.L) return DV_ERR_RANGE;
  Plan p;
  rc = plan_of(q, q_len, kv_len, u, &p);
  if (rc != DV_OK) return rc;
  if (tree && u->weigh) return DV_ERR_UNSUPPORTED;
  if (u->weigh && !q.weight) return DV_ERR_INVALID;
  int64_t tokens = 0;
  for (int64_t b = 0; b < v.B; ++b) {
    tokens += q_len[b];
    if (tree && q_len[b] > kv_len[b]) return DV_ERR_RANGE;
    if (tree && q_len[b] > dv::kMaxDrafts) return DV_ERR_UNSUPPORTED;
  }
  if (u->rows < tokens) return DV_ERR_SPACE;
  if (tokens == 0) return DV_OK;
  const int64_t D = v.D;
  const int64_t strides[4] = {u->q_token, u->q_head, u->out_token, u->out_head};
  for (int64_t s : strides)
    if (s < 0 || s % 8 != 0 || s >= (1ll << 31)) return DV_ERR_INVALID;
  if (tree && (!parent || !aligned4(parent))) return DV_ERR_INVALID;
  if (!u->q || !u->out || !aligned16(u->q) || !aligned16(u->out) || !aligned4(u->slopes) ||
      !aligned4(u->lse) || !aligned16(u->workspace))
    return DV_ERR_INVALID;
  // rows of the result must not lie on each other
  if (collide(tokens, u->out_token, u->q_heads, u->out_head, D)) return DV_ERR_INVALID;
  if (u->workspace_bytes < p.bytes) return DV_ERR_SPACE;
  if (p.bytes && !u->workspace) return DV_ERR_INVALID;
  if (tangled(q)) return DV_ERR_INVALID;
  const uint64_t packed = (uint64_t)tokens * u->q_heads * D * 2;
  const bool q_one = u->q_head == D && u->q_token == u->q_heads * D;
  const bool o_one = u->out_head == D && u->out_token == u->q_heads * D;
  const uint64_t qn = q_one ? packed : D * 2, on = o_one ? packed : D * 2;
  const uint64_t ln = held(u->lse, (uint64_t)tokens * u->q_heads * 4), wn = p.bytes;
  const uint64_t sn = held(u->slopes, (uint64_t)u->q_heads * 4);
  if (overlaps(u->q, qn, u->out, on) || overlaps(u->q, qn, u->lse, ln) ||
      overlaps(u->q, qn, u->workspace, wn) || overlaps(u->out, on, u->lse, ln) ||
      overlaps(u->out, on, u->workspace, wn) || overlaps(u->lse, ln, u->workspace, wn) ||
      overlaps(u->slopes, sn, u->out, on) || overlaps(u->slopes, sn, u->lse, ln) ||
      overlaps(u->slopes, sn, u->workspace, wn) || hits(q, u->out, on) ||
      (ln && hits(q, u->lse, ln)) || (wn && hits(q, u->workspace, wn)) ||
      (tree && (overlaps(parent, tokens * 4, u->out, on) ||
                overlaps(parent, tokens * 4, u->lse, ln) ||
                overlaps(parent, tokens * 4, u->workspace, wn))) ||
      (u->weigh && (overlaps(u->q, qn, q.weight, q.slot_bytes) ||
                    overlaps(u->slopes, sn, q.weight, q.slot_bytes))))
    return DV_ERR_INVALID;

  const int64_t G = u->q_heads / v.H;
  hipStream_t st = static_cast<hipStream_t>(stream);
  char* w = static_cast<char*>(u->workspace);
  dv::AttendArgs a;
  memset(&a, 0, sizeof a);
  a.q = layout_args(q);
  a.q_token = u->q_token;
  a.q_head = u->q_head;
  a.o_token = u->out_token;
  a.o_head = u->out_head;
  a.slopes = u->slopes;
  a.lse = u->lse;
  a.part = reinterpret_cast<float*>(w);
  a.ml = reinterpret_cast<float*>(w + p.part);
  a.scores = p.scores ? reinterpret_cast<float*>(w + p.part + p.ml) : nullptr;
  a.row_lse = p.lse ? reinterpret_cast<float*>(w + p.part + p.ml + p.scores) : nullptr;
  a.sums = reinterpret_cast<float*>(w + p.part + p.ml + p.scores + p.lse);
  a.scale2 = u->scale * 1.4426950408889634f;
  a.decay = u->decay;
  a.layer = layer;
  a.G = (int32_t)G;
  a.d_G = dv::fast_div((uint32_t)G);
  a.q_heads = u->q_heads;
  a.chunk = p.chunk;
  a.weigh = u->weigh != 0;
  a.bf16 = u->type == DV_BF16;
  // Codes of 96 MB and more do not stay in the last-level cache, and are read
  // faster past it: 138 MB 36.1 us instead of 40.9, 268 MB 79.2 instead of 87.2,
  // but 63 MB 24.5 instead of 23.5.
  int64_t codes = 0;
  for (int64_t b = 0; b < v.B; ++b)
    if (q_len[b] > 0) codes += kv_len[b] * v.H * D * 2;
  a.nt = codes >= 96 << 20;
  int64_t row0 = 0;
  for (int64_t b0 = 0; b0 < v.B; b0 += kQSeqs) {
    const int nseq = (int)std::min<int64_t>(kQSeqs, v.B - b0);
    a.b0 = (int32_t)b0;
    a.nseq = nseq;
    a.row0 = (int32_t)row0;
    a.query = static_cast<const uint16_t*>(u->q) + row0 * u->q_token;
    a.out = static_cast<uint16_t*>(u->out) + row0 * u->out_token;
    a.parent = tree ? parent + row0 : nullptr;
    const auto items = [&](int64_t b) {
      return (q_len[b] * G + p.R - 1) / p.R * v.H * splits_of(p, kv_len[b]);
    };
    if (tree)
      fill_tree(&a, q_len, kv_len, b0, nseq, !p.split, items);
    else
      fill(&a, q_len, kv_len, b0, nseq, G, v.H, items);
    row0 += a.tok[kQSeqs];
    if (a.items == 0) continue;
    hipError_t e = p.split ? dv::launch_attend_split(a, p.R / 16, p.direct, st)
                           : dv::launch_attend_tile(a, p.direct, st);
    if (e == hipSuccess && !p.direct) e = dv::launch_attend_join(a, p.R, st);
    if (e == hipSuccess && a.weigh && !p.split) {
      fill(&a, q_len, kv_len, b0, nseq, G, v.H, [&](int64_t b) {
        return v.H * (((int64_t)kv_len[b] + dv::kWeighTokens - 1) / dv::kWeighTokens);
      });
      if (a.items) e = dv::launch_attend_weigh(a, shares_of(p, a.items), st);
    }
    if (e != hipSuccess) return dv::hip_fail(e, "attention launch");
  }
  return DV_OK;
}

}  // namespace

extern "C" {

int dv_quant_scale_bytes(const dv_quant* c, uint64_t* out_bytes) {
  Quant q;
  const int rc = layout8(c, &q);
  if (rc != DV_OK) return rc;
  if (!out_bytes) return DV_ERR_INVALID;
  *out_bytes = q.scale_bytes;
  return DV_OK;
}

int dv_quant_in(const dv_quant* dst, int32_t mb, int32_t l0, int32_t l1, const int32_t* t0,
                const int32_t* t1, const void* src, uint64_t src_bytes, int32_t type,
                void* stream) {
  Quant q;
  int rc = quant_of(dst, mb, &q);
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
  if (need > src_bytes) return DV_ERR_SPACE;
  if (need == 0) return DV_OK;
  if (!src || !aligned16(src) || hits(q, src, need) || tangled(q)) return DV_ERR_INVALID;

  dv::QuantArgs a;
  memset(&a, 0, sizeof a);
  a.q = layout_args(q);
  a.w_slab = v.H * v.D * 2 * N;
  a.bf16 = type == DV_BF16;
  // As few lanes to a block as hold its 16-element units in registers, two each,
  // or four where 64 lanes would not do: with 16 tokens of 128 dimensions (128
  // units) a pool of 32 x 128 to 4096 tokens (two layers of 8 heads) takes 162 us,
  // with room for four 165, and with that room and half of it empty 204; with 64
  // tokens (512 units) four take 174 and two, which read most units again, 190.
  const int64_t units = std::min<int64_t>(a.q.bs, longest) * v.D / 16;
  a.held = units <= 128 ? 2 : 4;
  while (a.lanes_log2 < 6 && (a.held << a.lanes_log2) < units) ++a.lanes_log2;
  return by_launches(q, l0, l1, t0, t1, src, a, [&](int32_t nl, const QuantArgs& x) {
    return launch_quant(x, 2 * nl, static_cast<hipStream_t>(stream));
  });
}

int dv_attend_bytes(const dv_quant* c, const int32_t* q_len, const int32_t* kv_len,
                    const dv_attend_args* a, uint64_t* out_bytes) {
  Quant q;
  int rc = layout8(c, &q);
  if (rc != DV_OK) return rc;
  if (!a || !out_bytes) return DV_ERR_INVALID;
  // With and without slopes, whose tables in LDS make other splits best.
  static const float slope = 0.f;
  uint64_t most = 0;
  for (int i = 0; i < 2; ++i) {
    dv_attend_args x = *a;
    x.slopes = i ? &slope : nullptr;
    Plan p;
    rc = plan_of(q, q_len, kv_len, &x, &p);
    if (rc != DV_OK) return rc;
    most = std::max(most, p.bytes);
  }
  *out_bytes = most;
  return DV_OK;
}

int dv_attend(const dv_quant* c, int32_t mb, int32_t layer, const int32_t* q_len,
              const int32_t* kv_len, const dv_attend_args* a, void* stream) {
  return attend(c, mb, layer, q_len, kv_len, false, nullptr, a, stream);
}

int dv_attend_tree(const dv_quant* c, int32_t mb, int32_t layer, const int32_t* q_len,
                   const int32_t* kv_len, const int32_t* parent, const dv_attend_args* a,
                   void* stream) {
  static_assert(dv::kMaxDrafts == DV_MAX_DRAFTS, "the interface's limit");
  return attend(c, mb, layer, q_len, kv_len, true, parent, a, stream);
}

int dv_evict(const dv_quant* src, int32_t src_mb, const dv_quant* dst, int32_t dst_mb, int32_t l0,
             int32_t l1, const int32_t* len, const int32_t* keep, int32_t recent, int32_t* kept,
             int32_t kept_stride, void* stream) {
  Quant s, d;
  int rc = quant_of(src, src_mb, &s);
  if (rc != DV_OK) return rc;
  rc = quant_of(dst, dst_mb, &d);
  if (rc != DV_OK) return rc;
  const View &v = s.v, &w = d.v;
  if (v.L != w.L || v.H != w.H || v.D != w.D || v.B != w.B) return DV_ERR_INVALID;
  if (!len || !keep || !s.weight) return DV_ERR_INVALID;
  if (l0 < 0 || l1 < l0 || l1 > v.L || recent < 0 || kept_stride < 0) return DV_ERR_RANGE;
  int64_t most = 0, longest = 0;
  for (int64_t b = 0; b < v.B; ++b) {
    if (len[b] < 0 || len[b] > v.cap || keep[b] < 0) return DV_ERR_RANGE;
    const int64_t k = std::min(len[b], keep[b]);
    if (k > w.cap || k > kept_stride) return DV_ERR_RANGE;
    most = std::max(most, k);
    longest = std::max<int64_t>(longest, len[b]);
  }
  if (most == 0 || l1 == l0) return DV_OK;
  if (!kept || !aligned4(kept)) return DV_ERR_INVALID;
  const bool in_place = v.base == w.base;
  if (in_place && (v.kind != w.kind || v.bt != w.bt || v.cap != w.cap || v.NB != w.NB ||
                   s.sb != d.sb || s.scale != d.scale || s.weight != d.weight ||
                   s.position != d.position))
    return DV_ERR_INVALID;
  const uint64_t kn = (uint64_t)(l1 - l0) * v.B * v.H * kept_stride * 4;
  if (tangled(s) || tangled(d) || (!in_place && hits(s, d)) || hits(s, kept, kn) ||
      hits(d, kept, kn))
    return DV_ERR_INVALID;
  const int64_t blocks = (most + d.sb - 1) / d.sb;
  if (v.H * blocks >= kMaxItems) return DV_ERR_UNSUPPORTED;
  // Sequences of a launch: its grids' widths are theirs times heads, times blocks or
  // the lanes that select.
  const int64_t lanes = (int64_t)v.H * dv::evict_select_lanes((int)longest);
  const int64_t seqs = std::min({(int64_t)kQSeqs, kMaxItems / (v.H * blocks), UINT32_MAX / lanes});

  dv::EvictArgs a;
  memset(&a, 0, sizeof a);
  a.s = layout_args(s);
  a.d = layout_args(d);
  a.kept_stride = kept_stride;
  a.recent = recent;
  a.in_place = in_place;
  a.most = (int32_t)longest;
  a.blocks = (int32_t)blocks;
  // Blocks whose tokens are looked up together: 128 tokens, or a block a wave.
  // (Half of 32 x 128 to 4096 tokens, 8 heads: 64 tokens 78.3 us, 128 78.5, 256
  // 79.5, 512 89.3, 1024 126; a quarter of 8 x 512 to 1024, 40 heads: 64 and 128
  // 20, 256 and more 25.)
  a.group = (int32_t)std::max<int64_t>(4, 128 / a.d.bs / 4 * 4);
  a.d_du = dv::fast_div((uint32_t)(v.D / 16));
  hipStream_t st = static_cast<hipStream_t>(stream);
  for (int32_t l = l0; l < l1; l += kLayers) {
    a.l0 = l;
    a.nl = std::min(kLayers, l1 - l);
    a.kept = kept + (int64_t)(l - l0) * v.B * v.H * kept_stride;
    for (int64_t b0 = 0; b0 < v.B; b0 += seqs) {
      a.b0 = (int32_t)b0;
      a.nseq = (int32_t)std::min<int64_t>(seqs, v.B - b0);
      int64_t items = 0;
      for (int i = 0; i < kQSeqs; ++i) {
        a.item[i] = i < a.nseq ? (int32_t)items : INT32_MAX;
        if (i >= a.nseq) continue;
        a.len[i] = len[b0 + i];
        a.keep[i] = keep[b0 + i];
        const int64_t n = (std::min(len[b0 + i], keep[b0 + i]) + d.sb - 1) / d.sb;
        items += v.H * (in_place ? n > 0 : (n + a.group - 1) / a.group);
      }
      a.items = (int32_t)items;
      if (items == 0) continue;
      hipError_t e = dv::launch_evict_select(a, st);
      if (e == hipSuccess) e = dv::launch_evict_move(a, st);
      if (e != hipSuccess) return dv::hip_fail(e, "eviction launch");
    }
  }
  return DV_OK;
}

}  // extern "C"
