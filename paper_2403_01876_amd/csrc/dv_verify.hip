// Which drafted tokens the target's distribution accepts, and the token after them.
//
// All that is decided by comparisons of sums of exponentials, and the last by where
// a random number falls among as many of them as there are tokens.  That one takes
// 64 bits, exponentials and sums: in 32 it would, one time in a few hundred over 32000
// tokens, hang on the order of a sum or the last bit of an exponential.  A draft that
// was not drawn is accepted or not by one comparison with its row's sum, for which 32
// bits do unless the two sides lie within the sum's error of each other; then the row
// is added up again in 64.  Drafts that were drawn leave differences of the two
// distributions behind, whose rows are added up in 64 bits at once.
//
// Two launches.  The sums of every row's pieces, a wave to each; and a workgroup for
// each part of a sequence's last row.  Each of these walks down the tree by itself, from
// those sums and the drafts' own logits, adds up its part of the row that the walk
// ends at, and the one that comes last finds the token.
#include "dv_draft_internal.h"

namespace dv {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// 2^t for t of [-1020, 0] to 3e-13: the nearest whole power, which adding 1.5 * 2^52
// leaves in the low bits, and the series of 2^f = e^(f ln 2) for the rest, |f| <= 1/2,
// to f^10.
struct Series {
  double c[11];
  constexpr Series() : c{} {
    c[0] = 1;
    for (int i = 1; i < 11; ++i) c[i] = c[i - 1] * 0.693147180559945309417232121458 / i;
  }
};
__device__ __forceinline__ double pow2(double t) {
  constexpr Series s;
  const double z = t + 0x1.8p52, f = t - (z - 0x1.8p52);
  double y = s.c[10];
#pragma unroll
  for (int i = 9; i >= 0; --i) y = __builtin_fma(y, f, s.c[i]);
  return __hiloint2double(__double2hiint(y) + (__double2loint(z) << 20), __double2loint(y));
}

// How a row's logits become shares relative to its largest, 0 below 2^-1020.
struct Scale {
  double scale2;  // log2(e) / temperature
  float top;
  int arg;        // greedy rows (scale2 0): the one token that has it all
  // (Infinite logits share all: +infinity less itself would be NaN.)
  __device__ __forceinline__ bool flat() const { return scale2 == 0. || top == INFINITY; }
  __device__ __forceinline__ double flat_share(float x, int token) const {
    return x == top && (scale2 != 0. || token == arg) ? 1. : 0.;
  }
  // No branches: a few of these in a row hide each other's waits.
  __device__ __forceinline__ double share(float x) const {
    const double t = ((double)x - top) * scale2, y = pow2(fmax(t, -1021.));
    return t < -1020. ? 0. : y;
  }
  __device__ __forceinline__ double of(float x, int token) const {
    return flat() ? flat_share(x, token) : share(x);
  }
};

template <int TYPE>
__device__ __forceinline__ float one_of(const void* row, int i) {
  float x;
  if constexpr (TYPE == 2)
    x = ((const float*)row)[i];
  else if constexpr (TYPE == 1)
    x = __uint_as_float((uint32_t)((const uint16_t*)row)[i] << 16);
  else
    x = (float)__builtin_bit_cast(_Float16, ((const uint16_t*)row)[i]);
  return x == x ? x : -INFINITY;
}
template <int TYPE>
__device__ __forceinline__ const void* row_of(const VerifyArgs& a, int64_t row) {
  return (const uint8_t*)a.logits + row * a.logits_row * (TYPE == 2 ? 4 : 2);
}
// Tokens of 16 bytes.
template <int TYPE>
constexpr int kPer = TYPE == 2 ? 4 : 8;
// How many tokens the 16 bytes that a row begins in hold before it: a row's pieces are
// counted from there.
template <int TYPE>
__device__ __forceinline__ int lead_of(const void* row) {
  return (int)((uintptr_t)row & 15) / (TYPE == 2 ? 4 : 2);
}
// The logits of 16 bytes; nth: NaN as -infinity.  (Quieted: the larger of a signalling NaN and
// a number is NaN where the compiler makes one maximum of three out of two.)
template <int TYPE>
__device__ __forceinline__ float raw(const u32x4& w, int i) {
  if constexpr (TYPE == 2) return __builtin_canonicalizef(__uint_as_float(w[i]));
  if constexpr (TYPE == 1)
    return __builtin_canonicalizef(
        __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16));
  return (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? w[i / 2] >> 16 : w[i / 2]));
}
template <int TYPE>
__device__ __forceinline__ float nth(const u32x4& w, int i) {
  return __builtin_fmaxf(raw<TYPE>(w, i), -INFINITY);
}
// N times 16 bytes of a row: tokens first + i * step ..., -infinity outside [0, vocab).
template <int TYPE, int N>
__device__ __forceinline__ void load(const void* row, int first, int step, int vocab, bool inside,
                                     u32x4 (&w)[N]) {
  constexpr int kSize = TYPE == 2 ? 4 : 2;
  const uint8_t* p = (const uint8_t*)row + (int64_t)first * kSize;
  if (inside) {  // the same in all lanes
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = *(const u32x4*)(p + i * step * kSize);
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int at = first + i * step;
    if (at >= 0 && at + kPer<TYPE> <= vocab) {
      w[i] = *(const u32x4*)(p + i * step * kSize);
    } else {
#pragma unroll
      for (int k = 0; k < kPer<TYPE>; ++k) {
        const bool on = at + k >= 0 && at + k < vocab;
        if constexpr (TYPE == 2) {
          w[i][k] = on ? ((const uint32_t*)row)[at + k] : 0xff800000u;
        } else {
          const uint32_t x = on ? ((const uint16_t*)row)[at + k] : TYPE == 1 ? 0xff80u : 0xfc00u;
          w[i][k / 2] = k & 1 ? w[i][k / 2] | x << 16 : x;
        }
      }
    }
  }
}

// A number of [0, 1]: NaN counts as 1.
__device__ __forceinline__ double chance(float u) { return u < 1.f ? fmaxf(u, 0.f) : 1.; }
__device__ __forceinline__ float some(float q) { return q > 0.f ? fminf(q, 0x1.fffffep127f) : 0.f; }

// Sums over the lanes up to and with each one, by moves within rows of 16 and from
// row to row: a tenth of the wait of exchanges through LDS.
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double x) {  // 0 where nothing comes from
  return __hiloint2double(
      __builtin_amdgcn_update_dpp(0, __double2hiint(x), CTRL, ROWS, 0xf, false),
      __builtin_amdgcn_update_dpp(0, __double2loint(x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ double upto(double x) {
  x += moved<0x111, 0xf>(x);  // row_shr: 1, 2, 4, 8
  x += moved<0x112, 0xf>(x);
  x += moved<0x114, 0xf>(x);
  x += moved<0x118, 0xf>(x);
  x += moved<0x142, 0xa>(x);  // row_bcast: 15 and 31
  return x + moved<0x143, 0xc>(x);
}
__device__ __forceinline__ double lane_of(double x, int lane) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(x), lane),
                          __builtin_amdgcn_readlane(__double2loint(x), lane));
}

// The larger of two logits with their tokens, the lower token of equal ones.
__device__ __forceinline__ void larger(float& top, int& arg, float x, int i) {
  if (x > top || (x == top && i < arg)) {
    top = x;
    arg = i;
  }
}

// ---------------------------------------------------------------------------
// A piece of a row: its largest logit, and the sum of the shares relative to it; a
// wave's.  In 32 bits (not EXACT) a share is 2^t, t = s x + c with one rounding, c = -s top;
// c's own is the same for all and is put right in the sum.  t then errs by two half
// steps, s's among them: 1e-5 of the smallest share that counts, and the sum of 64 lanes'
// 32 shares by 40 half steps, 3e-6; by less than kSumError together.
// Bound by HBM in 32 bits, once the launch is paid: of 53 million logits in 16 bits half
// lie in rows that judge others, 43 MB read in 12 us (all rows: 21).  In 64 bits by the
// exponentials, 22 instructions each: 6.7 million 9.4 us.  (Pieces of 2048 tokens: chains
// 24.7 us a call, of 4096 26.3, of 8192 31.)
// ---------------------------------------------------------------------------
constexpr double kSumError = 0x1p-15;
// A pass over the row in 64 bits: 512 threads add up 2^15 of 2^24 shares each, one after
// another, which errs by 2^-38 of the sum; taking 127 of them away again, by 2^-46 of it.
constexpr double kPassError = 0x1p-36;

template <int TYPE, bool EXACT>
__global__ void __launch_bounds__(kThreads) verify_sums_kernel(VerifyArgs a) {
  constexpr int N = kPiece / 64 / kPer<TYPE>;
  const int l = threadIdx.x & 63;
  const int item = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)));
  const int row = item / (uint32_t)a.pieces, piece = item - row * a.pieces;
  if (row >= a.tok[kQSeqs]) return;
  int below = 0;  // sequences that begin at or before this row
  for (int i = 0; i < a.nseq; i += 64)
    below += __popcll(__ballot(i + l < a.nseq && a.tok[min(i + l, a.nseq - 1)] <= row));
  const double scale2 = a.scale2[below - 1];
  const int first_row = a.tok[below - 1], draft = row - first_row;
  if (piece == 0 && draft == 0 && l == 0) a.arrived[a.b0 + below - 1] = 0;
  if (!EXACT) {  // a row that no other draft follows judges none
    const int nq = a.tok[below] - first_row;
    const int32_t* parent = a.parent + a.row0 + first_row;
    const int up0 = l < nq ? parent[l] : -1, up1 = l + 64 < nq ? parent[l + 64] : -1;
    if (!__any(up0 == draft || up1 == draft)) return;
  }
  const void* p = row_of<TYPE>(a, a.row0 + row);
  const int start = piece * kPiece - lead_of<TYPE>(p), first = start + l * kPer<TYPE>;
  u32x4 w[N];
  load<TYPE>(p, first, 64 * kPer<TYPE>, a.vocab, start >= 0 && start + kPiece <= a.vocab, w);
  float top = -INFINITY;
  if constexpr (TYPE == 0) {
    f16x2 most = {(_Float16)-INFINITY, (_Float16)-INFINITY};
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {  // NaN is left out
        const uint32_t y = w[i][k];  // (a cast of the element itself reads the first one)
        most = __builtin_elementwise_max(most, __builtin_bit_cast(f16x2, y));
      }
    top = fmaxf((float)most[0], (float)most[1]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int k = 0; k < kPer<TYPE>; ++k) top = fmaxf(top, raw<TYPE>(w[i], k));
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
  int arg = 0;
  double sum = 0.;
  if (scale2 == 0. || top == INFINITY) {
    arg = INT32_MAX;
    int equal = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int k = 0; k < kPer<TYPE>; ++k)
        if (nth<TYPE>(w[i], k) == top) {
          arg = min(arg, first + i * 64 * kPer<TYPE> + k);
          ++equal;
        }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      arg = min(arg, __shfl_xor(arg, o));
      equal += __shfl_xor(equal, o);
    }
    sum = scale2 == 0. ? 1. : equal;
  } else if (top != -INFINITY) {
    if constexpr (EXACT) {
      const Scale scale{scale2, top, 0};
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int k = 0; k < kPer<TYPE>; ++k) sum += scale.share(nth<TYPE>(w[i], k));
      sum = lane_of(upto(sum), 63);
    } else {
      const float s = (float)fmin(scale2, 0x1p100), c = -top * s;
      float part = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int k = 0; k < kPer<TYPE>; ++k)
          part += __builtin_amdgcn_exp2f(__builtin_fmaf(raw<TYPE>(w[i], k), s, c));
      // Some NaN, or numbers so large that c's rounding is of the size of t: each by itself.
      if (__any(!(part < INFINITY)) || !(fabsf(c) < 0x1p20f)) {
        part = 0.f;
#pragma unroll 1
        for (int u = first; u < start + kPiece; u += 64 * kPer<TYPE>)
          for (int k = max(u, 0); k < min(u + kPer<TYPE>, a.vocab); ++k)
            // (halves: the difference of two logits may lie beyond 32 bits' range)
            part += __builtin_amdgcn_exp2f((0.5f * one_of<TYPE>(p, k) - 0.5f * top) * (2.f * s));
      } else {
        part *= __builtin_amdgcn_exp2f(__builtin_fmaf(-top, s, -c));
      }
      sum = lane_of(upto((double)part), 63);
    }
  }
  if (l == 0) a.sums[((int64_t)a.row0 + row) * a.pieces + piece] = PieceSum{sum, top, arg};
}

// ---------------------------------------------------------------------------
// The walk and the last row.  First every draft's row is put together from its pieces
// and its token's share of the row that judges it found, all at once; then the drafts
// are tried in order, of which a wave sees with one ballot those that follow the draft
// accepted last.  With Z the sum of what is left of a row (its shares, relative to its
// largest logit),
//   not drawn: a rejected token's share leaves Z, which takes a pass over the row where the
//          comparison lies within the error of Z or little is left,
//   drawn: what is left of a token's share w becomes max(w - q Z, 0), whose sum takes a
//          pass over the row where another draft is to be tried against it.
// Then each workgroup adds up its pieces of what is left in 64 bits, and the one that
// comes last of a sequence's finds the piece in which the random number falls, and the
// token there.  A row that judges no draft was not added up before: its pieces are
// relative to their own largest logits until that one.
// Bound by latency, a dozen steps that wait for each other: 32 sequences of 4 to 9 drafts
// over 32000 tokens 14 us, of 40 to 64 16, one sequence over 131071 13.  (512 threads: chains
// 26.9 us a call, 256 27.8, 1024 28.4; sums by exchanges through LDS instead of moves
// between lanes cost 4 us more.)  Passes are bound by exponentials, the whole row in every
// workgroup: a call for 32 sequences of 2, 4 and 16 drawn siblings over 32000 tokens takes 38,
// 82 and 565 us, since each pass goes through all rejections before it.
// ---------------------------------------------------------------------------
constexpr int kWalkers = 512, kWaves = kWalkers / 64;
constexpr int kEach = kPiece / kWalkers;  // tokens of a piece that a thread takes, in order
static_assert(kEach % 4 == 0 && kWaves <= 16, "four() tokens at a time; a row of lanes");

// The sum over the workgroup in a fixed order, in all of its threads.
__device__ __forceinline__ double sum_all(double x, double* part) {
  x = lane_of(upto(x), 63);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  return lane_of(upto(part[threadIdx.x & (kWaves - 1)]), kWaves - 1);
}

// Logits of tokens first ... first + 3, -infinity outside [0, vocab).
template <int TYPE>
__device__ __forceinline__ f32x4 four(const void* row, int first, int vocab) {
  f32x4 x;
  if (first >= 0 && first + 4 <= vocab) {
    u32x4 w;
    if constexpr (TYPE == 2) {
      w = *(const u32x4*)((const float*)row + first);
    } else {
      const uint2 y = *(const uint2*)((const uint16_t*)row + first);
      w = u32x4{y.x, y.y, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = nth<TYPE>(w, i);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float y = one_of<TYPE>(row, min(max(first + i, 0), vocab - 1));
      x[i] = first + i >= 0 && first + i < vocab ? y : -INFINITY;
    }
  }
  return x;
}
// Probabilities of the same (of any tokens outside).
__device__ __forceinline__ f32x4 drawn_four(const float* q, int first, int vocab) {
  f32x4 x;
  if (first >= 0 && first + 4 <= vocab && ((uintptr_t)(q + first) & 15) == 0) {
    x = *(const f32x4*)(q + first);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = q[min(max(first + i, 0), vocab - 1)];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = some(x[i]);
  return x;
}

// What is left of a share after `turns` rejections of drawn drafts: the row held `first`
// before the first of them, sums[i] before the i-th one after it.
__device__ __forceinline__ double after(double w, double q, double first, const double* sums,
                                        int turns) {
  if (turns > 0) w = fmax(w - q * first, 0.);
  for (int i = 1; i < turns; ++i) w = fmax(w - q * sums[i], 0.);
  return w;
}

// Bit i of two words of drafts, the lowest taken off.
__device__ __forceinline__ int next_of(uint64_t& lo, uint64_t& hi) {
  const int i = lo ? __builtin_ctzll(lo) : 64 + __builtin_ctzll(hi);
  if (lo)
    lo &= lo - 1;
  else
    hi &= hi - 1;
  return i;
}

template <int TYPE>
__global__ void __launch_bounds__(kWalkers) verify_walk_kernel(VerifyArgs a) {
  __shared__ double total[kMaxDrafts], share[kMaxDrafts], part[kWaves], parts[kWaves], sums[kMaxDrafts];
  __shared__ float tops[kWaves];
  __shared__ uint64_t firsts[2];
  __shared__ float top[kMaxDrafts], from[kMaxDrafts], lot[kMaxDrafts];
  __shared__ int arg[kMaxDrafts], token[kMaxDrafts], judges[kMaxDrafts], ends[kWaves][2];
  __shared__ bool last;
  const int tid = threadIdx.x, l = tid & 63, wave = tid >> 6;
  const int b = blockIdx.x / (uint32_t)a.parts, at = blockIdx.x - b * a.parts;
  const int tok = a.row0 + a.tok[b], nq = a.tok[b + 1] - a.tok[b], sb = a.b0 + b;
  const double scale2 = a.scale2[b];
  if (nq == 0) {
    if (tid == 0 && at == 0) a.count[sb] = 0;
    return;
  }
  // Drafts l and l + 64, in every wave: what they follow (-1: nothing, or not a token), and
  // their tokens.
  int up0 = -1, up1 = -1, x0 = -1, x1 = -1;
  if (l < nq) {
    up0 = a.parent[tok + l];
    x0 = a.token[tok + l];
  }
  if (l + 64 < nq) {
    up1 = a.parent[tok + l + 64];
    x1 = a.token[tok + l + 64];
  }
  if (tid < kMaxDrafts) judges[tid] = a.drawn != nullptr;
  const float chance_of = tid < nq ? a.uniform[tok + tid] : 0.f;
  // Rows: a group of lanes puts one together at a time, each its first pieces at once.
  int lanes = 8;
  while (lanes < 64 && lanes < a.pieces && nq * lanes * 2 <= kWalkers) lanes <<= 1;
  for (int i0 = 0; i0 < nq; i0 += kWalkers / lanes) {
    const int i = i0 + tid / lanes, k0 = tid & (lanes - 1);
    const PieceSum* s = a.sums + ((int64_t)tok + min(i, nq - 1)) * a.pieces;
    float t = -INFINITY;
    int g = INT32_MAX;
    constexpr int kHeld = 4;
    PieceSum held[kHeld];
#pragma unroll
    for (int j = 0; j < kHeld; ++j) held[j] = s[min(k0 + j * lanes, a.pieces - 1)];
#pragma unroll
    for (int j = 0; j < kHeld; ++j) larger(t, g, held[j].top, held[j].arg);  // (or again)
    for (int k = k0 + kHeld * lanes; k < a.pieces; k += lanes) larger(t, g, s[k].top, s[k].arg);
    for (int o = 1; o < lanes; o <<= 1) larger(t, g, __shfl_xor(t, o), __shfl_xor(g, o));
    const Scale scale{scale2, t, g};
    auto of = [&](const PieceSum& x) {
      return x.sum == 0. ? 0. : x.sum * scale.of(x.top, x.arg);
    };
    double sum = 0.;
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
      if (k0 + j * lanes < a.pieces) sum += of(held[j]);
    for (int k = k0 + kHeld * lanes; k < a.pieces; k += lanes) sum += of(s[k]);
    for (int o = 1; o < lanes; o <<= 1) sum += __shfl_xor(sum, o);
    if (k0 == 0 && i < nq) {
      total[i] = t == -INFINITY ? 0. : sum;
      top[i] = t;
      arg[i] = g;
    }
  }
  up0 = up0 >= 0 && up0 < l && x0 >= 0 && x0 < a.vocab ? up0 : -1;
  up1 = up1 >= 0 && up1 < l + 64 && x1 >= 0 && x1 < a.vocab ? up1 : -1;
  // Rows that a draft follows; of the others there are no sums where drafts were not drawn.
  __syncthreads();  // (cleared)
  if (wave == 0 && up0 >= 0) judges[up0] = 1;
  if (wave == 0 && up1 >= 0) judges[up1] = 1;
  // Threads below 128 stand for a draft each.
  const int up = wave ? up1 : up0, x = wave ? x1 : x0;
  float y = 0.f, d = 0.f;
  if (tid < kMaxDrafts && up >= 0) {
    y = one_of<TYPE>(row_of<TYPE>(a, tok + up), x);
    if (a.drawn) d = some(a.drawn[(int64_t)(tok + up) * a.drawn_row + x]);
  }
  __syncthreads();
  const double error = a.drawn || scale2 == 0. ? 0. : scale2 > 0x1p100 ? 1. : kSumError;
  if (wave < 2) {
    bool passes = false;  // as the first that is tried, beyond doubt
    if (up >= 0) {
      const Scale scale{scale2, top[up], arg[up]};
      const double sum = total[up], w = sum == 0. ? 0. : scale.of(y, x);
      passes = chance(chance_of) * (a.drawn ? (double)d : 1.) * sum < w - sum * error;
      share[tid] = w;
    }
    if (tid < nq) {
      from[tid] = d;
      lot[tid] = chance_of;
      token[tid] = x;
    }
    const uint64_t bits = __ballot(passes);
    if (l == 0) firsts[wave] = bits;
  }
  __syncthreads();

  const bool teller = tid == 0 && at == 0;
  int here = 0, n = 1, turns = 0;
  uint64_t gone0 = 0, gone1 = 0;  // drafts whose shares have left the row
  bool pending = false;           // whether the last rejection's sum is not known yet
  if (teller) a.path[tok] = 0;
  const uint64_t pass0 = firsts[0], pass1 = firsts[1];
  for (;;) {
    uint64_t try0 = __ballot(up0 == here), try1 = __ballot(up1 == here);
    if (!(try0 | try1)) break;
    const int next = try0 ? __builtin_ctzll(try0) : 64 + __builtin_ctzll(try1);
    if ((next < 64 ? pass0 >> next : pass1 >> (next - 64)) & 1) {  // most often
      here = next;
      if (teller) a.path[tok + n] = here;
      ++n;
      continue;
    }
    if (total[here] == 0.) break;
    const void* row = row_of<TYPE>(a, tok + here);
    const float* q = a.drawn ? a.drawn + (int64_t)(tok + here) * a.drawn_row : nullptr;
    const Scale scale{scale2, top[here], arg[here]};
    // The sum over the row's tokens of what is left of them, those of drafts out0 and out1 aside.
    auto pass = [&](int rejections, uint64_t out0, uint64_t out1) {
      double sum = 0.;
      const int lead = lead_of<TYPE>(row);
#pragma unroll 1
      for (int first = tid * 4 - lead; first < a.vocab; first += kWalkers * 4) {
        f32x4 z = four<TYPE>(row, first, a.vocab);
        f32x4 d = {0, 0, 0, 0};
        if (q) d = drawn_four(q, first, a.vocab);
        for (uint64_t g = out0, h = out1; g | h;) {
          const int y = token[next_of(g, h)] - first;
#pragma unroll
          for (int i = 0; i < 4; ++i) z[i] = i == y ? -INFINITY : z[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += after(scale.of(z[i], first + i), d[i], total[here], sums, rejections);
      }
      return sum_all(sum, part);
    };
    // Not drawn: `left` may be off by this much.
    double left = total[here], off = left * error;
    int taken = -1;
    while (try0 | try1) {
      const int i = next_of(try0, try1);
      const double u = chance(lot[i]);
      double r = share[i];
      if (q) {
        if (pending) {  // the sum of what the last rejection left
          const double sum = pass(turns + 1, 0, 0);
          if (sum > 0.) {
            ++turns;
            left = sum;
            if (tid == 0) sums[turns] = sum;  // (the pass's barriers were after the last reads)
            __syncthreads();
          }
        }
        pending = !(u * from[i] * left < after(r, from[i], total[here], sums, turns));
        if (!pending) taken = i;
      } else {
        const int x = token[i];  // the second guess of a token has nothing left
        if ((__ballot(up0 == here && x0 == x) & gone0) | (__ballot(up1 == here && x1 == x) & gone1))
          r = 0.;
        const uint64_t bit0 = i < 64 ? 1ull << i : 0, bit1 = i < 64 ? 0 : 1ull << (i & 63);
        double rest = left - r;
        if (r > 0. && (fabs(u * left - r) <= off || (u * left >= r && rest <= off))) {
          // Too near to tell, or little may be left: what the other tokens hold, added up in 64
          // bits.  A difference would err by the size of what it is taken from; this sum is 0
          // where nothing is left, and else right to its own size.
          rest = pass(0, gone0 | bit0, gone1 | bit1);
          left = rest + r;
          off = rest * kPassError;
        }
        if (u * left < r) {
          taken = i;
        } else if (r > 0. && rest > 0.) {
          left = rest;
          gone0 |= bit0;
          gone1 |= bit1;
        }
      }
      if (taken >= 0) break;
    }
    if (taken < 0) break;
    here = taken;
    turns = 0;
    gone0 = gone1 = 0;
    pending = false;
    if (teller) a.path[tok + n] = here;
    ++n;
  }
  if (teller) a.count[sb] = n;
  const bool bare = !judges[here];  // a row without sums: what is left of it is all of it
  if (!bare && total[here] == 0.) {  // nothing has any probability
    if (teller) a.next[sb] = -1;
    return;
  }

  // What this thread's tokens of a piece hold, and held before the last rejection.
  const void* row = row_of<TYPE>(a, tok + here);
  const float* q = a.drawn ? a.drawn + (int64_t)(tok + here) * a.drawn_row : nullptr;
  Scale scale{scale2, top[here], arg[here]};
  const int lead = lead_of<TYPE>(row);
  double now[kEach], was[kEach];
  auto sum_of = [](const double (&x)[kEach]) {
    double y = x[0];
#pragma unroll
    for (int i = 1; i < kEach; ++i) y += x[i];
    return y;
  };
  auto weigh = [&](int piece, bool alone) {
    const int first = piece * kPiece + tid * kEach - lead;
    float z[kEach], d[kEach];
#pragma unroll
    for (int i = 0; i < kEach; i += 4) {
      const f32x4 x = four<TYPE>(row, first + i, a.vocab);
      f32x4 y = {0, 0, 0, 0};
      if (q) y = drawn_four(q, first + i, a.vocab);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        z[i + k] = x[k];
        d[i + k] = y[k];
      }
    }
    if (alone) {  // shares relative to the piece's own largest logit
      float big = z[0];
      int at = first;
#pragma unroll
      for (int i = 1; i < kEach; ++i) larger(big, at, z[i], first + i);
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) larger(big, at, __shfl_xor(big, o), __shfl_xor(at, o));
      __syncthreads();
      if (l == 0) {
        tops[wave] = big;
        ends[wave][0] = at;
      }
      __syncthreads();
      big = tops[0];
      at = ends[0][0];
#pragma unroll
      for (int i = 1; i < kWaves; ++i) larger(big, at, tops[i], ends[i][0]);
      scale.top = big;
      scale.arg = at;
    }
    if (scale.flat()) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) was[i] = scale.flat_share(z[i], first + i);
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i) was[i] = scale.share(z[i]);
    }
    for (int k = 0; k < turns; ++k) {
      const double by = k ? sums[k] : total[here];
#pragma unroll
      for (int i = 0; i < kEach; ++i) was[i] = fmax(was[i] - d[i] * by, 0.);
    }
    const double by = !pending ? 0. : turns ? sums[turns] : total[here];
#pragma unroll
    for (int i = 0; i < kEach; ++i) now[i] = fmax(was[i] - d[i] * by, 0.);
    for (uint64_t g = gone0, h = gone1; g | h;) {
      const int y = token[next_of(g, h)] - first;
#pragma unroll
      for (int i = 0; i < kEach; ++i) now[i] = i == y ? 0. : now[i];
    }
  };
  double* const held_at = a.left + (int64_t)sb * a.pieces * 2;
  const int per = (a.pieces + a.parts - 1) / a.parts;  // pieces of a part
#pragma unroll 1
  for (int piece = at * per; piece < min(a.pieces, (at + 1) * per); ++piece) {
    weigh(piece, bare);
    double x = upto(sum_of(now));
    const double y = upto(sum_of(was));
    if (bare && scale.top == -INFINITY) x = 0.;
    __syncthreads();  // (what was in these has been read)
    if (l == 63) {
      part[wave] = x;
      parts[wave] = y;
    }
    __syncthreads();
    if (wave == 0) {
      const double u = upto(part[l & (kWaves - 1)]);
      const double v = bare ? (double)scale.top : upto(parts[l & (kWaves - 1)]);
      if (l == kWaves - 1) {
        __hip_atomic_store(held_at + 2 * piece, u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(held_at + 2 * piece + 1, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    }
  }
  // The sums are all that one workgroup reads of another's.  They are written and read at
  // the scope of the whole device, past each die's cache, and have arrived there (the
  // wait) before the count goes up; a release would write every dirty line of the cache
  // back.
  if (tid == kWaves - 1) {  // who wrote them
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    last = __hip_atomic_fetch_add(a.arrived + sb, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
           a.parts - 1;
  }
  __syncthreads();
  if (!last) return;

  // The pieces' sums, 64 at a time, in each wave alike.  What the last rejection leaves
  // counts, unless that is nothing.
  auto held = [&](int k, int which) {
    return k < a.pieces ? __hip_atomic_load(held_at + 2 * k + which, __ATOMIC_RELAXED,
                                            __HIP_MEMORY_SCOPE_AGENT)
                        : 0.;
  };
  int which = 0;
  double all = 0.;
  if (bare) {  // the row's largest logit, which shares are relative to from here on
    float big = -INFINITY;
    for (int k = l; k < a.pieces; k += 64) big = fmaxf(big, (float)held(k, 1));
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) big = fmaxf(big, __shfl_xor(big, o));
    scale.top = big;
    if (big == -INFINITY) {  // nothing has any probability
      if (tid == 0) a.next[sb] = -1;
      return;
    }
  }
  bool found = false;  // greedy: the first piece that has the largest logit is all there is
  auto amount = [&](int k) {
    const double x = held(k, which);
    if (!bare) return x;
    const double y = x == 0. ? 0. : x * scale.of((float)held(k, 1), scale.arg);
    if (scale2 != 0.) return y;
    const uint64_t have = __ballot(k < a.pieces && x != 0. && (float)held(k, 1) == scale.top);
    const bool mine = have && !found && l == __builtin_ctzll(have);
    found |= have != 0;
    return mine ? 1. : 0.;
  };
  for (int k = l; k < a.pieces + l; k += 64) all += amount(k);
  all = lane_of(upto(all), 63);
  if (!bare && !(all > 0.)) {
    which = 1;
    all = 0.;
    for (int k = l; k < a.pieces; k += 64) all += held(k, 1);
    all = lane_of(upto(all), 63);
  }
  // (1 passes no sum: as a product it could, where sums of other groupings round up)
  const double u = chance(lot[0]), goal = u < 1. ? u * all : INFINITY;
  found = false;
  double before = 0., sum = 0.;
  int place = 0;  // the first piece whose sum passes the goal, or the last that holds anything
  for (int k = 0; k < a.pieces; k += 64) {
    const double z = amount(k + l), up = upto(z);
    const uint64_t past = __ballot(z > 0. && sum + up > goal), any = __ballot(z > 0.);
    if (any) {
      const int i = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(any);
      place = k + i;
      before = sum + lane_of(up - z, i);
    }
    if (past) break;
    sum += lane_of(up, 63);
  }
  weigh(place, bare && scale2 == 0.);
  if (which) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) now[i] = was[i];
  }
  const double mine_here = sum_of(now), here_too = upto(mine_here);
  __syncthreads();
  if (l == 63) part[wave] = here_too;
  __syncthreads();
  const double waves = upto(part[l & (kWaves - 1)]);
  double run = before + (here_too - mine_here) + (wave ? lane_of(waves, max(wave - 1, 0)) : 0.);
  // The first token whose sum passes the goal, or the last that holds anything.
  int hit = -1, end = -1;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int y = place * kPiece - lead + tid * kEach + i;
    run += now[i];
    if (now[i] > 0.) {
      end = y;
      if (run > goal && hit < 0) hit = y;
    }
  }
  const uint64_t hits = __ballot(hit >= 0), any = __ballot(end >= 0);
  if (l == 0) {
    ends[wave][0] = hits ? __builtin_amdgcn_readlane(hit, __builtin_ctzll(hits)) : -1;
    ends[wave][1] = any ? __builtin_amdgcn_readlane(end, 63 - __builtin_clzll(any)) : -1;
  }
  __syncthreads();
  if (wave == 0) {
    const int h = ends[l & (kWaves - 1)][0], e = ends[l & (kWaves - 1)][1];
    const uint64_t hs = __ballot(h >= 0), es = __ballot(e >= 0 && l < kWaves);
    if (l == (hs ? __builtin_ctzll(hs) : es ? 63 - __builtin_clzll(es) : 0)) a.next[sb] = hs ? h : e;
  }
}

hipError_t start(const void* fn, const VerifyArgs& a, uint32_t groups, int threads,
                 hipStream_t s) {
  void* args[] = {const_cast<VerifyArgs*>(&a)};
  return hipLaunchKernel(fn, dim3(groups), dim3(threads), args, 0, s);
}

template <bool EXACT>
const void* sums_of(int type) {
  return type == 0   ? (const void*)&verify_sums_kernel<0, EXACT>
         : type == 1 ? (const void*)&verify_sums_kernel<1, EXACT>
                     : (const void*)&verify_sums_kernel<2, EXACT>;
}

}  // namespace

hipError_t launch_verify_sums(const VerifyArgs& a, hipStream_t s) {
  const uint32_t waves = (uint32_t)a.tok[kQSeqs] * a.pieces, per = kThreads / 64;
  return start(a.drawn ? sums_of<true>(a.type) : sums_of<false>(a.type), a,
               (waves + per - 1) / per, kThreads, s);
}
hipError_t launch_verify_walk(const VerifyArgs& a, hipStream_t s) {
  return start(a.type == 0   ? (const void*)&verify_walk_kernel<0>
               : a.type == 1 ? (const void*)&verify_walk_kernel<1>
                             : (const void*)&verify_walk_kernel<2>,
               a, (uint32_t)a.nseq * a.parts, kWalkers, s);
}

}  // namespace dv
