// Which drafted tokens the target's distribution accepts, and the token after them.
//
// All that is decided by comparisons of sums of exponentials, and the last by where
// a random number falls among as many of them as there are tokens: sums, and the
// exponentials, are held in 64 bits, so that neither the order of a sum nor the last
// bit of an exponential moves a border that anyone could tell (32 bits would, one time
// in a few hundred over 32000 tokens).
//
// Three launches: the sums of every row's pieces; the walk down the tree, a workgroup
// to a sequence, from those sums and the drafts' own logits; and the last row again,
// piece by piece, of which the workgroup that comes last finds the token.
#include "dv_draft_internal.h"

namespace dv {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 2^t for t <= 0 to 1e-14 (0 below 2^-1060, and for NaN): the nearest whole power and
// the series of 2^f = e^(f ln 2) for the rest, |f| <= 1/2, to f^11.
struct Series {
  double c[12];
  constexpr Series() : c{} {
    c[0] = 1;
    for (int i = 1; i < 12; ++i) c[i] = c[i - 1] * 0.693147180559945309417232121458 / i;
  }
};
__device__ __forceinline__ double pow2(double t) {
  constexpr Series s;
  const double n = __builtin_rint(t), f = t - n;
  double y = s.c[11];
#pragma unroll
  for (int i = 10; i >= 0; --i) y = __builtin_fma(y, f, s.c[i]);
  return t > -1060. ? __builtin_ldexp(y, (int)n) : 0.;
}

// A logit's share relative to the row's largest; greedy rows (scale2 0): one token's.
// (+infinity less itself is NaN: infinite logits share all.)
__device__ __forceinline__ double weight_of(float x, int token, float top, int arg, double scale2) {
  if (scale2 == 0.) return token == arg ? 1. : 0.;
  return x == top ? (x == -INFINITY ? 0. : 1.) : pow2(((double)x - top) * scale2);
}

template <int TYPE>
__device__ __forceinline__ float one_of(const void* row, int i) {
  if constexpr (TYPE == 2) return ((const float*)row)[i];
  const uint16_t x = ((const uint16_t*)row)[i];
  if constexpr (TYPE == 1) return __uint_as_float((uint32_t)x << 16);
  return (float)__builtin_bit_cast(_Float16, x);
}
template <int TYPE>
__device__ __forceinline__ const void* row_of(const VerifyArgs& a, int64_t row) {
  return (const uint8_t*)a.logits + row * a.logits_row * (TYPE == 2 ? 4 : 2);
}

// Tokens to a lane, and what a lane holds of a piece: tokens first ... first + kEach - 1 of
// a row, those outside [0, vocab) and NaN as -infinity.
constexpr int kEach = kPiece / kThreads;
// The token of a row's first lane: 0, or the start of its 16 bytes, which is before it.
template <int TYPE>
__device__ __forceinline__ int lead_of(const void* row) {
  return (int)((uintptr_t)row & 15) / (TYPE == 2 ? 4 : 2);
}
template <int TYPE>
__device__ __forceinline__ void load(const void* row, int first, int vocab, float (&x)[kEach]) {
  if (first >= 0 && first + kEach <= vocab) {
    constexpr int kSize = TYPE == 2 ? 4 : 2, kLoads = kEach * kSize / 16, kPer = 16 / kSize;
    const u32x4* p = (const u32x4*)((const uint8_t*)row + (int64_t)first * kSize);
    u32x4 w[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) w[i] = p[i];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if constexpr (TYPE == 2)
        x[i] = __uint_as_float(w[i / kPer][i % kPer]);
      else {
        const uint32_t y = w[i / kPer][i % kPer / 2];
        if constexpr (TYPE == 1)
          x[i] = __uint_as_float(i & 1 ? y & 0xffff0000u : y << 16);
        else
          x[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? y >> 16 : y));
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      x[i] = first + i >= 0 && first + i < vocab ? one_of<TYPE>(row, first + i) : -INFINITY;
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i) x[i] = x[i] == x[i] ? x[i] : -INFINITY;
}

// A number of [0, 1]: NaN counts as 1.
__device__ __forceinline__ double chance(float u) { return u < 1.f ? fmaxf(u, 0.f) : 1.; }
__device__ __forceinline__ float some(float q) { return q > 0.f ? q : 0.f; }

// The sum over a workgroup in a fixed order, in all of its threads (`part`: a number for
// each wave, free again after the next barrier).
__device__ __forceinline__ double sum_all(double x, double* part) {
  const int waves = blockDim.x >> 6;
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  double y = part[0];
  for (int i = 1; i < waves; ++i) y += part[i];
  return y;
}

// The larger of two logits with their tokens, the lower token of equal ones.
__device__ __forceinline__ void larger(float& top, int& arg, float x, int i) {
  if (x > top || (x == top && i < arg)) {
    top = x;
    arg = i;
  }
}

// ---------------------------------------------------------------------------
// A piece of a row: its largest logit, and the sum of the others' shares relative to it.
// ---------------------------------------------------------------------------
template <int TYPE>
__global__ void __launch_bounds__(kThreads) verify_sums_kernel(VerifyArgs a) {
  __shared__ float tops[kThreads / 64];
  __shared__ int args[kThreads / 64];
  __shared__ double part[kThreads / 64];
  const int tid = threadIdx.x, l = tid & 63, wave = tid >> 6;
  const int row = blockIdx.x / (uint32_t)a.pieces, piece = blockIdx.x - row * a.pieces;
  int below = 0;  // sequences that begin at or before this row
  for (int i = 0; i < a.nseq; i += 64)
    below += __popcll(__ballot(i + l < a.nseq && a.tok[min(i + l, a.nseq - 1)] <= row));
  const double scale2 = a.scale2[below - 1];
  const void* p = row_of<TYPE>(a, a.row0 + row);
  const int first = piece * kPiece + tid * kEach - lead_of<TYPE>(p);
  float x[kEach];
  load<TYPE>(p, first, a.vocab, x);
  float top = x[0];
  int arg = first;
#pragma unroll
  for (int i = 1; i < kEach; ++i) larger(top, arg, x[i], first + i);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) larger(top, arg, __shfl_xor(top, o), __shfl_xor(arg, o));
  if (l == 0) {
    tops[wave] = top;
    args[wave] = arg;
  }
  __syncthreads();
  for (int i = 0; i < kThreads / 64; ++i) larger(top, arg, tops[i], args[i]);
  double sum = 0.;
#pragma unroll
  for (int i = 0; i < kEach; ++i) sum += weight_of(x[i], first + i, top, arg, scale2);
  sum = sum_all(sum, part);
  if (tid == 0) a.sums[((int64_t)a.row0 + row) * a.pieces + piece] = PieceSum{sum, top, arg};
}

// ---------------------------------------------------------------------------
// The walk: a workgroup takes a sequence.  First every draft's row is put together and
// its token's share of the row that judges it read, all at once; then the drafts are
// tried in order, which every thread does alike.  A draft that is rejected and was
// drawn, with others to come that were drawn from the same distribution, takes a pass
// over the row for the sum of what is left.
// ---------------------------------------------------------------------------
constexpr int kWalkers = 1024;

// What r holds of token y after `turns` rejections of drawn drafts.
__device__ __forceinline__ double after(double r, double q, const double* norms, int turns) {
  for (int i = 0; i < turns; ++i) r = fmax(r - q, 0.) / norms[i];
  return r;
}

template <int TYPE>
__global__ void __launch_bounds__(kWalkers) verify_walk_kernel(VerifyArgs a) {
  __shared__ double total[kMaxDrafts], share[kMaxDrafts], part[kWalkers / 64], turns[kMaxDrafts];
  __shared__ float top[kMaxDrafts], from[kMaxDrafts], lot[kMaxDrafts];
  __shared__ int arg[kMaxDrafts], parent[kMaxDrafts], token[kMaxDrafts];
  const int tid = threadIdx.x, l = tid & 63, wave = tid >> 6;
  const int b = blockIdx.x, tok = a.row0 + a.tok[b], nq = a.tok[b + 1] - a.tok[b];
  const double scale2 = a.scale2[b];
  if (nq == 0) {
    if (tid == 0) {
      a.count[a.b0 + b] = 0;
      if (a.finals) a.finals[a.b0 + b].rejected = -1;
    }
    return;
  }
  // Rows: a wave puts one together at a time.
  for (int i = wave; i < nq; i += kWalkers / 64) {
    const PieceSum* s = a.sums + ((int64_t)tok + i) * a.pieces;
    float t = -INFINITY;
    int g = INT32_MAX;
    double sum = 0.;
    for (int k = l; k < a.pieces; k += 64) larger(t, g, s[k].top, s[k].arg);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) larger(t, g, __shfl_xor(t, o), __shfl_xor(g, o));
    for (int k = l; k < a.pieces; k += 64)
      sum += scale2 == 0.      ? (s[k].arg == g ? 1. : 0.)
             : s[k].sum == 0. ? 0.
             : s[k].top == t  ? s[k].sum
                              : s[k].sum * pow2(((double)s[k].top - t) * scale2);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    if (l == 0) {
      total[i] = t == -INFINITY ? 0. : sum;
      top[i] = t;
      arg[i] = g;
    }
  }
  if (tid < nq) {
    const int p = a.parent[tok + tid], x = a.token[tok + tid];
    parent[tid] = p >= 0 && p < tid && x >= 0 && x < a.vocab ? p : -1;
    token[tid] = x;
    lot[tid] = a.uniform[tok + tid];
  }
  __syncthreads();
  if (tid < nq && parent[tid] >= 0) {
    const int p = parent[tid], x = token[tid];
    float y = one_of<TYPE>(row_of<TYPE>(a, tok + p), x);
    y = y == y ? y : -INFINITY;
    share[tid] = total[p] == 0. ? 0. : weight_of(y, x, top[p], arg[p], scale2);
    from[tid] = a.drawn ? some(a.drawn[(int64_t)(tok + p) * a.drawn_row + x]) : 0.f;
  }
  __syncthreads();

  int here = 0, n = 1, rejected = 0;
  double covered = 0.;
  bool pending = false;  // whether the last rejection's sum is not known yet
  if (tid == 0) a.path[tok] = 0;
  for (int i = 1; i < nq; ++i) {
    if (parent[i] != here) continue;
    const double u = chance(lot[i]), sum = total[here];
    bool taken, changed = false;
    if (sum == 0.) break;  // nothing has any probability
    if (!a.drawn) {
      bool again = false;
      for (int k = 0; k < rejected; ++k) again |= (int)turns[k] == token[i];
      const double r = again ? 0. : share[i];
      taken = u * (sum - covered) < r;
      if (!taken && r > 0. && sum - covered - r > 0.) {
        covered += r;
        changed = true;
      }
      __syncthreads();
      if (changed && tid == 0) turns[rejected] = token[i];
      rejected += changed;
      __syncthreads();
    } else {
      if (pending) {  // the sum of what the last rejection left
        const void* row = row_of<TYPE>(a, tok + here);
        const float* q = a.drawn + (int64_t)(tok + here) * a.drawn_row;
        double left = 0.;
        for (int y = tid; y < a.vocab; y += kWalkers) {
          float x = one_of<TYPE>(row, y);
          x = x == x ? x : -INFINITY;
          const double w = weight_of(x, y, top[here], arg[here], scale2) / sum, d = some(q[y]);
          left += fmax(after(w, d, turns, rejected) - d, 0.);
        }
        left = sum_all(left, part);
        __syncthreads();
        if (left > 0. && tid == 0) turns[rejected] = left;
        rejected += left > 0.;
        pending = false;
        __syncthreads();
      }
      const double d = from[i], r = after(share[i] / sum, d, turns, rejected);
      taken = u * d < r;
      pending = !taken;
    }
    if (taken) {
      here = i;
      if (tid == 0) a.path[tok + n] = i;
      ++n;
      rejected = 0;
      covered = 0.;
      pending = false;
    }
  }
  for (int k = tid; k < rejected; k += kWalkers) a.turns[tok + k] = turns[k];
  if (tid == 0) {
    a.count[a.b0 + b] = n;
    const bool none = total[here] == 0.;
    if (none) a.next[a.b0 + b] = -1;
    a.finals[a.b0 + b] = Final{total[here], top[here], arg[here], tok + here,
                               none ? -1 : 2 * rejected + pending, 0, 0};
  }
}

// ---------------------------------------------------------------------------
// The last row: each workgroup adds up one piece of what is left of it, and the one that
// comes last of a sequence's finds the piece in which the random number falls, and the
// token there.
// ---------------------------------------------------------------------------
template <int TYPE>
__global__ void __launch_bounds__(kThreads) verify_next_kernel(VerifyArgs a) {
  __shared__ double part[kThreads / 64], scan[kThreads / 64], turns[kMaxDrafts];
  __shared__ double found_before;
  __shared__ int found, lowest[kThreads / 64];
  __shared__ bool last;
  const int tid = threadIdx.x, l = tid & 63, wave = tid >> 6;
  const int b = blockIdx.x / (uint32_t)a.pieces, piece = blockIdx.x - b * a.pieces;
  Final* const f = a.finals + a.b0 + b;
  if (f->rejected < 0) return;
  const int rejected = f->rejected >> 1, row = f->row, arg = f->arg;
  const bool pending = f->rejected & 1;
  const float top = f->top;
  const double scale2 = a.scale2[b], total = f->total;
  const int first_row = a.row0 + a.tok[b];
  for (int k = tid; k < rejected; k += kThreads) turns[k] = a.turns[first_row + k];
  __syncthreads();
  const void* p = row_of<TYPE>(a, row);
  const float* q = a.drawn ? a.drawn + (int64_t)row * a.drawn_row : nullptr;
  const int lead = lead_of<TYPE>(p);

  // What this thread's tokens of a piece hold, and held before the last rejection.
  double now[kEach], was[kEach];
  auto weigh = [&](int piece) {
    const int first = piece * kPiece + tid * kEach - lead;
    float x[kEach];
    load<TYPE>(p, first, a.vocab, x);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int y = first + i;
      was[i] = weight_of(x[i], y, top, arg, scale2);
      if (y < 0 || y >= a.vocab) was[i] = 0.;
      now[i] = was[i];
      if (q) {
        const double d = y >= 0 && y < a.vocab ? some(q[y]) : 0.f;
        was[i] = after(was[i] / total, d, turns, rejected);
        now[i] = pending ? fmax(was[i] - d, 0.) : was[i];
      }
    }
    if (!q)
      for (int k = 0; k < rejected; ++k) {
        const int y = (int)turns[k] - first;
#pragma unroll
        for (int i = 0; i < kEach; ++i) now[i] = i == y ? 0. : now[i];
      }
  };
  weigh(piece);
  double x = 0., y = 0.;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    x += now[i];
    y += was[i];
  }
  x = sum_all(x, part);
  y = sum_all(y, part);
  double* const left = a.left + (int64_t)(a.b0 + b) * a.pieces * 2;
  if (tid == 0) {
    __hip_atomic_store(left + 2 * piece, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(left + 2 * piece + 1, y, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    last = __hip_atomic_fetch_add(&f->arrived, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) ==
           a.pieces - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();

  // The pieces' sums, 64 at a time, in each wave alike.  What the last rejection leaves
  // counts, unless that is nothing.
  auto held = [&](int k, int which) {
    return k < a.pieces ? __hip_atomic_load(left + 2 * k + which, __ATOMIC_RELAXED,
                                            __HIP_MEMORY_SCOPE_AGENT)
                        : 0.;
  };
  double all[2] = {0., 0.};
  for (int k = l; k < a.pieces; k += 64) {
    all[0] += held(k, 0);
    all[1] += held(k, 1);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    all[0] += __shfl_xor(all[0], o);
    all[1] += __shfl_xor(all[1], o);
  }
  const int which = all[0] > 0. ? 0 : 1;
  const double goal = chance(a.uniform[first_row]) * all[which];
  double before = 0., sum = 0.;
  int at = -1;  // the first piece whose sum passes the goal, or the last that holds anything
  for (int k = 0; k < a.pieces; k += 64) {
    const double z = held(k + l, which);
    double up = z;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double y = __shfl_up(up, o);
      up += l >= o ? y : 0.;
    }
    const uint64_t past = __ballot(z > 0. && sum + up > goal), any = __ballot(z > 0.);
    if (any) {
      const int i = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(any);
      at = k + i;
      before = sum + __shfl(up - z, i);
    }
    if (past) break;
    sum += __shfl(up, 63);
  }
  if (at < 0) {
    if (tid == 0) a.next[a.b0 + b] = -1;
    return;
  }
  weigh(at);
  double mine = 0.;
#pragma unroll
  for (int i = 0; i < kEach; ++i) mine += which ? was[i] : now[i];
  double up = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double z = __shfl_up(up, o);
    up += l >= o ? z : 0.;
  }
  if (l == 63) scan[wave] = up;
  __syncthreads();
  double start = before;
  for (int i = 0; i < wave; ++i) start += scan[i];
  start += up - mine;
  // The first token whose sum passes the goal, in the first thread that has one; or the
  // last that holds anything.
  int hit = INT32_MAX, end = -1;
  double run = start;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const double z = which ? was[i] : now[i];
    const int token = at * kPiece + tid * kEach - lead + i;
    run += z;
    if (z > 0.) {
      end = token;
      if (run > goal && hit == INT32_MAX) hit = token;
    }
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    hit = min(hit, __shfl_xor(hit, o));
    end = max(end, __shfl_xor(end, o));
  }
  __syncthreads();
  if (l == 0) {
    lowest[wave] = hit;
    scan[wave] = end;
  }
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < kThreads / 64; ++i) {
      hit = min(hit, lowest[i]);
      end = max(end, (int)scan[i]);
    }
    a.next[a.b0 + b] = hit != INT32_MAX ? hit : end;
  }
}

template <typename F>
hipError_t by_type(const VerifyArgs& a, F f, uint32_t groups, int threads, hipStream_t s) {
  void* args[] = {const_cast<VerifyArgs*>(&a)};
  return hipLaunchKernel(f(a.type), dim3(groups), dim3(threads), args, 0, s);
}

}  // namespace

hipError_t launch_verify_sums(const VerifyArgs& a, hipStream_t s) {
  return by_type(a, [](int t) {
    return t == 0   ? (const void*)&verify_sums_kernel<0>
           : t == 1 ? (const void*)&verify_sums_kernel<1>
                    : (const void*)&verify_sums_kernel<2>;
  }, (uint32_t)a.tok[kQSeqs] * a.pieces, kThreads, s);
}
hipError_t launch_verify_walk(const VerifyArgs& a, hipStream_t s) {
  return by_type(a, [](int t) {
    return t == 0   ? (const void*)&verify_walk_kernel<0>
           : t == 1 ? (const void*)&verify_walk_kernel<1>
                    : (const void*)&verify_walk_kernel<2>;
  }, (uint32_t)a.nseq, kWalkers, s);
}
hipError_t launch_verify_next(const VerifyArgs& a, hipStream_t s) {
  return by_type(a, [](int t) {
    return t == 0   ? (const void*)&verify_next_kernel<0>
           : t == 1 ? (const void*)&verify_next_kernel<1>
                    : (const void*)&verify_next_kernel<2>;
  }, (uint32_t)a.nseq * a.pieces, kThreads, s);
}

}  // namespace dv
