// Attention over an 8-bit cache: e4m3 codes, a power-of-two scale per block.
//
// Codes become f16 or bf16 (the queries' type) as they enter the matrix units:
// the conversion multiplies by the scale, and code * 2^e is exact in both types
// within their range, so neither keys nor values are rounded a second time.
// Scores come out transposed, S^T = K Q^T, tokens down and queries across: a
// lane then holds several tokens of one query, which is how the second product,
// O^T = V^T P^T, wants its right operand, so probabilities never leave their
// registers.  (The order of tokens along that product's inner axis is free as
// long as V follows it.)
//
// Softmax runs in one pass in powers of two: s2 = score * log2(e), a reference m
// per query and sums relative to it.  m is set kLift below the largest score and
// moves only when a score exceeds that by more than 8, so the common step needs no
// exchange between lanes and no rescaling; probabilities then reach 2^(8 + kLift)
// at most, which costs no precision.  kLift is 7 for probabilities in f16, which stay
// normal numbers down to 2^-21 of the largest so (a value 2^12 times another's
// shows their rounding below 2^-14 otherwise), and -32 for those in bf16, which has
// f32's range: their sums with values up to f32's largest stay below it.
#include <algorithm>
#include <type_traits>

#include "dv_attn_internal.h"

namespace dv {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// "No score yet", the lowest number; a hidden score is -infinity.
constexpr float kLow = -3.402823466e38f;
constexpr float kLn2 = 0.69314718055994531f, kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.f;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

template <bool BF16>
struct Ty;
template <>
struct Ty<false> {
  static constexpr float kLift = 7.f;
  // bytes 0, 1 (or 2, 3) of w, times the scale
  template <bool HI>
  static __device__ __forceinline__ uint32_t cvt(uint32_t w, float s) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, HI));
  }
  // What f16 does not hold (a cache rounded from bf16) becomes its largest number: an
  // infinity would be NaN to every row that gives it a probability of 0, hidden
  // or not.  The largest scale whose products with all codes f16 holds, and two
  // converted numbers made finite:
  static constexpr float kHeld = 128.f;
  static __device__ __forceinline__ uint32_t finite(uint32_t w) {
    return w - ((w & 0x7fffu) == 0x7c00u) - ((uint32_t)((w & 0x7fff0000u) == 0x7c000000u) << 16);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
  }
  static __device__ __forceinline__ float lo(uint32_t w) {
    return (float)__builtin_bit_cast(f16x2, w)[0];
  }
  static __device__ __forceinline__ float hi(uint32_t w) {
    return (float)__builtin_bit_cast(f16x2, w)[1];
  }
  static __device__ __forceinline__ f32x4 mma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Ty<true> {
  static constexpr float kLift = -32.f;
  template <bool HI>
  static __device__ __forceinline__ uint32_t cvt(uint32_t w, float s) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, HI));
  }
  static constexpr float kHeld = INFINITY;  // (bf16 holds what f32 does)
  static __device__ __forceinline__ uint32_t finite(uint32_t w) { return w; }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
  }
  static __device__ __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
  static __device__ __forceinline__ float hi(uint32_t w) {
    return __uint_as_float(w & 0xffff0000u);
  }
  static __device__ __forceinline__ f32x4 mma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};

// The sequence that holds work item `item` (as find_seq of the streaming
// kernels: the count of first items at or below it names it).  Lanes load their
// sequences' entries together, so that the common launch of up to 64 sequences
// waits for memory once.
struct Seq {
  int b, k;           // index in the launch; the item's index in the sequence
  int len, tok, nq;   // tokens in the cache; queries of earlier sequences; its own
};
__device__ __forceinline__ Seq seq_of(const AttendArgs& a, int item) {
  const int lane = threadIdx.x & 63;
  const int first = a.item[lane], len = a.len[lane], t0 = a.tok[lane], t1 = a.tok[lane + 1];
  Seq q;
  q.b = __popcll(__ballot(first <= item)) - 1;
  if (q.b == 63 && a.nseq > 64) {
    for (int i = 64; i < a.nseq; i += 64) q.b += __popcll(__ballot(a.item[i + lane] <= item));
    q.b = __builtin_amdgcn_readfirstlane(q.b);
    q.k = item - a.item[q.b];
    q.len = a.len[q.b];
    q.tok = a.tok[q.b];
    q.nq = a.tok[q.b + 1] - q.tok;
    return q;
  }
  q.k = item - __builtin_amdgcn_readlane(first, q.b);
  q.len = __builtin_amdgcn_readlane(len, q.b);
  q.tok = __builtin_amdgcn_readlane(t0, q.b);
  q.nq = __builtin_amdgcn_readlane(t1, q.b) - q.tok;
  return q;
}

// log2 of the sum of a row's exponentials, from its sum relative to m.  (The lift is
// taken off first: a logarithm of its size would have as many bits fewer.)
__device__ __forceinline__ float lse2_of(float m, float sum, float lift) {
  return (m + lift) + __log2f(sum * exp2_(-lift));
}

// Positions as numbers in 32 bits: less the last token's, so that distances are exact
// up to 2^24 tokens back, however late in a text they stand.  (Slots are at most 2^24.)
__device__ __forceinline__ int last_position(const QLayout& q, const float* slopes, int64_t slots,
                                             int len) {
  return slopes && q.position && len > 0 ? q.position[slots + len - 1] : 0;
}
__device__ __forceinline__ float from_last(int position, int last) {
  return (float)(int)((uint32_t)position - (uint32_t)last);
}

// A value known to be the same in all lanes, as a scalar (quotients are not seen to be).
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Called on products' results before any branch: ends the wait for them in the
// block of the products.  Left to itself, the compiler (ROCm 7.2) counts the wait
// states between a product and the first read of its result along one path only
// where an `if` without `else` comes between, and read the last register too
// early on the path that skips it.
template <typename V>
__device__ __forceinline__ void settle(V& a) {
  asm volatile("s_nop 12" : "+v"(a));
}

// A barrier after which the workgroup's LDS writes are seen; unlike
// __syncthreads it leaves loads from memory in flight.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The sum over the 32 lanes of a half wave, in all of them: a row of 16 by
// rotations, then the two rows.
__device__ __forceinline__ float sum_of_half(float x) {
  auto turned = [](float v, auto by) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + decltype(by)::value,
                                                      0xf, 0xf, false));  // row_ror
  };
  x += turned(x, std::integral_constant<int, 8>{});
  x += turned(x, std::integral_constant<int, 4>{});
  x += turned(x, std::integral_constant<int, 2>{});
  x += turned(x, std::integral_constant<int, 1>{});
  return x + __shfl_xor(x, 16);
}

// 0x80 in each byte of w that is a NaN code.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
}

// NaN values of tokens that are hidden from some rows leave the products (as
// zeros), since 0 times NaN is NaN.  Once the results are written this makes NaN
// of those that they belong to: rows [r0, r0 + nr) that see such a token of
// [from, to).  `part`: sums of a split (rows of DP), or null: the call's results.
__device__ __forceinline__ void spread_nan(const AttendArgs& a, int sb, int h, int len, int nq,
                                        int tok, int from, int to, int r0, int nr, float* part,
                                        int DP) {
  const QLayout& q = a.q;
  const uint8_t* vb = q.codes + (2 * (int64_t)a.layer + 1) * q.s_slab + sb * q.s_b + h * q.s_h;
  for (int x = threadIdx.x; x < nr * q.D; x += kThreads) {
    const int r = x / q.D, d = x - r * q.D, i = (r0 + r) / a.G, head = h * a.G + r0 + r - i * a.G;
    bool nan = false;
    for (int t = from; t < min(to, len - nq + i + 1); ++t) {
      const int j = q.d_bs.div(t);
      const int64_t blk = q.bt ? q.bt[(int64_t)sb * q.max_blocks + j] : j;
      if (q.bt && (uint64_t)blk >= (uint64_t)q.num_blocks) continue;
      nan |= (vb[blk * q.s_blk + (int64_t)(t - j * q.bs) * q.D + d] & 127) == 127;
    }
    if (!nan) continue;
    if (part)
      part[(int64_t)r * DP + d] = NAN;
    else
      ((uint16_t*)a.out)[(int64_t)(tok + i) * a.o_token + (int64_t)head * a.o_head + d] = 0x7fff;
  }
}

// The weights of a chunk's tokens [c0, c0 + cn) from the scores that were kept, four
// tokens to a lane, and its nr rows' lse2 (in LDS).  Short chunks deal the rows to
// as many groups of lanes as there are, whose sums are added in order (`part`, 4 KB
// of LDS).
__device__ __forceinline__ void add_weights(const AttendArgs& a, const Seq& seq, int sb, int h,
                                            int nr, int c0, int cn, const float* lse2s,
                                            f32x4* part) {
  const QLayout& q = a.q;
  const int64_t pitch = (seq.len + 31) & ~31;
  const float* sc = a.scores + (int64_t)a.soff[seq.b] * 32 + (int64_t)h * nr * pitch;
  float* weight = q.weight + (((int64_t)a.layer * q.batch + sb) * q.heads + h) * (int64_t)q.cap;
  const int tid = threadIdx.x;
  int lanes = kThreads;
  while (lanes > 32 && lanes * 2 >= cn) lanes >>= 1;  // half as many still cover the chunk
  const int groups = kThreads / lanes, group = tid / lanes, lane = tid & (lanes - 1);
  for (int t0 = 0; t0 < cn; t0 += lanes * 4) {  // (scores are padded to 32 tokens)
    const int t = t0 + lane * 4;
    f32x4 w = {0, 0, 0, 0};
    if (t < cn) {
#pragma unroll 8
      for (int r = group; r < nr; r += groups) {
        const f32x4 s2 = *(const f32x4*)(sc + r * pitch + c0 + t);
#pragma unroll
        for (int i = 0; i < 4; ++i)  // hidden tokens get 0 also where lse is NaN
          w[i] += s2[i] == -INFINITY ? 0.f : exp2_(s2[i] - lse2s[r]);
      }
    }
    if (groups > 1) {  // (one step: the lanes of a group cover the chunk)
      part[tid] = w;
      __syncthreads();
      for (int g = 1; g < groups; ++g) w += part[g * lanes + lane];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (group == 0 && t + i < cn) {
        float* to = weight + c0 + t + i;
        *to = a.decay == 0.f ? w[i] : a.decay * *to + w[i];
      }
  }
}

// ---------------------------------------------------------------------------
// Few rows (decode steps): a workgroup takes a chunk of one head's tokens, its
// four waves 32 tokens at a time in turn; 16x16x32 products, queries in RT tiles
// of 16 columns.
// Each wave copies its own steps' codes from memory to LDS, whole rows at a time
// and without passing through registers: the next step's keys as soon as these
// have been read, its values likewise.  No barrier is needed.
// 16-byte pieces of a row are stored at (piece ^ key(token)), which spreads both
// kinds of reads over the banks.  Keys are read as the left operand wants them
// (lane: token l % 16, 16 bytes); values by the transposing read, which gives a
// lane eight tokens of one dim.
// Codes become 16-bit numbers as they are, without their scales: a key's scale
// multiplies its score, a value's its probability, both in 32 bits.  The second
// product runs in bf16 for either type (codes are exact in it, and so is the
// range of scaled probabilities), with each probability as the sum of two
// numbers, which keeps 16 bits of it; the matrix unit has time to spare.
// Bound by HBM and, per workgroup, by what comes before the first product (table
// entries, scales, the first codes, one after another) and after the last (the
// waves' results): 32 sequences of 128 to 4096 tokens, 8 heads, 140 MB 29 us, 4.8
// TB/s; one of 131071, 273 MB (and 34 MB of scores written) 62 us, 4.9 TB/s.  A
// wave lives for 54 % of the first and 72 % of the second; 59 % of the 56 us of 64
// rows (143 MB), whose registers hold two workgroups a CU.
// ---------------------------------------------------------------------------
// 16 bytes a lane from memory to LDS: to lds + 16 * lane.
template <bool NT>
__device__ __forceinline__ void copy_to_lds(const uint8_t* from, uint32_t lds) {
  if constexpr (NT)
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt"
                 ::"v"(from), "s"(lds)
                 : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
                 ::"v"(from), "s"(lds)
                 : "memory", "m0");
}
// Waits until at most N of this wave's accesses to memory are on their way.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// Waits for this wave's LDS reads.
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

__device__ __forceinline__ u32x2 read_tr8(const uint8_t* p) {
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)p));
}

template <bool BF16, int DP, int RT>
__global__ void __launch_bounds__(kThreads, split_waves(DP, RT))
    attend_split_kernel(AttendArgs a, int direct) {
  using T = Ty<BF16>;
  using B = Ty<true>;
  constexpr int CH = DP / 16, KS = DP / 32, OJ = DP / 16;
  constexpr int kHalf = kSplitStep * DP;  // bytes of a step's keys, or values
  constexpr bool kInLds = split_queries(DP, RT) > 0;  // the queries
  constexpr int kLoads = kHalf / 1024;  // copies of a half
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  const QLayout& q = a.q;
  const int tid = threadIdx.x, l = tid & 63, c = l & 15, g = l >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  const int item = blockIdx.x;
  const Seq seq = seq_of(a, item);
  const int b = seq.b, sb = a.b0 + b, len = seq.len, nq = seq.nq, rows = nq * a.G;
  const int nsplit = max(1, scalar((len + a.chunk - 1) / a.chunk));
  const int h = scalar(seq.k / nsplit), c0 = (seq.k - h * nsplit) * a.chunk;
  const int cn = min(a.chunk, len - c0);  // tokens of this chunk

  uint8_t* const kl = lds + wave * 2 * kHalf;
  uint8_t* const vl = kl + kHalf;
  u32x4* const ql = (u32x4*)(lds + 8 * kHalf) + l;  // [tile][product][lane]
  float* const tables = (float*)(lds + 8 * kHalf + split_queries(DP, RT));
  uint32_t* off = (uint32_t*)tables;  // each token's row, in 16 bytes from the head's base
  float* ks = tables + a.chunk;       // key scales times the scores' factor; NaN: unmapped
  float* vs = tables + 2 * a.chunk;   // value scales
  float* pos = tables + 3 * a.chunk;
  f32x4* columns = (f32x4*)(tables + (a.slopes ? 4 : 3) * a.chunk);  // limit, slope, position
  int* odd = (int*)(columns + RT * 16);
  const int64_t slab = 2 * (int64_t)a.layer;
  const uint8_t* kb = q.codes + slab * q.s_slab + sb * q.s_b + h * q.s_h;
  const uint8_t* vb = kb + q.s_slab;
  const float* sk = q.scale + slab * q.c_slab + sb * q.c_b + h * q.c_h;
  const int64_t slots = (((int64_t)a.layer * q.batch + sb) * q.heads + h) * (int64_t)q.cap;
  const int last_at = last_position(q, a.slopes, slots, len);
  int bad = 0;
  for (int i = tid; i < ((cn + kSplitStep - 1) & -kSplitStep); i += kThreads) {
    const int t = min(c0 + i, len - 1), j = q.d_bs.div(t);
    int64_t blk = j;
    bool hole = false;
    if (q.bt) {
      blk = q.bt[(int64_t)sb * q.max_blocks + j];
      hole = (uint64_t)blk >= (uint64_t)q.num_blocks;
      blk = hole ? 0 : blk;
    }
    off[i] = (uint32_t)((blk * q.s_blk + (int64_t)(t - j * q.bs) * q.D) >> 4);
    ((int*)ks)[i] = hole ? -1 : (int)blk;
    if (a.slopes) pos[i] = q.position ? from_last(q.position[slots + t], last_at) : (float)t;
    bad |= hole;
  }

  // The queries, and what each column (row c of tile rt) may see.
  u32x4 qr[kInLds ? 1 : RT][KS];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = rt * 16 + c, i = r / a.G, head = h * a.G + (r - i * a.G);
    const bool on = r < rows;
    const uint16_t* src = (const uint16_t*)a.query +
                          (int64_t)(on ? seq.tok + i : 0) * a.q_token + (int64_t)head * a.q_head;
    const bool mine = rt % 4 == wave;  // what goes to LDS is one wave's to read
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int d = (s >> 1) * 64 + g * 16 + (s & 1) * 8;
      const u32x4 x = on && d < q.D && (!kInLds || mine) ? *(const u32x4*)(src + d)
                                                         : u32x4{0, 0, 0, 0};
      if constexpr (!kInLds) qr[rt][s] = x;
      if (kInLds && mine) ql[(rt * KS + s) * 64] = x;
    }
    if (mine && g == 0) {
      const int limit = on ? len - nq + i : -1;
      float slope = 0.f, here = 0.f;
      if (a.slopes && limit >= 0) {
        slope = a.slopes[head] * kLog2e;
        here = q.position ? from_last(q.position[slots + limit], last_at) : (float)limit;
      }
      columns[r] = f32x4{__int_as_float(limit), slope, here, 0.f};
    }
  }
  // (LDS is all that the workgroup shares so far: loads may stay in flight)
  const bool any_bad = __any(bad);
  if (l == 0) odd[wave] = any_bad;
  lds_barrier();
  const bool holes = odd[0] | odd[1] | odd[2] | odd[3];
  const int all_see = len - nq;  // slots up to this one are seen by every row

  // Copy n of a half: tokens n * 64 / CH ..., lane's token l / CH of them, piece
  // l % CH of its place.  Pieces past head_dim repeat the row's first one: they
  // meet zeros of the queries, or make dims that are not written.
  auto key_of = [](int tok) { return tok / (16 / CH) & (CH - 1); };
  const uint32_t k_to = __builtin_amdgcn_readfirstlane(
      (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)kl);
  uint32_t piece[kLoads];
#pragma unroll
  for (int n = 0; n < kLoads; ++n) {
    piece[n] = (l % CH) ^ key_of(n * (64 / CH) + l / CH);
    piece[n] = (int)piece[n] * 16 < q.D ? piece[n] : 0;
  }
  auto fetch = [&](const uint8_t* from, uint32_t to, int t) {
    const uint32_t* row = off + t + l / CH;
    uint32_t at[kLoads];
#pragma unroll
    for (int n = 0; n < kLoads; ++n) at[n] = row[n * (64 / CH)] + piece[n];
    wait_lds();
    if (a.nt) {
#pragma unroll
      for (int n = 0; n < kLoads; ++n)
        copy_to_lds<true>(from + (uint64_t)at[n] * 16, to + n * 1024);
    } else {
#pragma unroll
      for (int n = 0; n < kLoads; ++n)
        copy_to_lds<false>(from + (uint64_t)at[n] * 16, to + n * 1024);
    }
  };

  f32x4 o[RT][OJ];
  float m[RT], sum[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = kLow;
    sum[rt] = 0.f;
#pragma unroll
    for (int j = 0; j < OJ; ++j) o[rt][j] = f32x4{0, 0, 0, 0};
  }
  const int64_t pitch = (len + 31) & ~31;
  int nan_from = INT32_MAX, nan_to = 0;  // where values became zeros (spread_nan)
  // where this lane reads: its keys' row, and its row of a transposed read
  const int krow = c * DP, kkey = key_of(c);
  const int vtok = (l & 15) >> 1, vrow = (vtok < 4 ? g * 4 + vtok : 12 + g * 4 + vtok);
  const int vkey = key_of(vrow);
  const uint8_t* const vread = vl + vrow * DP + (l & 1) * 8;

  // Stores count as accesses on their way, in order: none before the wait for the
  // values, unless the scores' registers are wanted.
  constexpr bool kLate = RT == 1;
  auto store_scores = [&](f32x4 (&s)[RT][2], int first) {
    if (!a.weigh) return;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      if (rt * 16 + c >= rows) continue;
      float* to = a.scores + (int64_t)a.soff[b] * 32 +
                  ((int64_t)h * rows + rt * 16 + c) * pitch + first;
      *(f32x4*)to = s[rt][0];
      *(f32x4*)(to + 16) = s[rt][1];
    }
  };
  auto step = [&](int t, bool more) {
    wait_loads<kLoads>();  // the keys; the values may still come
    f32x4 s[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) s[rt][0] = s[rt][1] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < KS / 2; ++i) {
      u32x4 x[2];
#pragma unroll
      for (int u = 0; u < 2; ++u)  // 16 tokens on the key is the same
        x[u] = *(const u32x4*)(kl + u * 16 * DP + krow + (((g + 4 * i) ^ kkey) << 4));
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        u32x4 y[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
          y[u] = u32x4{T::template cvt<false>(x[u][2 * e], 1.f), T::template cvt<true>(x[u][2 * e], 1.f),
                       T::template cvt<false>(x[u][2 * e + 1], 1.f),
                       T::template cvt<true>(x[u][2 * e + 1], 1.f)};
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const u32x4 z = kInLds ? ql[(rt * KS + 2 * i + e) * 64] : qr[kInLds ? 0 : rt][2 * i + e];
          s[rt][0] = T::mma16(y[0], z, s[rt][0]);
          s[rt][1] = T::mma16(y[1], z, s[rt][1]);
        }
      }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      settle(s[rt][0]);
      settle(s[rt][1]);
    }
    if (more) fetch(kb, k_to, t + kSplitRound);
    const int first = c0 + t + g * 4;  // this lane's tokens: first + 16 u + r
    const bool mask = holes || c0 + t + kSplitStep - 1 > all_see;
    const f32x4 kscale[2] = {*(const f32x4*)(ks + t + g * 4), *(const f32x4*)(ks + t + 16 + g * 4)};
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
      for (int u = 0; u < 2; ++u) s[rt][u] = s[rt][u] * kscale[u];
      if (a.slopes) {
        const f32x4 column = columns[rt * 16 + c];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const f32x4 at = *(const f32x4*)(pos + t + u * 16 + g * 4);
#pragma unroll
          for (int r = 0; r < 4; ++r) s[rt][u][r] += column[1] * (at[r] - column[2]);
        }
      }
      if (mask) {
        const int limit = __float_as_int(columns[rt * 16 + c][0]);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const bool sees = first + u * 16 + r <= limit && kscale[u][r] == kscale[u][r];
            s[rt][u][r] = sees ? s[rt][u][r] : -INFINITY;
          }
      }
      float most = s[rt][0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) most = fmaxf(most, s[rt][i >> 2][i & 3]);
      if (__any(most > m[rt] + (kSlack + B::kLift))) {
        float up = fmaxf(most - B::kLift, m[rt]);
        up = fmaxf(up, __shfl_xor(up, 16));
        up = fmaxf(up, __shfl_xor(up, 32));
        const float f = exp2_(m[rt] - up);
        m[rt] = up;
        sum[rt] *= f;
#pragma unroll
        for (int j = 0; j < OJ; ++j) o[rt][j] = o[rt][j] * f;
      }
    }
    if (!kLate) store_scores(s, first);
    const f32x4 vscale[2] = {*(const f32x4*)(vs + t + g * 4), *(const f32x4*)(vs + t + 16 + g * 4)};
    u32x4 hi[RT], lo[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int u = i >> 1, r = (2 * i) & 3;
        float p0 = exp2_(s[rt][u][r] - m[rt]), p1 = exp2_(s[rt][u][r + 1] - m[rt]);
        sum[rt] += p0 + p1;
        p0 *= vscale[u][r];
        p1 *= vscale[u][r + 1];
        hi[rt][i] = B::pack(p0, p1);
        lo[rt][i] = B::pack(p0 - B::lo(hi[rt][i]), p1 - B::hi(hi[rt][i]));
      }
    }
    if (more && (kLate || !a.weigh))
      wait_loads<kLoads>();  // the values; the next keys may still come
    else
      wait_loads<0>();
    if (mask) {
      uint32_t any = 0;
#pragma unroll
      for (int n = 0; n < kLoads; ++n) {
        u32x4* const at = (u32x4*)(vl + n * 1024 + l * 16);
        u32x4 w = *at;
        uint32_t nan = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t x = nan_bytes(w[e]);
          nan |= x;
          w[e] &= ~((x >> 7) * 0xffu);
        }
        if (nan) *at = w;
        any |= nan;
      }
      if (__any(any != 0)) {
        nan_from = min(nan_from, c0 + t);
        nan_to = c0 + t + kSplitStep;
      }
      wait_lds();
    }
    u32x2 w[OJ];
#pragma unroll
    for (int j = 0; j < OJ; ++j) w[j] = read_tr8(vread + ((j ^ vkey) << 4));
#pragma unroll
    for (int j = 0; j < OJ; ++j) {
      const u32x4 v = {B::cvt<false>(w[j][0], 1.f), B::cvt<true>(w[j][0], 1.f),
                       B::cvt<false>(w[j][1], 1.f), B::cvt<true>(w[j][1], 1.f)};
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) o[rt][j] = B::mma16(v, hi[rt], o[rt][j]);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) o[rt][j] = B::mma16(v, lo[rt], o[rt][j]);
    }
    if (kLate) store_scores(s, first);
    if (more) fetch(vb, k_to + kHalf, t + kSplitRound);
  };

  int t = wave * kSplitStep;
  if (t < cn) {
    fetch(kb, k_to, t);
    fetch(vb, k_to + kHalf, t);
  }
  // The scales follow the first codes: both are on their way at once.
  for (int i = tid; i < ((cn + kSplitStep - 1) & -kSplitStep); i += kThreads) {
    const int blk = ((const int*)ks)[i];
    // (a probability of 0 times a scale that nothing wrote may be NaN)
    ks[i] = blk < 0 ? NAN : sk[blk * q.c_blk] * a.scale2;
    vs[i] = blk < 0 ? 0.f : sk[blk * q.c_blk + q.c_slab];
  }
  lds_barrier();
  for (; t < cn; t += kSplitRound) step(t, t + kSplitRound < cn);

  // Join the four waves.
  __syncthreads();  // the tables are done with
  float* sums = (float*)lds;                      // [wave][16][DP]
  float* mls = sums + 4 * 16 * DP;                // [wave][RT * 16][2]
  int* nans = (int*)(mls + 4 * RT * 16 * 2);      // [wave][2]
  if (l == 0) {
    nans[wave * 2] = nan_from;
    nans[wave * 2 + 1] = nan_to;
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    sum[rt] += __shfl_xor(sum[rt], 16);
    sum[rt] += __shfl_xor(sum[rt], 32);
    if (g == 0) {
      mls[(wave * RT * 16 + rt * 16 + c) * 2] = m[rt];
      mls[(wave * RT * 16 + rt * 16 + c) * 2 + 1] = sum[rt];
    }
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    __syncthreads();
    if (rt * 16 >= rows) break;
    float most = kLow;
    for (int w = 0; w < 4; ++w) most = fmaxf(most, mls[(w * RT * 16 + rt * 16 + c) * 2]);
    const float f = exp2_(m[rt] - most);
    if (rt * 16 + c < rows)
#pragma unroll
      for (int j = 0; j < OJ; ++j)  // dims 16 j + 4 g ...
        *(f32x4*)(sums + (wave * 16 + c) * DP + j * 16 + g * 4) = o[rt][j] * f;
    __syncthreads();
    for (int e = tid * 4; e < min(16, rows - rt * 16) * DP; e += kThreads * 4) {
      const int rr = e / DP, d = e % DP, r = rt * 16 + rr;
      f32x4 v = *(const f32x4*)(sums + e);
#pragma unroll
      for (int w = 1; w < 4; ++w) v += *(const f32x4*)(sums + w * 16 * DP + e);
      float top = kLow, total = 0.f;
      for (int w = 0; w < 4; ++w) top = fmaxf(top, mls[(w * RT * 16 + r) * 2]);
      for (int w = 0; w < 4; ++w)
        total += mls[(w * RT * 16 + r) * 2 + 1] * exp2_(mls[(w * RT * 16 + r) * 2] - top);
      if (!direct) {
        *(f32x4*)(a.part + ((int64_t)item * RT * 16 + r) * DP + d) = v;
        if (d == 0) {
          a.ml[((int64_t)item * RT * 16 + r) * 2] = top;
          a.ml[((int64_t)item * RT * 16 + r) * 2 + 1] = total;
        }
      } else {
        const int i = r / a.G, head = h * a.G + (r - i * a.G);
        const float inv = total == 0.f ? 0.f : 1.f / total;
        if (d < q.D)
          *(u32x2*)((uint16_t*)a.out + (int64_t)(seq.tok + i) * a.o_token +
                    (int64_t)head * a.o_head + d) =
              u32x2{T::pack(v[0] * inv, v[1] * inv), T::pack(v[2] * inv, v[3] * inv)};
        if (a.lse && d == 0)
          a.lse[(int64_t)(a.row0 + seq.tok + i) * a.q_heads + head] =
              total == 0.f ? -INFINITY : lse2_of(top, total, B::kLift) * kLn2;
      }
    }
  }
  nan_from = min(min(nans[0], nans[2]), min(nans[4], nans[6]));
  nan_to = max(max(nans[1], nans[3]), max(nans[5], nans[7]));
  if (direct && a.weigh) {  // the workgroup's own scores are all there are
    float* lse2s = sums;
    wait_loads<0>();
    __syncthreads();
    if (tid < rows) {
      float top = kLow, total = 0.f;
      for (int w = 0; w < 4; ++w) top = fmaxf(top, mls[(w * RT * 16 + tid) * 2]);
      for (int w = 0; w < 4; ++w)
        total += mls[(w * RT * 16 + tid) * 2 + 1] * exp2_(mls[(w * RT * 16 + tid) * 2] - top);
      lse2s[tid] = total == 0.f ? INFINITY : lse2_of(top, total, B::kLift);
    }
    __syncthreads();
    add_weights(a, seq, sb, h, rows, c0, cn, lse2s, (f32x4*)(sums + 64));
  }
  if (nan_from < nan_to) {
    wait_loads<0>();
    __syncthreads();
    spread_nan(a, sb, h, len, nq, seq.tok, nan_from, min(nan_to, c0 + cn), 0, rows,
               direct ? nullptr : a.part + (int64_t)item * RT * 16 * DP, DP);
  }
}

// ---------------------------------------------------------------------------
// Many rows (prompt chunks): a workgroup takes 128 rows (queries and heads of a
// group together, so that all share the head's tokens), 32 to a wave, and 32
// tokens at a time (a tile); 32x32x16 products.
// Codes come to LDS four tiles ahead, as they are.  The lanes that asked for them
// turn them into 16-bit rows, scale and all, for the four waves: keys two tiles
// ahead, values one, read transposed (ds_read_tr).  A step holds its tile's
// scores already: it turns them into probabilities while the matrix unit makes
// the next tile's scores and the products with its values.
// Places and scales of 256 tokens (a segment) stand in LDS; the next segment's are
// brought in between: table entries, then scales, by the same kind of copy.
// Probabilities are rounded to the queries' type for the second product: in bf16, 4
// sequences of 1500 to 4000 tokens, the last 700 to 1024 queries of 8 heads of 8
// each, are 2.3e-3 from 64 bits (rounding the result alone, 1.7e-3) in 382 us a
// call; with each as the sum of two numbers it took 472.
// Bound by the matrix units, vector instructions and LDS, which are busy 27, 36 and
// 38 % of that time and take turns within a wave more than they overlap: 265 GFLOP
// 0.385 ms, 0.69 PFLOP/s, 57 % of what a large matrix product reaches.  (When this
// took 0.51 ms, 64 rows a wave instead of 32 took 0.69, results moved between
// register files, and 64 tokens a tile 0.54, spilled.)
// ---------------------------------------------------------------------------
constexpr int kTile = 32, kSegment = 256, kPerSegment = kSegment / kTile, kAhead = 4;

// As copy_to_lds, 4 bytes a lane: to lds + 4 * lane.
__device__ __forceinline__ void copy_word_to_lds(const void* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off"
               ::"v"(from), "s"(lds)
               : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)p;
}

__device__ __forceinline__ u32x2 read_tr(const uint8_t* p) {
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
}

// LDS: two tiles of keys and of values as 16-bit rows, the copied codes, two
// segments' tables (place, key scale, value scale, position, table entry).
template <int DP>
struct TileLds {
  static constexpr int kPitch = DP * 2 + 16, vPitch = DP * 2 + 32;  // bytes of a token's row
  static constexpr int kBuf = kTile * kPitch, vBuf = kTile * vPitch, kRaw = 2 * kTile * DP;
  static constexpr int kKeys = 0, kValues = 2 * kBuf, kCodes = kValues + 2 * vBuf;
  static constexpr int kTables = kCodes + kAhead * kRaw, kTable = 5 * kSegment * 4;
  static constexpr int kFlags = kTables + 2 * kTable;  // holes [2][4], NaN [4][2]
  static constexpr int kBytes = kFlags + 16 * 4;
};

template <bool BF16, int DP>
__global__ void __launch_bounds__(kThreads, tile_waves(DP))
    attend_tile_kernel(AttendArgs a, int direct) {
  using T = Ty<BF16>;
  using L = TileLds<DP>;
  constexpr int KS = DP / 16, DB = DP / 32, CH = DP / 16;
  constexpr int kPitch = L::kPitch, vPitch = L::vPitch;
  constexpr int kUnits = kTile * CH;            // of 16 codes, of keys
  constexpr int UT = 2 * kUnits / kThreads;     // units a thread brings, keys' first
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  int* const holes_of = (int*)(lds + L::kFlags);
  int* const nans_of = holes_of + 8;
  const QLayout& q = a.q;
  const int tid = threadIdx.x, l = tid & 63, c = l & 31, hf = l >> 5;
  const int wave = scalar(tid >> 6);

  const int item = blockIdx.x;
  const Seq seq = seq_of(a, item);
  const int b = seq.b, sb = a.b0 + b, len = seq.len, nq = seq.nq, rows = nq * a.G;
  const int nsplit = max(1, scalar((len + a.chunk - 1) / a.chunk));
  const int tiles = (rows + kTileRows - 1) / kTileRows;
  const int h = scalar(seq.k / (tiles * nsplit)), kk = seq.k - h * tiles * nsplit;
  // the last rows see the most tokens: they go first
  const int tile = tiles - 1 - scalar(kk / nsplit), split = kk - (tiles - 1 - tile) * nsplit;
  const int r0 = tile * kTileRows, r = r0 + wave * 32 + c;
  const bool on = r < rows;
  const int i0 = r / a.G, head = h * a.G + (r - i0 * a.G);
  const int limit = on ? len - nq + i0 : -1;
  const int all_see = len - nq + scalar(r0 / a.G);
  const int last = len - nq + scalar((min(rows, r0 + kTileRows) - 1) / a.G);  // last slot seen
  const int begin = split * a.chunk, end = min(min(begin + a.chunk, len), last + 1);
  const int N = end > begin ? (end - begin + kTile - 1) / kTile : 0;

  const int64_t slab = 2 * (int64_t)a.layer;
  const uint8_t* kb = q.codes + slab * q.s_slab + sb * q.s_b + h * q.s_h;
  const float* sk = q.scale + slab * q.c_slab + sb * q.c_b + h * q.c_h;
  const int32_t* bt = q.bt ? q.bt + (int64_t)sb * q.max_blocks : nullptr;
  const int64_t slots = (((int64_t)a.layer * q.batch + sb) * q.heads + h) * (int64_t)q.cap;

  u32x4 qr[KS];
  {
    const uint16_t* src = (const uint16_t*)a.query +
                          (int64_t)(on ? seq.tok + i0 : 0) * a.q_token + (int64_t)head * a.q_head;
    // The scores' factor counts as positive below: its sign goes to the queries.
    const uint32_t flip = a.scale2 < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int d = s * 16 + hf * 8;
      qr[s] = on && d < q.D ? *(const u32x4*)(src + d) : u32x4{0, 0, 0, 0};
      qr[s] ^= flip;
    }
  }
  // (A factor of 0 makes equal scores; as a tiny one it leaves hidden ones at -infinity.)
  const float factor = fmaxf(fabsf(a.scale2), 0x1p-126f);
  float slope = 0.f, here = 0.f;
  const int last_at = last_position(q, a.slopes, slots, len);
  if (a.slopes && limit >= 0) {
    slope = a.slopes[head] * kLog2e;
    here = q.position ? from_last(q.position[slots + limit], last_at) : (float)limit;
  }

  // ---- segments: thread tid stands for token begin + 256 g + tid ----
  auto table = [&](int g, int which) {
    return (float*)(lds + L::kTables + (g & 1) * L::kTable) + which * kSegment;
  };
  enum { kPlace, kKeyScale, kValueScale, kPosition, kEntry };
  auto slot_of = [&](int g) { return min(begin + g * kSegment + tid, len - 1); };
  // The table entry known: the place, and whether there is one.  Returns the block.
  auto place = [&](int g, int entry) {
    const int slot = slot_of(g), j = q.d_bs.div(slot);
    int blk = bt ? entry : j;
    const bool hole = bt && (uint32_t)blk >= (uint32_t)q.num_blocks;
    blk = hole ? 0 : blk;
    ((uint32_t*)table(g, kPlace))[tid] =
        (uint32_t)(((int64_t)blk * q.s_blk + (int64_t)(slot - j * q.bs) * q.D) >> 4);
    ((int*)table(g, kEntry))[tid] = hole ? -1 : 0;
    const bool any = __any(hole);
    if (l == 0) holes_of[(g & 1) * 4 + wave] = any;
    if (a.slopes && !q.position) table(g, kPosition)[tid] = (float)slot;
    return blk;
  };

  // ---- codes: unit u = tid + 256 i, the keys' kUnits first ----
  const uint32_t raw = scalar(lds_address(lds + L::kCodes));
  // 0: keys, 1: values
  auto half_of = [&](int i) {
    if constexpr (kUnits >= kThreads)
      return i / (kUnits / kThreads);
    else
      return wave * 64 / kUnits;
  };
  const uint8_t* const vb = kb + q.s_slab;
  auto fetch = [&](int n, int last) {  // past the last tile: that one again
    const int from = min(n, last);
    const uint32_t* row =
        (const uint32_t*)table(from / kPerSegment, kPlace) + from % kPerSegment * kTile;
    uint32_t at[UT];
#pragma unroll
    for (int i = 0; i < UT; ++i) {
      const int u = (tid + kThreads * i) % kUnits, p = u % CH;
      at[i] = row[u / CH] + (p * 16 < q.D ? p : 0);
    }
    wait_lds();
#pragma unroll
    for (int i = 0; i < UT; ++i)
      copy_to_lds<false>((half_of(i) ? vb : kb) + (uint64_t)at[i] * 16,
                         raw + (n & (kAhead - 1)) * L::kRaw + (wave * 64 + kThreads * i) * 16);
  };
  auto any_hole = [&](int g) {
    const int* f = holes_of + (g & 1) * 4;
    return bt && scalar(f[0] | f[1] | f[2] | f[3]);
  };
  int nan_from = INT32_MAX, nan_to = 0;  // tiles
  // Whether this segment, and the next, have unmapped slots.
  bool holes = false, next_holes = false;
  auto holes_at = [&](int n, int now) { return n / kPerSegment == now / kPerSegment ? holes : next_holes; };
  // From codes to rows, unit i: of the keys of tile n + 2 or the values of tile n + 1.
  struct Raw {
    u32x4 x;
    float scale;
    int entry;
  };
  auto tile_of = [&](int i, int n) { return half_of(i) ? n + 1 : n + 2; };
  auto take = [&](int i, int n, bool holes) {
    Raw y;
    const int tok = n % kPerSegment * kTile + (tid + kThreads * i) % kUnits / CH;
    y.x = *(const u32x4*)(lds + L::kCodes + (n & (kAhead - 1)) * L::kRaw +
                          (tid + kThreads * i) * 16);
    y.scale = table(n / kPerSegment, kKeyScale + half_of(i))[tok];
    y.entry = holes ? ((const int*)table(n / kPerSegment, kEntry))[tok] : 0;
    return y;
  };
  auto put = [&](Raw y, int i, int n, bool holes) {
    const int half = half_of(i), u = (tid + kThreads * i) % kUnits, tok = u / CH, p = u % CH;
    uint8_t* to = lds + (half ? L::kValues + (n & 1) * L::vBuf : L::kKeys + (n & 1) * L::kBuf) +
                  tok * (half ? vPitch : kPitch) + p * 32;
    if (y.entry < 0 || p * 16 >= q.D) y.x = u32x4{0, 0, 0, 0};  // not there
    if (y.entry < 0) y.scale = 1.f;  // (0 times a scale that nothing wrote may be NaN)
    // Values that some row does not see: NaN becomes 0 (spread_nan).
    if (half && (begin + (n + 1) * kTile - 1 > all_see || holes)) {
      uint32_t nan = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t z = nan_bytes(y.x[w]);
        nan |= z;
        y.x[w] &= ~((z >> 7) * 0xffu);
      }
      if (__any(nan != 0)) {
        nan_from = min(nan_from, n);
        nan_to = n + 1;
      }
    }
    u32x4 x[2];
#pragma unroll
    for (int e = 0; e < 2; ++e)
      x[e] = u32x4{
          T::template cvt<false>(y.x[2 * e], y.scale), T::template cvt<true>(y.x[2 * e], y.scale),
          T::template cvt<false>(y.x[2 * e + 1], y.scale),
          T::template cvt<true>(y.x[2 * e + 1], y.scale)};
    if (__any(y.scale > T::kHeld)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i / 4][i % 4] = T::finite(x[i / 4][i % 4]);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) *(u32x4*)(to + e * 16) = x[e];
  };

  f32x16 o[DB], s;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  float m = kLow, sum = 0.f;
  bool scaled = a.slopes != nullptr;  // whether scores get their factor by themselves
  auto key = [&](int n, int e) {
    return *(const u32x4*)(lds + L::kKeys + (n & 1) * L::kBuf + c * kPitch + e * 32 + hf * 16);
  };

  if (N > 0) {
    const int slot = slot_of(0), blk = place(0, bt ? bt[q.d_bs.div(slot)] : 0);
    table(0, kKeyScale)[tid] = sk[blk * q.c_blk];
    table(0, kValueScale)[tid] = sk[blk * q.c_blk + q.c_slab];
    if (a.slopes && q.position)
      table(0, kPosition)[tid] = from_last(q.position[slots + slot], last_at);
    __syncthreads();
    holes = any_hole(0);
    for (int n = 0; n < kAhead; ++n) fetch(n, N - 1);
    wait_loads<0>();
#pragma unroll
    for (int i = 0; i < UT; ++i) {
      put(take(i, 0, holes), i, 0, holes);
      if (!half_of(i) && N > 1) put(take(i, 1, holes), i, 1, holes);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
  for (int e = 0; e < KS; ++e) s = T::mma32(key(0, e), qr[e], s);
  settle(s);

  for (int n = 0; n < N; ++n) {
    const int t = begin + n * kTile, g = n / kPerSegment;
    // The next segment's tables, before this tile's codes: each is there when the
    // waits below have let what was asked for two steps ago arrive.
    if (n % kPerSegment == 0 && n > 0) holes = next_holes;
    if ((g + 1) * kPerSegment < N) {
      if (n % kPerSegment == 4) {
        next_holes = any_hole(g + 1);
        if (a.slopes && q.position) {  // what this lane asked for
          float* x = table(g + 1, kPosition) + tid;
          *x = from_last(*(const int*)x, last_at);
        }
      }
      if (n % kPerSegment == 0 && bt)
        copy_word_to_lds(bt + q.d_bs.div(slot_of(g + 1)),
                         scalar(lds_address(table(g + 1, kEntry) + wave * 64)));
      if (n % kPerSegment == 2) {
        const int blk = place(g + 1, bt ? ((const int*)table(g + 1, kEntry))[tid] : 0);
        const float* from = sk + blk * q.c_blk;
        copy_word_to_lds(from, scalar(lds_address(table(g + 1, kKeyScale) + wave * 64)));
        copy_word_to_lds(from + q.c_slab,
                         scalar(lds_address(table(g + 1, kValueScale) + wave * 64)));
        if (a.slopes && q.position)
          copy_word_to_lds(q.position + slots + slot_of(g + 1),
                           scalar(lds_address(table(g + 1, kPosition) + wave * 64)));
      }
    }
    fetch(n + kAhead, N - 1);
    u32x4 y[KS];
#pragma unroll
    for (int e = 0; e < KS; ++e) y[e] = key(n + 1, e);

    // This tile's scores: bias, what is hidden, the reference.
    float mul = factor;
    if (scaled) {
      mul = 1.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] *= factor;
      if (a.slopes) {
        const float* at = table(g, kPosition) + n % kPerSegment * kTile + hf * 4;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] += slope * (at[(i / 4) * 8 + i % 4] - here);
      }
    }
    const bool mask = holes || t + kTile - 1 > all_see;
    if (mask) {
      const int* entry = (const int*)table(g, kEntry) + n % kPerSegment * kTile + hf * 4;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int at = (i / 4) * 8 + i % 4;
        const bool sees = t + at + hf * 4 <= limit && !(holes && entry[at] < 0);
        s[i] = sees ? s[i] : -INFINITY;
      }
    }
    float most = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) most = fmaxf(most, s[i]);
    most *= mul;
    if (__any(most > m + (kSlack + T::kLift))) {
      float up = fmaxf(most - T::kLift, m);
      up = fmaxf(up, __shfl_xor(up, 32));
      const float f = exp2_(m - up);
      m = up;
      sum *= f;
#pragma unroll
      for (int d = 0; d < DB; ++d) o[d] = o[d] * f;
      // The reference is a rounded score; scores this large pass it by powers of two
      // that the types do not hold unless they are rounded first too.
      if (!scaled && __any(fabsf(m) > 0x1p22f && m > kLow)) {
        scaled = true;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] *= mul;
        mul = 1.f;
      }
    }
    const uint8_t* vt = lds + L::kValues + (n & 1) * L::vBuf + (hf * 4 + ((l & 15) >> 2)) * vPitch + ((l >> 4) & 1) * 32 +
                        (l & 3) * 8;
    // Products with exponentials in between (the barriers keep them so): the next
    // tile's scores, of which the last is out of range and used by nothing, ...
    auto value = [&](int e, int d) {
      const u32x2 v0 = read_tr(vt + e * 16 * vPitch + d * 64);
      const u32x2 v1 = read_tr(vt + (e * 16 + 8) * vPitch + d * 64);
      return u32x4{v0[0], v0[1], v1[0], v1[1]};
    };
    f32x16 z;
    u32x4 p[2], v[DB];  // p: 16 tokens each, slots hf * 8 + 0..7 of the inner axis
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
#pragma unroll
    for (int e = 0; e < KS; ++e) {
      z = T::mma32(y[e], qr[e], z);
#pragma unroll
      for (int i = e * 8 / KS; i < (e + 1) * 8 / KS; ++i) {
        const float p0 = exp2_(s[2 * i] * mul - m), p1 = exp2_(s[2 * i + 1] * mul - m);
        sum += p0 + p1;
        p[i / 4][i % 4] = T::pack(p0, p1);
        asm volatile("" : "+v"(p[i / 4][i % 4]));  // here, not where it is first used
      }
      if (e >= DB) v[e - DB] = value(0, e - DB);
      __builtin_amdgcn_sched_barrier(0);
    }
    // ... and the products with the values, the codes' conversion in between.  What
    // was asked for up to two steps ago is there: the keys of tile n + 2.
    // (Past the last tile too, where nothing reads what comes of it: no branch keeps
    // products and exponentials apart.)
    wait_loads<2 * UT>();
    Raw raws[UT];
#pragma unroll
    for (int i = 0; i < UT; ++i)
      raws[i] = take(i, tile_of(i, n), holes_at(tile_of(i, n), n));
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      o[d] = T::mma32(v[d], p[0], o[d]);
      v[d] = value(1, d);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < UT; ++i)
      put(raws[i], i, tile_of(i, n), holes_at(tile_of(i, n), n));
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = T::mma32(v[d], p[1], o[d]);
    settle(z);
    s = z;
    lds_barrier();
  }

  sum += __shfl_xor(sum, 32);
  if (l == 0) {
    nans_of[wave * 2] = nan_from;
    nans_of[wave * 2 + 1] = nan_to;
  }
  const int64_t at = (int64_t)item * kTileRows + wave * 32 + c;
  if (on && !direct) {
    if (hf == 0) {
      a.ml[at * 2] = m;
      a.ml[at * 2 + 1] = sum;
    }
    if (N > 0) {
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *(f32x4*)(a.part + at * DP + d * 32 + (i / 4) * 8 + hf * 4) =
              f32x4{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
    }
  }
  if (on && direct) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    uint16_t* out = (uint16_t*)a.out + (int64_t)(seq.tok + i0) * a.o_token +
                    (int64_t)head * a.o_head;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int x = d * 32 + (i / 4) * 8 + hf * 4;
        if (x < q.D)
          *(u32x2*)(out + x) = u32x2{T::pack(o[d][i] * inv, o[d][i + 1] * inv),
                                     T::pack(o[d][i + 2] * inv, o[d][i + 3] * inv)};
      }
    if (hf == 0) {
      const float lse2 = lse2_of(m, sum, T::kLift);
      const int64_t row = (int64_t)(seq.tok + i0) * a.q_heads + head;
      if (a.lse) a.lse[(int64_t)a.row0 * a.q_heads + row] = sum == 0.f ? -INFINITY : lse2 * kLn2;
      if (a.weigh) a.row_lse[row] = sum == 0.f ? INFINITY : lse2;
    }
  }
  wait_loads<0>();
  __syncthreads();
  nan_from = min(min(nans_of[0], nans_of[2]), min(nans_of[4], nans_of[6]));
  nan_to = max(max(nans_of[1], nans_of[3]), max(nans_of[5], nans_of[7]));
  if (nan_from < nan_to)
    spread_nan(a, sb, h, len, nq, seq.tok, begin + nan_from * kTile,
               min(end, begin + nan_to * kTile), r0, min(kTileRows, rows - r0),
               direct ? nullptr : a.part + (int64_t)item * kTileRows * DP, DP);
}

// ---------------------------------------------------------------------------
// Joins the splits of the kernels above: R rows a work item, a workgroup for each
// split of a head and 32 of its rows (64 rows: 45.0 us with the split kernel, with
// one workgroup 46.9; 128: 104 and 106).  They add up the results: four dims to a
// lane, a group of lanes to a row.  Up to 16 splits are one group's where there
// are more rows than splits; more, or of few rows, are dealt to all of a
// workgroup's groups (8 rows of 14 splits: 14.9 us instead of 16.3 with the split
// kernel; 16 rows of 4: 38.5 instead of 24.5).  The last row of the grid,
// where the scores were kept, adds up the weights of the split's own tokens, four to a lane, for which
// it needs every row's sum.
// Bound by latency: two rounds through memory.  4 to 5 us a decode step, of which
// 2 are the launch; 15 us where it reads 34 MB of scores (131071 tokens, 8 heads
// of 8 queries).
// ---------------------------------------------------------------------------
template <bool BF16, int DP>
__global__ void __launch_bounds__(kThreads) attend_join_kernel(AttendArgs a, int R) {
  using T = Ty<BF16>;
  constexpr int DL = DP / 4, P = kThreads / DL;  // lanes to a row; groups
  constexpr int kAlone = 16;
  __shared__ float lse2s[kTileRows], tops[P], totals[P];
  __shared__ __attribute__((aligned(16))) float acc[kThreads * 4];
  const QLayout& q = a.q;
  const int tid = threadIdx.x;
  const int item = blockIdx.x;
  const Seq seq = seq_of(a, item);
  const int b = seq.b, sb = a.b0 + b, len = seq.len, nq = seq.nq, rows = nq * a.G;
  const int nsplit = max(1, scalar((len + a.chunk - 1) / a.chunk));
  const int tiles = scalar((rows + R - 1) / R);
  const int h = scalar(seq.k / (tiles * nsplit)), kk = seq.k - h * tiles * nsplit;
  const int tile = tiles - 1 - scalar(kk / nsplit), split = kk - (tiles - 1 - tile) * nsplit;
  const int r0 = tile * R, nr = min(R, rows - r0);
  const float2* ml = (const float2*)a.ml + ((int64_t)item - split) * R;
  const float lift = R == kTileRows ? T::kLift : Ty<true>::kLift;  // of the kernel before

  const int shares = gridDim.y - (a.scores ? 1 : 0), share = blockIdx.y;
  if (share < shares) {
    const bool alone = nsplit <= 2 || (nsplit <= kAlone && nr > nsplit);
    const int group = tid / DL, d = tid % DL * 4, per = alone ? P : 1;
    for (int rb = (share * nsplit + split) * per; rb < nr; rb += shares * nsplit * per) {
      const int r = min(alone ? rb + group : rb, nr - 1);
      const float* part = a.part + (((int64_t)item - split) * R + r) * DP + d;
      f32x4 v = {0, 0, 0, 0};
      float top = kLow, total = 0.f;
#pragma unroll 4
      for (int s = alone ? 0 : group; s < nsplit; s += alone ? 1 : P) {
        const float2 x = ml[(int64_t)s * R + r];
        const f32x4 y = *(const f32x4*)(part + (int64_t)s * R * DP);
        const float up = fmaxf(top, x.x), f0 = exp2_(top - up), f1 = exp2_(x.x - up);
        total = total * f0 + x.y * f1;
#pragma unroll
        for (int i = 0; i < 4; ++i)  // a split that saw nothing wrote no results
          v[i] = v[i] * f0 + (x.y != 0.f ? y[i] * f1 : 0.f);
        top = up;
      }
      if (!alone) {
        __syncthreads();
        *(f32x4*)(acc + tid * 4) = v;
        if (d == 0) {
          tops[group] = top;
          totals[group] = total;
        }
        __syncthreads();
        if (tid < DL) {
          for (int p = 1; p < P; ++p) {
            const float up = fmaxf(top, tops[p]), f0 = exp2_(top - up), f1 = exp2_(tops[p] - up);
            total = total * f0 + totals[p] * f1;
            const f32x4 y = *(const f32x4*)(acc + (p * DL + tid) * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = v[i] * f0 + y[i] * f1;
            top = up;
          }
        }
      }
      if (alone ? rb + group >= nr : tid >= DL) continue;
      const int i = (r0 + r) / a.G, head = h * a.G + (r0 + r - i * a.G);
      const float inv = total == 0.f ? 0.f : 1.f / total;
      if (d < q.D)
        *(u32x2*)((uint16_t*)a.out + (int64_t)(seq.tok + i) * a.o_token +
                  (int64_t)head * a.o_head + d) =
            u32x2{T::pack(v[0] * inv, v[1] * inv), T::pack(v[2] * inv, v[3] * inv)};
      if (d == 0) {
        const float lse2 = lse2_of(top, total, lift);
        const int64_t row = (int64_t)(seq.tok + i) * a.q_heads + head;
        if (a.lse)
          a.lse[(int64_t)a.row0 * a.q_heads + row] = total == 0.f ? -INFINITY : lse2 * kLn2;
        if (a.row_lse) a.row_lse[row] = total == 0.f ? INFINITY : lse2;
      }
    }
    return;
  }

  for (int r = tid / 32; r < nr; r += kThreads / 32) {
    float m = kLow, sum = 0.f;
    for (int s = tid % 32; s < nsplit; s += 32) {
      const float2 x = ml[(int64_t)s * R + r];
      const float up = fmaxf(m, x.x);
      sum = sum * exp2_(m - up) + x.y * exp2_(x.x - up);
      m = up;
    }
    float up = m;
#pragma unroll
    for (int x = 16; x; x >>= 1) up = fmaxf(up, __shfl_xor(up, x));
    sum *= exp2_(m - up);
#pragma unroll
    for (int x = 16; x; x >>= 1) sum += __shfl_xor(sum, x);
    if (tid % 32 == 0) lse2s[r] = sum == 0.f ? INFINITY : lse2_of(up, sum, lift);
  }
  __syncthreads();
  add_weights(a, seq, sb, h, nr, split * a.chunk, min(a.chunk, len - split * a.chunk), lse2s,
              (f32x4*)acc);
}

// ---------------------------------------------------------------------------
// Weights from many rows: a workgroup takes 128 tokens of a head and the rows that
// may see them, or where that leaves the card empty one of several shares of
// those; p = exp2(s2 - lse2).  A wave holds 64 tokens' keys and takes
// every other 32 rows, which the workgroup copies to LDS two steps ahead (16-byte
// pieces stored at piece ^ key(row), as above).  Each sum is one lane's; the
// lanes', then the two waves', are added in a fixed order.
// Bound by the exponentials and the product: 132 GFLOP (the case of the tile kernel)
// 0.22 ms, 0.60 PFLOP/s, the matrix units busy 24 % of the time and vector
// instructions 48 %.  Three heads, 1647 tokens, up to 413 queries
// of 16: 52 us in shares of the rows and 5 to add them, 216 without shares.
// ---------------------------------------------------------------------------
template <bool BF16, int DP>
__global__ void __launch_bounds__(kThreads, weigh_waves(DP)) attend_weigh_kernel(AttendArgs a) {
  using T = Ty<BF16>;
  constexpr int KS = DP / 16, CH = DP / 8;       // products; 16-byte pieces of a row
  constexpr int kStep = 64, kBytes = kStep * DP * 2, kRing = 3;
  constexpr int kLoads = kBytes / 1024 / 4;      // copies of a wave
  __shared__ __attribute__((aligned(1024))) uint8_t rows_of[kRing * kBytes];
  __shared__ __attribute__((aligned(16))) float words[kRing][2][128];  // rows' lse, slope, position
  __shared__ __attribute__((aligned(16))) float token_at[kWeighTokens];  // positions
  __shared__ float part[2][64];
  const QLayout& q = a.q;
  const int tid = threadIdx.x, l = tid & 63, c = l & 31, hf = l >> 5;
  const int wave = scalar(tid >> 6), odd = wave >> 1;
  const int item = blockIdx.x;
  const Seq seq = seq_of(a, item);
  const int b = seq.b, sb = a.b0 + b, len = seq.len, nq = seq.nq, rows = nq * a.G;
  const int tiles = (len + kWeighTokens - 1) / kWeighTokens;
  const int h = scalar(seq.k / tiles), t0 = (seq.k - h * tiles) * kWeighTokens;
  const int tw = t0 + (wave & 1) * 64;  // this wave's tokens

  const int64_t slab = 2 * (int64_t)a.layer;
  const int64_t slots = (((int64_t)a.layer * q.batch + sb) * q.heads + h) * (int64_t)q.cap;
  u32x4 kr[2][KS];
  uint32_t mapped[2];  // bit i: token tw + 32 u + i
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int tok = min(tw + u * 32 + c, len - 1), j = q.d_bs.div(tok);
    int64_t blk = q.bt ? q.bt[(int64_t)sb * q.max_blocks + j] : j;
    const bool hole = q.bt && (uint64_t)blk >= (uint64_t)q.num_blocks;
    blk = hole ? 0 : blk;
    mapped[u] = (uint32_t)__ballot(!hole);
    const uint8_t* p = q.codes + slab * q.s_slab + sb * q.s_b + h * q.s_h + blk * q.s_blk +
                       (int64_t)(tok - j * q.bs) * q.D;
    const float scale = q.scale[slab * q.c_slab + sb * q.c_b + h * q.c_h + blk * q.c_blk];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int d = s * 16 + hf * 8;
      u32x2 w = {0, 0};
      if (d < q.D) w = *(const u32x2*)(p + d);
      kr[u][s] = u32x4{T::template cvt<false>(w[0], scale), T::template cvt<true>(w[0], scale),
                       T::template cvt<false>(w[1], scale), T::template cvt<true>(w[1], scale)};
#pragma unroll
      for (int i = 0; i < 4; ++i) kr[u][s][i] = T::finite(kr[u][s][i]);
    }
  }
  const int last_at = last_position(q, a.slopes, slots, len);
  if (a.slopes && tid < kWeighTokens) {
    const int x = min(t0 + tid, len - 1);
    token_at[tid] = q.position ? from_last(q.position[slots + x], last_at) : (float)x;
  }

  const int before = len - nq;  // query i sees slots up to before + i
  // the first row that sees the workgroup's first token
  const int from = max(0, t0 - before) * a.G & -kStep;
  const int all = rows > from ? (rows - from + kStep - 1) / kStep : 0;
  const int shares = gridDim.y, per = scalar((all + shares - 1) / shares);
  const int k0 = blockIdx.y * per, first = from + k0 * kStep, steps = max(0, min(per, all - k0));
  auto key_of = [](int row) { return CH == 8 ? (row >> 1) & 7 : row & 15; };
  const uint32_t rows_at = scalar(lds_address(rows_of)), words_at = scalar(lds_address(words));
  // (Rows past the last are the last again, and so are steps; both are hidden.)
  auto fetch = [&](int k) {
    const int r0 = first + min(k, steps - 1) * kStep, slot = k % kRing;
    wait_lds();
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int u = tid + kThreads * i, row = u / CH, r = min(r0 + row, rows - 1);
      const int qi = a.d_G.div(r), head = h * a.G + (r - qi * a.G);
      const int d = (u % CH ^ key_of(row)) * 8;
      copy_to_lds<false>((const uint8_t*)((const uint16_t*)a.query +
                                          (uint64_t)(uint32_t)(seq.tok + qi) * (uint32_t)a.q_token +
                                          (uint64_t)(uint32_t)head * (uint32_t)a.q_head +
                                          (d < q.D ? d : 0)),
                         rows_at + slot * kBytes + (wave * 64 + kThreads * i) * 16);
    }
    const int r = min(r0 + odd * 32 + c, rows - 1), qi = a.d_G.div(r), head = h * a.G + r - qi * a.G;
    const float* word = a.row_lse + (int64_t)(seq.tok + qi) * a.q_heads + head;
    if (a.slopes) {  // the two waves of these rows bring half each
      if (hf) word = a.slopes + head;
      if ((wave & 1) && q.position) word = (const float*)(q.position + slots + max(0, before + qi));
    }
    copy_word_to_lds(word, words_at + (slot * 4 + wave) * 256);
  };

  float sum[2][16];
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[u][i] = 0.f;
  if (steps > 0) {
    fetch(0);
    fetch(1);
  }
  for (int k = 0; k < steps; ++k) {
    wait_loads<kLoads + 1>();  // all but the next step's
    lds_barrier();
    fetch(k + 2);
    const int slot = k % kRing, r0 = first + k * kStep + odd * 32;
    const uint8_t* ql = rows_of + slot * kBytes + (odd * 32 + c) * DP * 2;
    const int kk = key_of(c);  // (32 rows on the key is the same)
    f32x16 s[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) s[0][i] = s[1][i] = 0.f;
#pragma unroll
    for (int e = 0; e < KS; ++e) {
      // (pieces past head_dim repeat the row's first: they meet zeros of the keys)
      const u32x4 y = *(const u32x4*)(ql + (((2 * e + hf) ^ kk) << 4));
      s[0] = T::mma32(kr[0][e], y, s[0]);
      s[1] = T::mma32(kr[1][e], y, s[1]);
    }
    settle(s[0]);
    settle(s[1]);
    const float* w = words[slot][odd];
    const float lse2 = w[c];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[u][i] = s[u][i] * a.scale2 - lse2;
    const int limit = r0 + c < rows ? before + (int)a.d_G.div(r0 + c) : -1;
    if (a.slopes) {
      const float slope = w[32 + c] * kLog2e;
      const float here = q.position ? from_last(__float_as_int(w[64 + c]), last_at) : (float)limit;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[u][i] += slope * (token_at[tw - t0 + u * 32 + (i / 4) * 8 + hf * 4 + i % 4] - here);
    }
    // (lse is +infinity for a row that sees nothing: its p are 0, or NaN, and hidden)
    if (before + scalar(r0 / a.G) < tw + 63 || r0 + 32 > rows ||
        (mapped[0] & mapped[1]) != 0xffffffffu) {
      const int last = lse2 == INFINITY ? -1 : limit - tw - hf * 4;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint32_t there = mapped[u] >> (hf * 4);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int o = (i / 4) * 8 + i % 4;
          s[u][i] = u * 32 + o <= last && ((there >> o) & 1) ? s[u][i] : -INFINITY;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[u][i] += exp2_(s[u][i]);
  }
  wait_loads<0>();  // (nothing arrives after the workgroup's end)
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      sum[u][i] = sum_of_half(sum[u][i]);
      if (odd && c == i) part[wave & 1][u * 32 + (i / 4) * 8 + hf * 4 + i % 4] = sum[u][i];
    }
  __syncthreads();
  if (odd) return;
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int o = u * 32 + (i / 4) * 8 + hf * 4 + i % 4;
      if (c == i && tw + o < len) {
        float* to = q.weight + slots + tw + o;
        const float total = sum[u][i] + part[wave & 1][o];
        if (shares > 1)
          a.sums[((int64_t)blockIdx.y * a.items + item) * kWeighTokens + (tw - t0) + o] = total;
        else
          *to = a.decay == 0.f ? total : a.decay * *to + total;
      }
    }
}

// Adds the shares' sums, in order: a workgroup for the tokens of one above.
// 5 us, of which 2 are the launch.
__global__ void __launch_bounds__(kWeighTokens) attend_share_kernel(AttendArgs a, int shares) {
  const QLayout& q = a.q;
  const int item = blockIdx.x;
  const Seq seq = seq_of(a, item);
  const int tiles = (seq.len + kWeighTokens - 1) / kWeighTokens, h = seq.k / tiles;
  const int t = (seq.k - h * tiles) * kWeighTokens + threadIdx.x;
  if (t >= seq.len) return;
  const float* from = a.sums + (int64_t)item * kWeighTokens + threadIdx.x;
  float total = 0.f;
#pragma unroll 8
  for (int i = 0; i < shares; ++i) total += from[(int64_t)i * a.items * kWeighTokens];
  float* to = q.weight + (((int64_t)a.layer * q.batch + a.b0 + seq.b) * q.heads + h) * (int64_t)q.cap + t;
  *to = a.decay == 0.f ? total : a.decay * *to + total;
}

template <typename... More>
hipError_t launch(const void* fn, dim3 groups, size_t lds, hipStream_t s, const AttendArgs& a,
                  More... more) {
  void* args[] = {const_cast<AttendArgs*>(&a), &more...};
  return hipLaunchKernel(fn, groups, dim3(kThreads), args, lds, s);
}

template <bool BF16, int DP>
struct Kernels {
  static const void* split(int rt) {
    if (rt == 1) return (const void*)&attend_split_kernel<BF16, DP, 1>;
    if (rt == 2) return (const void*)&attend_split_kernel<BF16, DP, 2>;
    if constexpr (DP < 256) return (const void*)&attend_split_kernel<BF16, DP, 4>;
    return nullptr;
  }
  static const void* tile() { return (const void*)&attend_tile_kernel<BF16, DP>; }
  static const void* join() { return (const void*)&attend_join_kernel<BF16, DP>; }
  static const void* weigh() { return (const void*)&attend_weigh_kernel<BF16, DP>; }
};

// f(Kernels<type, padded head_dim>) for a launch's type and head_dim
template <typename F>
const void* pick(const AttendArgs& a, F f) {
  const int dp = padded(a.q.D);
  if (a.bf16)
    return dp == 64    ? f(Kernels<true, 64>())
           : dp == 128 ? f(Kernels<true, 128>())
                       : f(Kernels<true, 256>());
  return dp == 64    ? f(Kernels<false, 64>())
         : dp == 128 ? f(Kernels<false, 128>())
                     : f(Kernels<false, 256>());
}

}  // namespace

hipError_t launch_attend_split(const AttendArgs& a, int rt, bool direct, hipStream_t s) {
  const void* fn = pick(a, [&](auto k) { return decltype(k)::split(rt); });
  return launch(fn, dim3(a.items), split_lds(padded(a.q.D), rt, a.chunk, a.slopes != nullptr), s, a,
                (int)direct);
}

hipError_t launch_attend_tile(const AttendArgs& a, bool direct, hipStream_t s) {
  const void* fn = pick(a, [](auto k) { return decltype(k)::tile(); });
  const int dp = padded(a.q.D);
  const size_t lds = dp == 64    ? TileLds<64>::kBytes
                     : dp == 128 ? TileLds<128>::kBytes
                                 : TileLds<256>::kBytes;
  return launch(fn, dim3(a.items), lds, s, a, (int)direct);
}

hipError_t launch_attend_join(const AttendArgs& a, int rows, hipStream_t s) {
  return launch(pick(a, [](auto k) { return decltype(k)::join(); }),
                dim3(a.items, std::max(1, rows / 32) + (a.scores ? 1 : 0)), 0, s, a, rows);
}

hipError_t launch_attend_weigh(const AttendArgs& a, int shares, hipStream_t s) {
  const hipError_t e = launch(pick(a, [](auto k) { return decltype(k)::weigh(); }),
                              dim3(a.items, shares), 0, s, a);
  if (e != hipSuccess || shares == 1) return e;
  void* args[] = {const_cast<AttendArgs*>(&a), &shares};
  return hipLaunchKernel((const void*)&attend_share_kernel, dim3(a.items), dim3(kWeighTokens), args,
                         0, s);
}

}  // namespace dv
