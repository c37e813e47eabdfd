// Reading an 8-bit cache back into a 16-bit stream, and keeping the accepted ones of
// the drafted tokens in it.
#include "dv_draft_internal.h"
#include "dv_scale.h"

namespace dv {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------
// Back to 16 bits: a group of lanes takes a block of one head, 8 codes to a lane at
// a time, so that a wave reads 512 contiguous bytes and writes 1024.  Codes times
// powers of two are exact in both types but for f16's smallest; beyond the type's
// largest number is that.
// Bound by HBM: 1 byte read and 2 written per element.  378 MB (8 prompts of 512 to 1024
// tokens, 40 heads of 128, two layers) 63 us, 6.0 TB/s; a step's 1 to 6 tokens of 32
// sequences, 20 layers of 8 heads, 12 MB of rows of 128 bytes, 5.4 us, of which 2 are the
// launch.
// ---------------------------------------------------------------------------
template <bool BF16>
__device__ __forceinline__ uint32_t two(uint32_t w, bool high, float scale, bool large) {
  uint32_t y;
  if constexpr (BF16)
    y = high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true))
             : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
  else
    y = high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, true))
             : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, false));
  if (large) {  // infinities become the number below them
    constexpr uint32_t inf = BF16 ? 0x7f80u : 0x7c00u;
    y -= ((y & 0x7fffu) == inf) + ((uint32_t)((y >> 16 & 0x7fffu) == inf) << 16);
  }
  return y;
}

template <bool BF16>
__global__ void __launch_bounds__(kThreads) quant_out_kernel(QuantArgs a) {
  __shared__ int32_t first[kQSeqs];
  for (int i = threadIdx.x; i < a.nseq; i += kThreads) first[i] = a.item[i];
  __syncthreads();
  const int group = 1 << a.lanes_log2, lane = threadIdx.x & (group - 1);
  const uint32_t item = (blockIdx.x * (uint32_t)kThreads + threadIdx.x) >> a.lanes_log2;
  if (item >= (uint32_t)a.items) return;
  int b = 0;
  for (int step = 128; step; step >>= 1)
    if (b + step < a.nseq && first[b + step] <= (int)item) b += step;

  const QLayout& q = a.q;
  const int t0 = a.t0[b], n = a.tok[b + 1] - a.tok[b], t1 = t0 + n;
  const int j0 = q.d_bs.div(t0), nb = q.d_bs.div(t1 - 1) - j0 + 1;
  const int k = (int)item - first[b], h = (uint32_t)k / (uint32_t)nb, j = j0 + (k - h * nb);
  const int64_t slab = a.slab0 + (int64_t)blockIdx.y;
  const int sb = a.b0 + b;
  const int lo = max(t0, j * q.bs), hi = min(t1, (j + 1) * q.bs);
  const int64_t blk = q.bt ? q.bt[(int64_t)sb * q.max_blocks + j] : j;
  if (q.bt && (uint64_t)blk >= (uint64_t)q.num_blocks) return;
  const float scale = q.scale[slab * q.c_slab + sb * q.c_b + blk * q.c_blk + h * q.c_h];
  const u32x2* src = (const u32x2*)(q.codes + slab * q.s_slab + sb * q.s_b + blk * q.s_blk +
                                    h * q.s_h + (int64_t)(lo - j * q.bs) * q.D);
  u32x4* dst = (u32x4*)(const_cast<uint8_t*>(a.wire) + (int64_t)blockIdx.y * a.w_slab +
                        ((int64_t)a.tok[b] * q.heads + (int64_t)h * n + (lo - t0)) * q.D * 2);
  const int units = (hi - lo) * (q.D / 8);
  // the smallest scale whose product with the largest code the type does not hold
  const bool large = scale >= (BF16 ? 0x1p120f : 256.f);
  auto wide = [&](u32x2 w) {
    return u32x4{two<BF16>(w[0], false, scale, large), two<BF16>(w[0], true, scale, large),
                 two<BF16>(w[1], false, scale, large), two<BF16>(w[1], true, scale, large)};
  };
  constexpr int kHeld = 4;
  int u = lane;
  for (; u + (kHeld - 1) * group < units; u += kHeld * group) {
    u32x2 w[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) w[i] = __builtin_nontemporal_load(src + u + i * group);
#pragma unroll
    for (int i = 0; i < kHeld; ++i) __builtin_nontemporal_store(wide(w[i]), dst + u + i * group);
  }
  for (; u < units; u += group) __builtin_nontemporal_store(wide(src[u]), dst + u);
}

// ---------------------------------------------------------------------------
// The accepted drafts' tokens move to consecutive slots: a wave takes one head of a
// sequence in one layer, keys and values, and makes the blocks that they go to, in order.  Where each
// kept token lies and its scale are looked up first, all at once, before any scale
// is written; a lane holds those of two tokens.  A block's tokens come from its own
// slots or later ones, so that a wave which has read a block's (or, of larger blocks,
// 64 units of 16 codes of it, in order) may write over them.  Zeros under any scale stay
// zeros: the ratio of scales is kept finite.
// Bound by latency: four rounds through memory, of rows of 128 bytes that lie megabytes
// apart.  32 sequences, 8 heads, 20 layers, 1 to 8 tokens each, 11 MB: 12 us; a wave for
// each half took 13, and reading a block only once the last was written no less.
// ---------------------------------------------------------------------------
__device__ __forceinline__ float amax_of(const u32x4& c, float scale, float m) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // fmaxf drops NaN
    const f32x2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[i], scale, false);
    const f32x2 y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[i], scale, true);
    m = fmaxf(m, fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(y[0]), fabsf(y[1]))));
  }
  return m;
}
__device__ __forceinline__ u32x4 again(u32x4 c, float ratio) {
  ratio = fminf(fmaxf(ratio, 0x1p-126f), 0x1p126f);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[i], ratio, false);
    const f32x2 y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[i], ratio, true);
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    c[i] = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], w, true);
  }
  return c;
}

__global__ void __launch_bounds__(kThreads) keep_kernel(KeepArgs a) {
  const int l = threadIdx.x & 63;
  const QLayout& q = a.q;
  const int item = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)));
  const int b = a.d_heads.div(item), h = item - b * q.heads;
  if (b >= a.nseq) return;
  const int sb = a.b0 + b, base = a.base[b], tok = a.tok[b], nq = a.tok[b + 1] - tok;
  const int64_t layer = a.l0 + (int64_t)blockIdx.y;
  if (nq == 0) return;

  // Nothing below waits for what it does not need: the path, its count and the places of the
  // blocks that it goes to first; then where its tokens lie; then codes and scales.
  const int j0 = q.d_bs.div(base);
  const int32_t* path = a.path + tok;
  const int32_t* table = q.bt ? q.bt + (int64_t)sb * q.max_blocks : nullptr;
  const int left = a.count[b];
  int p0 = l < nq ? path[l] : INT32_MAX, p1 = l + 64 < nq ? path[l + 64] : INT32_MAX;
  auto place = [&](int j) { return table ? table[j] : j; };
  const int most_j = q.d_bs.div(base + nq - 1);  // the last block that may be needed
  const int to0 = place(min(j0 + l, most_j)), to1 = place(min(j0 + 64 + l, most_j));
  auto to_of = [&](int k) {  // the place of block j0 + k; -1: none
    const int x = __builtin_amdgcn_readlane(k < 64 ? to0 : to1, k & 63);
    return table && (uint32_t)x >= (uint32_t)q.num_blocks ? -1 : x;
  };

  // The path, entries l and l + 64, as far as it is one.
  const int most = min(left, nq);
  p0 = l < most ? p0 : INT32_MAX;
  p1 = l + 64 < most ? p1 : INT32_MAX;
  int before0 = __shfl_up(p0, 1), before1 = __shfl_up(p1, 1);
  const int end0 = __builtin_amdgcn_readlane(p0, 63);
  before0 = l == 0 ? -1 : before0;
  before1 = l == 0 ? end0 : before1;
  const uint64_t bad0 = ~__ballot(p0 > before0 && p0 < nq), bad1 = ~__ballot(p1 > before1 && p1 < nq);
  const int n = bad0 ? __builtin_ctzll(bad0) : 64 + (bad1 ? __builtin_ctzll(bad1) : 64);
  if (n == 0) return;

  uint8_t* const codes = q.codes + 2 * layer * q.s_slab + sb * q.s_b + h * q.s_h;
  float* const scales = q.scale + 2 * layer * q.c_slab + sb * q.c_b + h * q.c_h;
  // Tokens l and l + 64 of the path: their rows, in 16 bytes from the head's first, and scales.
  const int t0 = base + (l < n ? p0 : 0), t1 = base + (l + 64 < n ? p1 : 0);
  const int k0 = q.d_bs.div(t0), k1 = q.d_bs.div(t1);
  const int b0 = place(k0), b1 = place(k1);
  const bool in0 = !table || (uint32_t)b0 < (uint32_t)q.num_blocks;
  const bool in1 = !table || (uint32_t)b1 < (uint32_t)q.num_blocks;
  const uint32_t at0 =
      in0 ? (uint32_t)((b0 * q.s_blk + (int64_t)(t0 - k0 * q.bs) * q.D) >> 4) : ~0u;
  const uint32_t at1 =
      in1 ? (uint32_t)((b1 * q.s_blk + (int64_t)(t1 - k1 * q.bs) * q.D) >> 4) : ~0u;

  const int du = q.D / 16, last = base + n, blocks = q.d_bs.div(last - 1) - j0 + 1;
  // Where unit u of the tokens from k on lies (nowhere at `units` and beyond).
  auto where = [&](int k, int u, int units) {
    const int tk = a.d_du.div(min(u, units - 1)), part = u - tk * du;
    const uint32_t x0 = __shfl((int)at0, (k + tk) & 63), x1 = __shfl((int)at1, (k + tk) & 63);
    const uint32_t x = k + tk < 64 ? x0 : x1;
    return u < units && x != ~0u ? (int64_t)((uint64_t)x + part) * 16 : -1;
  };
  auto code = [&](int64_t at, int half) {
    return at < 0 ? u32x4{0, 0, 0, 0} : *(const u32x4*)(codes + half * q.s_slab + at);
  };
  constexpr int kHeld = 2;
  struct Block {
    int lo, units, to;
    u32x4 c[2][kHeld];  // keys, values
  };
  auto read = [&](int k, Block& x) {  // block j0 + k
    const int j = j0 + k;
    x.lo = max(base, j * q.bs);
    x.units = (min(last, (j + 1) * q.bs) - x.lo) * du;
    x.to = to_of(k);
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      x.c[0][i] = x.c[1][i] = u32x4{0, 0, 0, 0};
      if (i * 64 < x.units) {
        const int64_t at = where(x.lo - base, l + i * 64, x.units);
        x.c[0][i] = code(at, 0);
        x.c[1][i] = code(at, 1);
      }
    }
  };
  Block x;
  read(0, x);
  const bool begun = x.to >= 0 && base > j0 * q.bs;  // the first block holds tokens from before
  float first_scale[2], scale0[2], scale1[2];
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const float* from = scales + half * q.c_slab;
    first_scale[half] = begun ? from[x.to * q.c_blk] : 0.f;
    scale0[half] = in0 ? from[b0 * q.c_blk] : 1.f;
    scale1[half] = in1 ? from[b1 * q.c_blk] : 1.f;
  }
  float w0 = 0.f, w1 = 0.f;
  float* const weight =
      q.weight ? q.weight + ((layer * q.batch + sb) * q.heads + h) * (int64_t)q.cap + base : nullptr;
  if (weight) {
    w0 = weight[l < n ? p0 : 0];
    w1 = weight[l + 64 < n ? p1 : 0];
  }
  auto scale_of = [&](int k, int u, int units, int half) {
    const int tk = k + a.d_du.div(min(u, units - 1));
    const float x0 = __shfl(scale0[half], tk & 63), x1 = __shfl(scale1[half], tk & 63);
    return tk < 64 ? x0 : x1;
  };

  for (int k = 0; k < blocks; ++k) {
    // The next block's tokens come from its own slots or later ones, none of which this
    // block's writes touch.
    Block y = x;
    if (k + 1 < blocks) read(k + 1, y);
    if (x.to >= 0) {
      const int from = x.lo - base, held = x.lo - (j0 + k) * q.bs;  // (held: in the first block)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const float old = held ? first_scale[half] : 0.f;
        float s[kHeld], m = 0.f;
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
          if (i * 64 < x.units) {
            s[i] = scale_of(from, l + i * 64, x.units, half);
            m = amax_of(x.c[half][i], s[i], m);
          }
        for (int u = kHeld * 64; u < x.units; u += 64)
          m = amax_of(code(where(from, l + u, x.units), half),
                      scale_of(from, l + u, x.units, half), m);
#pragma unroll
        for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
        const float p = fmaxf(scale_for(m), old), inv = inverse(p);
        u32x4* const out = (u32x4*)(codes + half * q.s_slab + x.to * q.s_blk);
        u32x4* const to = out + held * du;
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
          if (l + i * 64 < x.units) to[l + i * 64] = again(x.c[half][i], s[i] * inv);
        for (int u = kHeld * 64; u < x.units; u += 64) {
          const u32x4 c = code(where(from, l + u, x.units), half);
          const float z = scale_of(from, l + u, x.units, half);
          if (l + u < x.units) to[l + u] = again(c, z * inv);
        }
        if (held && p > old)  // the codes from before, to the larger scale
          for (int u = l; u < held * du; u += 64) out[u] = again(out[u], old * inv);
        if (l == 0 && p != old) scales[half * q.c_slab + x.to * q.c_blk] = p;
      }
    }
    x = y;
  }
  if (weight) {
    if (l < n) weight[l] = w0;
    if (l + 64 < n) weight[l + 64] = w1;
  }
}

}  // namespace

hipError_t launch_quant_out(const QuantArgs& a, uint32_t nslabs, hipStream_t s) {
  const void* fn = a.bf16 ? (const void*)&quant_out_kernel<true> : (const void*)&quant_out_kernel<false>;
  const uint32_t per = kThreads >> a.lanes_log2;
  void* args[] = {const_cast<QuantArgs*>(&a)};
  return hipLaunchKernel(fn, dim3(((uint32_t)a.items + per - 1) / per, nslabs), dim3(kThreads),
                         args, 0, s);
}

hipError_t launch_keep(const KeepArgs& a, uint32_t layers, hipStream_t s) {
  const uint32_t waves = (uint32_t)a.nseq * a.q.heads, per = kThreads / 64;
  void* args[] = {const_cast<KeepArgs*>(&a)};
  return hipLaunchKernel((const void*)&keep_kernel, dim3((waves + per - 1) / per, layers),
                         dim3(kThreads), args, 0, s);
}

}  // namespace dv
