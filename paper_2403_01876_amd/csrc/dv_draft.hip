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
// sequence in one slab and makes the blocks that they go to, in order.  Where each
// kept token lies and its scale are looked up first, all at once, before any scale
// is written; a lane holds those of two tokens.  A block's tokens come from its own
// slots or later ones, so that a wave which has read a block's (or, of larger blocks,
// 64 units of 16 codes of it, in order) may write over them.
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
  ratio = fmaxf(ratio, 0x1p-126f);
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
  const int64_t slab = a.slab0 + (int64_t)blockIdx.y;
  if (nq == 0) return;

  // The path, entries l and l + 64, as far as it is one.
  const int most = min(a.count[b], nq);
  const int32_t* path = a.path + tok;
  const int p0 = l < most ? path[l] : INT32_MAX, p1 = l + 64 < most ? path[l + 64] : INT32_MAX;
  int before0 = __shfl_up(p0, 1), before1 = __shfl_up(p1, 1);
  const int end0 = __shfl(p0, 63);
  before0 = l == 0 ? -1 : before0;
  before1 = l == 0 ? end0 : before1;
  const uint64_t bad0 = ~__ballot(p0 > before0 && p0 < nq), bad1 = ~__ballot(p1 > before1 && p1 < nq);
  const int n = bad0 ? __builtin_ctzll(bad0) : 64 + (bad1 ? __builtin_ctzll(bad1) : 64);
  if (n == 0) return;

  const uint8_t* codes = q.codes + slab * q.s_slab + sb * q.s_b + h * q.s_h;
  float* scales = q.scale + slab * q.c_slab + sb * q.c_b + h * q.c_h;
  auto block_of = [&](int j) -> int64_t {  // -1: none
    if (!q.bt) return j;
    const int64_t blk = q.bt[(int64_t)sb * q.max_blocks + j];
    return (uint64_t)blk >= (uint64_t)q.num_blocks ? -1 : blk;
  };
  // Tokens l and l + 64 of the path: their rows, in 16 bytes from the head's first, and scales.
  uint32_t at[2] = {~0u, ~0u};
  float scale[2] = {1.f, 1.f};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (l + i * 64 >= n) continue;
    const int t = base + (i ? p1 : p0), j = q.d_bs.div(t);
    const int64_t blk = block_of(j);
    if (blk < 0) continue;
    at[i] = (uint32_t)((blk * q.s_blk + (int64_t)(t - j * q.bs) * q.D) >> 4);
    scale[i] = scales[blk * q.c_blk];
  }
  if ((slab & 1) == 0 && q.weight) {
    float* w = q.weight + (((slab >> 1) * q.batch + sb) * q.heads + h) * (int64_t)q.cap + base;
    const float w0 = l < n ? w[p0] : 0.f, w1 = l + 64 < n ? w[p1] : 0.f;
    if (l < n) w[l] = w0;
    if (l + 64 < n) w[l + 64] = w1;
  }

  const int du = q.D / 16;
  struct Unit {
    u32x4 c;
    float scale;
  };
  // Unit u (of this lane; none at `units` and beyond) of the tokens from k0 on.
  auto read = [&](int k0, int u, int units) {
    const int tk = a.d_du.div(min(u, units - 1)), k = k0 + tk, part = u - tk * du;
    const uint32_t x0 = __shfl((int)at[0], k & 63), x1 = __shfl((int)at[1], k & 63);
    const float s0 = __shfl(scale[0], k & 63), s1 = __shfl(scale[1], k & 63);
    const uint32_t x = k < 64 ? x0 : x1;
    Unit y{u32x4{0, 0, 0, 0}, k < 64 ? s0 : s1};
    if (u < units && x != ~0u) y.c = *(const u32x4*)(codes + ((uint64_t)x + part) * 16);
    return y;
  };
  constexpr int kHeld = 4;
  const int last = base + n;
  for (int j = q.d_bs.div(base); j * q.bs < last; ++j) {
    const int lo = max(base, j * q.bs), hi = min(last, (j + 1) * q.bs), k0 = lo - base;
    const int held = lo - j * q.bs, units = (hi - lo) * du;
    const int64_t blk = block_of(j);
    if (blk < 0) continue;
    float* const to_scale = scales + blk * q.c_blk;
    const float old = held ? *to_scale : 0.f;
    Unit x[kHeld];
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      x[i] = Unit{u32x4{0, 0, 0, 0}, 1.f};
      if (i * 64 < units) x[i] = read(k0, l + i * 64, units);
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i) m = amax_of(x[i].c, x[i].scale, m);
    for (int u = kHeld * 64; u < units; u += 64) {
      const Unit y = read(k0, l + u, units);
      m = amax_of(y.c, y.scale, m);
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    const float p = fmaxf(scale_for(m), old), inv = inverse(p);
    u32x4* const out = (u32x4*)(const_cast<uint8_t*>(codes) + blk * q.s_blk);
    u32x4* const to = out + held * du;
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (l + i * 64 < units) to[l + i * 64] = again(x[i].c, x[i].scale * inv);
    for (int u = kHeld * 64; u < units; u += 64) {
      const Unit y = read(k0, l + u, units);
      if (l + u < units) to[l + u] = again(y.c, y.scale * inv);
    }
    if (held && p > old)  // the codes from before, to the larger scale
      for (int u = l; u < held * du; u += 64) out[u] = again(out[u], old * inv);
    if (l == 0) *to_scale = p;
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

hipError_t launch_keep(const KeepArgs& a, uint32_t nslabs, hipStream_t s) {
  const uint32_t waves = (uint32_t)a.nseq * a.q.heads, per = kThreads / 64;
  void* args[] = {const_cast<KeepArgs*>(&a)};
  return hipLaunchKernel((const void*)&keep_kernel, dim3((waves + per - 1) / per, nslabs),
                         dim3(kThreads), args, 0, s);
}

}  // namespace dv
