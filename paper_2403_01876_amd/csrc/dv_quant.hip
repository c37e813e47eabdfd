// Rounding a 16-bit stream into an 8-bit cache: e4m3 codes with a power-of-two
// scale for each block of tokens of a head.
//
// A block's elements are contiguous in the stream and, one byte each, in the
// cache.  A group of lanes, a wave at most, holds them in registers while it finds the
// largest magnitude, so that each is read once; blocks too large for that are read
// again (from L2): the prompts below, on the same buffers each time, take 65 us a call
// with a scale for 16 tokens, 73 for 64 and 184 for 1024.
// Bound by HBM: 2 bytes read and 1 written per element.  378 MB (8 prompts of 512
// to 1024 tokens, 40 heads of 128, two layers) 68 us, 5.6 TB/s; a step's 32
// tokens of 20 layers 5 us, of which 2 are the launch and the rest the way to a
// block's place and scale.
#include "dv_attn_internal.h"
#include "dv_scale.h"

namespace dv {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <bool BF16>
__device__ __forceinline__ float lo_f32(uint32_t w) {
  if constexpr (BF16) return __uint_as_float(w << 16);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)w);
}
template <bool BF16>
__device__ __forceinline__ float hi_f32(uint32_t w) {
  if constexpr (BF16) return __uint_as_float(w & 0xffff0000u);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)(w >> 16));
}

// The largest number of the format that the type still holds: 0.9375 * 2^16
// (f16) or * 2^128; 256 / 448 steps above it the type has only infinity.
template <bool BF16>
__device__ __forceinline__ float limit() {
  return BF16 ? __uint_as_float(0x7f700000u) : 61440.f;
}

// Sixteen numbers in eight words to sixteen codes.  inv is a power of two, so
// the products are exact and only the conversion rounds (nearest even).
template <bool BF16>
__device__ __forceinline__ u32x4 encode(const u32x4& a, const u32x4& b, float inv) {
  const float lim = limit<BF16>();
  auto one = [&](float x) {
    const float y = fminf(fmaxf(x, -lim), lim);
    return (x != x ? x : y) * inv;
  };
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w0 = i < 2 ? a[2 * i] : b[2 * i - 4], w1 = i < 2 ? a[2 * i + 1] : b[2 * i - 3];
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(one(lo_f32<BF16>(w0)), one(hi_f32<BF16>(w0)), 0, false);
    r[i] = __builtin_amdgcn_cvt_pk_fp8_f32(one(lo_f32<BF16>(w1)), one(hi_f32<BF16>(w1)), c, true);
  }
  return r;
}

template <bool BF16>
__device__ __forceinline__ float amax_of(const u32x4& a, float m) {
#pragma unroll
  for (int i = 0; i < 4; ++i)  // fmaxf drops NaN
    m = fmaxf(m, fmaxf(fabsf(lo_f32<BF16>(a[i])), fabsf(hi_f32<BF16>(a[i]))));
  return m;
}

// HELD: units that a lane holds.
template <bool BF16, int HELD>
__global__ void __launch_bounds__(kThreads) quant_kernel(QuantArgs a) {
  __shared__ int32_t first[kQSeqs];
  for (int i = threadIdx.x; i < a.nseq; i += kThreads) first[i] = a.item[i];
  __syncthreads();
  const int group = 1 << a.lanes_log2, lane = threadIdx.x & (group - 1);
  const uint32_t item = (blockIdx.x * (uint32_t)kThreads + threadIdx.x) >> a.lanes_log2;
  if (item >= (uint32_t)a.items) return;  // whole groups leave
  // the last sequence whose first item is not past this one (empty sequences
  // share their successor's)
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
  if ((slab & 1) == 0 && (q.weight || q.position)) {  // slots, mapped or not
    const int64_t at = (((slab >> 1) * q.batch + sb) * q.heads + h) * (int64_t)q.cap;
    const int next = q.position && t0 > 0 ? q.position[at + t0 - 1] + 1 : 0;
    for (int t = lo + lane; t < hi; t += group) {
      if (q.weight) q.weight[at + t] = 0.f;
      if (q.position) q.position[at + t] = next + (t - t0);
    }
  }
  const int64_t blk = q.bt ? q.bt[(int64_t)sb * q.max_blocks + j] : j;
  if (q.bt && (uint64_t)blk >= (uint64_t)q.num_blocks) return;
  uint8_t* codes = q.codes + slab * q.s_slab + sb * q.s_b + blk * q.s_blk + h * q.s_h;
  float* scale = q.scale + slab * q.c_slab + sb * q.c_b + blk * q.c_blk + h * q.c_h;
  const int held = lo - j * q.bs;  // slots the block already holds
  const float old = held ? *scale : 0.f;

  const int units = (hi - lo) * (q.D / 16);
  const u32x4* src = (const u32x4*)(a.wire + (int64_t)blockIdx.y * a.w_slab +
                                    ((int64_t)a.tok[b] * q.heads + (int64_t)h * n + (lo - t0)) *
                                        q.D * 2);
  u32x4 x[HELD][2];
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    const int u = lane + i * group;
    if (u < units) {
      x[i][0] = __builtin_nontemporal_load(src + 2 * u);
      x[i][1] = __builtin_nontemporal_load(src + 2 * u + 1);
    } else {
      x[i][0] = x[i][1] = u32x4{0, 0, 0, 0};
    }
  }
#pragma unroll
  for (int i = 0; i < HELD; ++i) m = amax_of<BF16>(x[i][0], amax_of<BF16>(x[i][1], m));
  for (int u = lane + HELD * group; u < units; u += group)
    m = amax_of<BF16>(src[2 * u], amax_of<BF16>(src[2 * u + 1], m));
  for (int o = group >> 1; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  const float p = fmaxf(scale_for(fminf(m, limit<BF16>())), old), inv = inverse(p);

  u32x4* dst = (u32x4*)(codes + (int64_t)held * q.D);
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    const int u = lane + i * group;
    if (u < units) dst[u] = encode<BF16>(x[i][0], x[i][1], inv);
  }
  for (int u = lane + HELD * group; u < units; u += group)
    dst[u] = encode<BF16>(src[2 * u], src[2 * u + 1], inv);
  if (held && p > old) {  // the codes from before, to the larger scale
    u32x4* was = (u32x4*)codes;
    const float down = fmaxf(old * inv, 0x1p-126f);
    for (int u = lane; u < held * (q.D / 16); u += group) {
      u32x4 c = was[u];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[i], down, false);
        const f32x2 v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[i], down, true);
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(v0[0], v0[1], 0, false);
        c[i] = __builtin_amdgcn_cvt_pk_fp8_f32(v1[0], v1[1], w, true);
      }
      was[u] = c;
    }
  }
  if (lane == 0 && p != old) *scale = p;
}

}  // namespace

hipError_t launch_quant(const QuantArgs& a, uint32_t nslabs, hipStream_t s) {
  const bool few = a.held == 2;
  const void* fn = a.bf16 ? few ? (const void*)&quant_kernel<true, 2>
                                : (const void*)&quant_kernel<true, 4>
                   : few  ? (const void*)&quant_kernel<false, 2>
                          : (const void*)&quant_kernel<false, 4>;
  const uint32_t per = kThreads >> a.lanes_log2;
  void* args[] = {const_cast<QuantArgs*>(&a)};
  return hipLaunchKernel(fn, dim3(((uint32_t)a.items + per - 1) / per, nslabs), dim3(kThreads),
                         args, 0, s);
}

}  // namespace dv
