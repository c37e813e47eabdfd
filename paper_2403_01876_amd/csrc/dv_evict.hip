// Eviction: which tokens of each head stay, and the compaction of what they own.
#include "dv_attn_internal.h"

namespace dv {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Numbers in their order as unsigned integers; -0 as 0, NaN below all.
__device__ __forceinline__ uint32_t key_of(float w) {
  const uint32_t b = __float_as_uint(w + 0.f);
  return w != w ? 0 : b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u);
}

// ---------------------------------------------------------------------------
// A workgroup takes one head of one sequence.  The k-th largest key of the older
// tokens is found a byte at a time from the top: a histogram of that byte over
// the keys that agree with what is known, then the bin in which the k-th falls.
// Keys above it stay, and of those equal to it the first ones; a pass over the
// tokens in order counts both and writes slots, weights and positions.
// The first kKeys * NT keys are held in registers, the others read each time.
// ---------------------------------------------------------------------------
constexpr int kKeys = 16;

template <int NT>
__global__ void __launch_bounds__(NT) evict_select_kernel(EvictArgs a) {
  __shared__ int32_t hist[256];
  __shared__ uint32_t found[2];  // the bin, and how many of it are wanted
  __shared__ int2 counts[2][NT / 64];
  const int tid = threadIdx.x, l = tid & 63, wave = tid >> 6;
  const int b = blockIdx.x / (uint32_t)a.s.heads, h = blockIdx.x - b * a.s.heads, sb = a.b0 + b;
  const int layer = blockIdx.y;
  const int n = a.len[b], k = min(n, a.keep[b]), r = min(a.recent, k);
  const int old = n - r, want = k - r;  // older tokens, and how many of them stay
  const int64_t row = ((int64_t)(a.l0 + layer) * a.s.batch + sb) * a.s.heads + h;
  const float* w = a.s.weight + row * a.s.cap;

  uint32_t keys[kKeys];
  if (want > 0 && want < old) {
#pragma unroll
    for (int i = 0; i < kKeys; ++i) keys[i] = i * NT + tid < old ? key_of(w[i * NT + tid]) : 0;
  }
  uint32_t line = 0;  // the want-th largest key, as far as it is known
  int equal = want;   // how many of the keys equal to it stay
  if (want > 0 && want < old) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += NT) hist[i] = 0;
      __syncthreads();
      auto count = [&](uint32_t key) {
        if (shift == 24 || key >> ((shift + 8) & 31) == line >> ((shift + 8) & 31))
          atomicAdd(&hist[(key >> shift) & 255], 1);
      };
#pragma unroll
      for (int i = 0; i < kKeys; ++i)
        if (i * NT + tid < old) count(keys[i]);
      for (int t = kKeys * NT + tid; t < old; t += NT) count(key_of(w[t]));
      __syncthreads();
      if (wave == 0) {  // lane l: bins 255 - 4 l and the three below
        int32_t c[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += c[i] = hist[255 - 4 * l - i];
        int32_t above = sum;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) {
          const int32_t y = __shfl_up(above, x);
          if (l >= x) above += y;
        }
        above -= sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (above < equal && equal <= above + c[i]) {
            found[0] = 255 - 4 * l - i;
            found[1] = equal - above;
          }
          above += c[i];
        }
      }
      __syncthreads();
      line |= found[0] << shift;
      equal = found[1];
    }
  }

  int32_t* kept = a.kept + (((int64_t)layer * a.s.batch + sb) * a.s.heads + h) * a.kept_stride;
  const int32_t* p = a.s.position ? a.s.position + row * a.s.cap : nullptr;
  float* dw = a.d.weight ? a.d.weight + row * a.d.cap : nullptr;
  int32_t* dp = a.d.position ? a.d.position + row * a.d.cap : nullptr;
  int more = 0, same = 0;  // tokens before this step above the line, and on it
  for (int t0 = 0, step = 0; t0 < n; t0 += NT, step ^= 1) {
    const int t = t0 + tid;
    const float wt = t < n ? w[t] : 0.f;
    const int32_t pt = t < n && p ? p[t] : t;
    bool up = t < n, on = false;
    if (t < old) {
      const uint32_t key = key_of(wt);
      up = want == old || (want > 0 && key > line);
      on = !up && want > 0 && key == line;
    }
    const uint64_t ups = __ballot(up), ons = __ballot(on);
    if (l == 0) counts[step][wave] = make_int2(__popcll(ups), __popcll(ons));
    __syncthreads();  // and every load of this step is done: dst may be src
    int before = more, level = same;
    for (int i = 0; i < NT / 64; ++i) {
      const int2 c = counts[step][i];
      before += i < wave ? c.x : 0;
      level += i < wave ? c.y : 0;
      more += c.x;
      same += c.y;
    }
    const uint64_t mine = (1ull << l) - 1;
    before += __popcll(ups & mine);
    level += __popcll(ons & mine);
    if (up || (on && level < equal)) {
      const int at = before + min(level, equal);
      kept[at] = t;
      if (dw) dw[at] = wt;
      if (dp) dp[at] = pt;
    }
  }
}

// ---------------------------------------------------------------------------
// Codes and scales: a wave takes one block of the result.  Its tokens are read
// (rows of head_dim bytes), the largest magnitude gives the new scale, and since
// scales are powers of two the codes change only where a smaller one grows past
// them.  In place a workgroup takes all of a head's blocks in order, four at a
// time: a block's tokens come from its own slots or later ones, so once the four
// waves have read, what they write over is no longer needed.  (A block too large
// for a wave's registers is read again after its scale is known; in place such
// blocks are taken one at a time, 64 units in order, which keeps that true.)
// Bound by HBM.
// ---------------------------------------------------------------------------
constexpr int kHeld = 4;

__global__ void __launch_bounds__(kThreads) evict_move_kernel(EvictArgs a, int groups) {
  const int l = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int g = blockIdx.x % (uint32_t)groups, bh = blockIdx.x / (uint32_t)groups;
  const int b = bh / a.s.heads, h = bh - b * a.s.heads, sb = a.b0 + b;
  const int k = min(a.len[b], a.keep[b]);
  const int layer = blockIdx.y >> 1;
  const int64_t slab = 2 * (int64_t)a.l0 + blockIdx.y;
  const int32_t* kept = a.kept + (((int64_t)layer * a.s.batch + sb) * a.s.heads + h) *
                                     a.kept_stride;
  const QLayout &s = a.s, &d = a.d;
  const uint8_t* from = s.codes + slab * s.s_slab + sb * s.s_b + h * s.s_h;
  const float* from_scale = s.scale + slab * s.c_slab + sb * s.c_b + h * s.c_h;
  uint8_t* to = d.codes + slab * d.s_slab + sb * d.s_b + h * d.s_h;
  float* to_scale = d.scale + slab * d.c_slab + sb * d.c_b + h * d.c_h;
  const int du = s.D / 16, blocks = d.d_bs.div(k + d.bs - 1);

  // Sixteen codes of unit u of the result's block j, and their scale.
  auto read = [&](int j, int u, float* scale) {
    const int tok = a.d_du.div(u), part = u - tok * du;
    const int t = kept[j * d.bs + tok], sj = s.d_bs.div(t);
    int64_t blk = s.bt ? s.bt[(int64_t)sb * s.max_blocks + sj] : sj;
    *scale = 1.f;
    if (s.bt && (uint64_t)blk >= (uint64_t)s.num_blocks) return u32x4{0, 0, 0, 0};
    *scale = from_scale[blk * s.c_blk];
    return *(const u32x4*)(from + blk * s.s_blk + (int64_t)(t - sj * s.bs) * s.D + part * 16);
  };
  auto amax = [&](const u32x4& c, float scale, float m) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[i], scale, false);
      const f32x2 y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[i], scale, true);
      m = fmaxf(m, fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(y[0]), fabsf(y[1]))));
    }
    return m;
  };
  auto again = [&](u32x4 c, float ratio) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[i], ratio, false);
      const f32x2 y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[i], ratio, true);
      const int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
      c[i] = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], w, true);
    }
    return c;
  };

  const int step = groups * waves;
  for (int j0 = g * waves; j0 < blocks; j0 += step) {
    const int j = j0 + wave;
    const int units = j < blocks ? min(d.bs, k - j * d.bs) * du : 0;
    u32x4 c[kHeld];
    float scale[kHeld], m = 0.f;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int u = l + i * 64;
      c[i] = u32x4{0, 0, 0, 0};
      scale[i] = 1.f;
      if (u < units) c[i] = read(j, u, &scale[i]);
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i) m = amax(c[i], scale[i], m);
    for (int u = l + kHeld * 64; u < units; u += 64) {
      float x;
      const u32x4 y = read(j, u, &x);
      m = amax(y, x, m);
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    if (a.in_place) __syncthreads();
    int64_t blk = 0;
    bool hole = units == 0;
    if (!hole) {
      blk = d.bt ? d.bt[(int64_t)sb * d.max_blocks + j] : j;
      hole = d.bt && (uint64_t)blk >= (uint64_t)d.num_blocks;
    }
    if (!hole) {
      const float p = scale_for(m), inv = inverse(p);
      u32x4* out = (u32x4*)(to + blk * d.s_blk);
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (l + i * 64 < units) out[l + i * 64] = again(c[i], fmaxf(scale[i] * inv, 0x1p-126f));
      for (int u = l + kHeld * 64; u < units; u += 64) {
        float x;
        const u32x4 y = read(j, u, &x);
        out[u] = again(y, fmaxf(x * inv, 0x1p-126f));
      }
      if (l == 0) to_scale[blk * d.c_blk] = p;
    }
    if (a.in_place) __syncthreads();
  }
}

}  // namespace

hipError_t launch_evict_select(const EvictArgs& a, hipStream_t s) {
  const bool wide = a.most > kKeys * 256;
  const void* fn = wide ? (const void*)&evict_select_kernel<1024>
                        : (const void*)&evict_select_kernel<256>;
  void* args[] = {const_cast<EvictArgs*>(&a)};
  return hipLaunchKernel(fn, dim3((uint32_t)a.nseq * a.s.heads, a.nl), dim3(wide ? 1024 : 256),
                         args, 0, s);
}

hipError_t launch_evict_move(const EvictArgs& a, hipStream_t s) {
  const int waves = a.in_place && (int64_t)a.s.bs * a.s.D > kHeld * 1024 ? 1 : 4;
  int groups = a.in_place ? 1 : (a.blocks + waves - 1) / waves;
  void* args[] = {const_cast<EvictArgs*>(&a), &groups};
  return hipLaunchKernel((const void*)&evict_move_kernel,
                         dim3((uint32_t)a.nseq * a.s.heads * groups, 2 * a.nl), dim3(waves * 64),
                         args, 0, s);
}

}  // namespace dv
