// Eviction: which tokens of each head stay, and the compaction of what they own.
#include "dv_attn_internal.h"
#include "dv_scale.h"

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
// Which tokens stay: a workgroup takes one head of one sequence.  The k-th largest
// key of the older tokens is found a byte at a time from the top: a histogram of
// that byte (one for each wave) over the keys that agree with what is known, then
// the bin in which the k-th falls, until all of that bin stay or its keys are
// equal.  Keys above it stay, and of those equal to it the first ones.  Then every
// wave counts both in its tokens, and the counts before them place the tokens that
// stay.
// KH * NT weights at a time are in registers: of up to so many each is
// read once, of more once for each histogram and once to place them.
// Bound by latency: one round through memory, the rest in LDS.  512 heads of up to
// 4096 tokens 15 us, 8 heads of 100 6 us.  KH * NT is the least that holds the
// longest sequence: 800 tokens, call 16.6 us with 4 weights a lane, 19.1 with 16;
// 6000 29.2 with 1024 lanes, 37.1 with 256.
// ---------------------------------------------------------------------------
constexpr int kBins = 256;

template <int NT, int KH>
__global__ void __launch_bounds__(NT) evict_select_kernel(EvictArgs a) {
  constexpr int W = NT / 64;
  __shared__ int32_t hist[W][kBins];
  __shared__ int32_t sums[4];
  __shared__ int32_t found[3];  // the bin, how many of it are wanted, its keys
  __shared__ int2 counts[KH * W], totals;
  const int tid = threadIdx.x, l = tid & 63, wave = tid >> 6;
  const int b = blockIdx.x / (uint32_t)a.s.heads, h = blockIdx.x - b * a.s.heads, sb = a.b0 + b;
  const int layer = blockIdx.y;
  const int n = a.len[b], k = min(n, a.keep[b]), r = min(a.recent, k);
  const int old = n - r, want = k - r;  // older tokens, and how many of them stay
  const int64_t row = ((int64_t)(a.l0 + layer) * a.s.batch + sb) * a.s.heads + h;
  const float* w = a.s.weight + row * a.s.cap;
  if (k == 0) return;

  float held[KH];
  auto load = [&](int t0) {
#pragma unroll
    for (int i = 0; i < KH; ++i) {
      held[i] = w[min(t0 + i * NT + tid, n - 1)];  // (no condition: all at once)
    }
  };
  load(0);
  const bool several = n > KH * NT;
  uint32_t line = 0;  // the want-th largest key, as far as it is known
  int equal = want;   // how many of the keys equal to it stay
  const bool choose = want > 0 && want < old;
  if (choose) {
    for (int shift = 24; shift >= 0; shift -= 8) {
#pragma unroll
      for (int i = 0; i < kBins / 64; ++i) hist[wave][i * 64 + l] = 0;
      for (int t0 = 0; t0 < old; t0 += KH * NT) {
        if (several) load(t0);
#pragma unroll
        for (int i = 0; i < KH; ++i) {
          if (t0 + i * NT >= old) break;
          const uint32_t key = key_of(held[i]);
          const bool agrees = shift == 24 || (key ^ line) >> ((shift + 8) & 31) == 0;
          if (t0 + i * NT + tid < old && agrees) atomicAdd(&hist[wave][(key >> shift) & 255], 1);
        }
      }
      __syncthreads();
      int32_t c = 0, above = 0;  // thread tid < 256: bin 255 - tid
      if (tid < kBins) {
#pragma unroll
        for (int i = 0; i < W; ++i) c += hist[i][kBins - 1 - tid];
        above = c;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) {
          const int32_t y = __shfl_up(above, x);
          if (l >= x) above += y;
        }
        if (l == 63) sums[wave] = above;
        above -= c;
      }
      __syncthreads();
      if (tid < kBins) {
        for (int i = 0; i < 4; ++i) above += i < wave ? sums[i] : 0;
        if (above < equal && equal <= above + c) {
          found[0] = kBins - 1 - tid;
          found[1] = equal - above;
          found[2] = c;
        }
      }
      __syncthreads();
      line |= (uint32_t)found[0] << shift;
      equal = found[1];
      if (equal == found[2] && line > 0) {  // all of the bin stay: the line lies below it
        line -= 1;
        equal = 0;
        break;
      }
    }
  }

  int32_t* kept = a.kept + (((int64_t)layer * a.s.batch + sb) * a.s.heads + h) * a.kept_stride;
  const int32_t* p = a.s.position ? a.s.position + row * a.s.cap : nullptr;
  float* dw = a.d.weight ? a.d.weight + row * a.d.cap : nullptr;
  int32_t* dp = a.d.position ? a.d.position + row * a.d.cap : nullptr;
  int more = 0, same = 0;  // tokens before this round above the line, and on it
  for (int t0 = 0; t0 < n; t0 += KH * NT) {
    if (several) load(t0);
    int32_t pos[KH];
    if (p && dp) {
#pragma unroll
      for (int i = 0; i < KH; ++i) {
        pos[i] = p[min(t0 + i * NT + tid, n - 1)];
      }
    }
    uint64_t ups[KH], ons[KH];
#pragma unroll
    for (int i = 0; i < KH; ++i) {
      const int t = t0 + i * NT + tid;
      const uint32_t key = key_of(held[i]);
      const bool up = t < n && (t >= old || (choose ? key > line : want == old));
      const bool on = t < old && choose && key == line;
      ups[i] = __ballot(up);
      ons[i] = __ballot(on);
      if (l == 0) counts[i * W + wave] = make_int2(__popcll(ups[i]), __popcll(ons[i]));
    }
    __syncthreads();  // and what this round reads has been read: dst may be src
    if (wave == 0) {  // sums of the counts before each, a lane to each of 64 at a time
      int x0 = more, y0 = same;
#pragma unroll
      for (int g = 0; g < KH * W; g += 64) {
        const int2 c = g + l < KH * W ? counts[g + l] : make_int2(0, 0);
        int x = c.x, y = c.y;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const int u = __shfl_up(x, o), v = __shfl_up(y, o);
          if (l >= o) {
            x += u;
            y += v;
          }
        }
        if (g + l < KH * W) counts[g + l] = make_int2(x0 + x - c.x, y0 + y - c.y);
        x0 += __builtin_amdgcn_readlane(x, 63);
        y0 += __builtin_amdgcn_readlane(y, 63);
      }
      if (l == 0) totals = make_int2(x0, y0);
    }
    __syncthreads();
    more = totals.x;
    same = totals.y;
    const uint64_t mine = (1ull << l) - 1;
#pragma unroll
    for (int i = 0; i < KH; ++i) {
      const int t = t0 + i * NT + tid;
      const int2 base = counts[i * W + wave];
      const int level = base.y + __popcll(ons[i] & mine);
      const bool up = (ups[i] >> l) & 1, on = (ons[i] >> l) & 1;
      if (up || (on && level < equal)) {
        const int at = base.x + __popcll(ups[i] & mine) + (choose ? min(level, equal) : 0);
        kept[at] = t;
        if (dw) dw[at] = held[i];
        if (dp) dp[at] = p ? pos[i] : t;
      }
    }
    __syncthreads();
  }
}

// The largest magnitude of sixteen codes times their scale, and m; NaN is left out.
__device__ __forceinline__ float amax_of(const u32x4& c, float scale, float m) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[i], scale, false);
    const f32x2 y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c[i], scale, true);
    m = fmaxf(m, fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(y[0]), fabsf(y[1]))));
  }
  return m;
}
// The codes of ratio times what sixteen codes stand for.
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

// ---------------------------------------------------------------------------
// Codes and scales: a workgroup takes a group of blocks of the result, keys and
// values.  It first looks up where each of their tokens lies and its scales (LDS),
// then a wave takes a block of one half at a time: its tokens' rows come from
// memory, the largest magnitude gives the new scale, and since scales are powers
// of two the codes change only where a smaller one grows past them.  The next
// block's rows are on their way meanwhile.
// In place a workgroup takes all of a head's blocks in order, four at a time: a
// block's tokens come from its own slots or later ones, so once the four waves
// have read, what they write over is no longer needed.
// Bound by HBM: 286 MB (32 sequences of 128 to 4096 tokens, 8 heads of 128, half
// stay) 75 us, 3.8 TB/s, of rows of 128 bytes from places that the weights choose;
// 148 MB are read and 140 written, no more than the work needs.
// Stores go past the caches: 75.6 us, through them 78.6.
// On the same buffers each time, the eviction takes 74 us a call, and in place, with
// positions and weights to move too, 151; of one sequence of 131071 tokens, 8 heads,
// 0.36 ms and 3.4.
// ---------------------------------------------------------------------------
constexpr int kHeld = 4;  // units of 16 codes that a lane holds: a block has 64 times as many

__global__ void __launch_bounds__(kThreads) evict_move_kernel(EvictArgs a) {
  extern __shared__ uint32_t table[];  // place, key scale, value scale of a group's tokens
  const int tid = threadIdx.x, l = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int below = 0;
  for (int i = 0; i < a.nseq; i += 64)
    below += __popcll(__ballot(a.item[i + l] <= (int)blockIdx.x));
  const int b = __builtin_amdgcn_readfirstlane(below - 1), sb = a.b0 + b;
  const int k = min(a.len[b], a.keep[b]);
  const QLayout &s = a.s, &d = a.d;
  const int blocks = d.d_bs.div(k + d.bs - 1);
  const int groups = a.in_place ? 1 : (blocks + a.group - 1) / a.group;
  const int item = (int)blockIdx.x - a.item[b];
  const int h = __builtin_amdgcn_readfirstlane(item / groups), g0 = item - h * groups;
  const int layer = blockIdx.y, du = s.D / 16, span = a.group * d.bs;
  const int64_t slab = 2 * ((int64_t)a.l0 + layer);
  const int32_t* kept = a.kept + (((int64_t)layer * a.s.batch + sb) * a.s.heads + h) *
                                     a.kept_stride;
  const uint8_t* from = s.codes + slab * s.s_slab + sb * s.s_b + h * s.s_h;
  const float* from_scale = s.scale + slab * s.c_slab + sb * s.c_b + h * s.c_h;
  uint8_t* to = d.codes + slab * d.s_slab + sb * d.s_b + h * d.s_h;
  float* to_scale = d.scale + slab * d.c_slab + sb * d.c_b + h * d.c_h;
  float* scales = (float*)table + span;

  for (int g = g0; g * a.group < blocks; g += groups) {
    const int j0 = g * a.group, tokens = min(span, k - j0 * d.bs);
    for (int i = tid; i < tokens; i += kThreads) {
      const int t = kept[j0 * d.bs + i], sj = s.d_bs.div(t);
      int64_t blk = s.bt ? s.bt[(int64_t)sb * s.max_blocks + sj] : sj;
      const bool hole = s.bt && (uint64_t)blk >= (uint64_t)s.num_blocks;
      table[i] = hole ? ~0u : (uint32_t)((blk * s.s_blk + (int64_t)(t - sj * s.bs) * s.D) >> 4);
      // (zeros times another block's scale, which nothing may have written, may be NaN)
      scales[i] = hole ? 1.f : from_scale[blk * s.c_blk];
      scales[span + i] = hole ? 1.f : from_scale[blk * s.c_blk + s.c_slab];
    }
    __syncthreads();
    // jobs: blocks j0 + wave + 4 x, keys then values
    struct Job {
      u32x4 c[kHeld];
      float scale[kHeld];
    };
    const int jobs = 2 * ((min(a.group, blocks - j0) + 3) / 4);
    auto units_of = [&](int job) {
      const int j = j0 + wave + 4 * (job >> 1);
      return j < blocks ? min(d.bs, k - j * d.bs) * du : 0;
    };
    auto read = [&](Job& x, int job) {
      const int first = (wave + 4 * (job >> 1)) * d.bs, units = units_of(job);
#pragma unroll
      for (int i = 0; i < kHeld; ++i) {
        const int u = l + i * 64;
        x.c[i] = u32x4{0, 0, 0, 0};
        x.scale[i] = 1.f;
        if (u < units) {
          const int tok = a.d_du.div(u), part = u - tok * du;
          const uint32_t at = table[first + tok];
          if (at != ~0u)
            x.c[i] = *(const u32x4*)(from + (job & 1) * s.s_slab + ((uint64_t)at + part) * 16);
          x.scale[i] = scales[(job & 1) * span + first + tok];
        }
      }
    };
    auto write = [&](const Job& x, int job) {
      const int j = j0 + wave + 4 * (job >> 1), units = units_of(job);
      float m = 0.f;
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (i * 64 < units) m = amax_of(x.c[i], x.scale[i], m);
#pragma unroll
      for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
      if (units == 0) return;
      const int64_t blk = d.bt ? d.bt[(int64_t)sb * d.max_blocks + j] : j;
      if (d.bt && (uint64_t)blk >= (uint64_t)d.num_blocks) return;
      const float p = scale_for(m), inv = inverse(p);
      u32x4* out = (u32x4*)(to + (job & 1) * d.s_slab + blk * d.s_blk);
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (l + i * 64 < units)
          __builtin_nontemporal_store(again(x.c[i], x.scale[i] * inv), out + l + i * 64);
      if (l == 0) to_scale[(job & 1) * d.c_slab + blk * d.c_blk] = p;
    };
    Job x, y;
    read(x, 0);
    for (int job = 0; job < jobs; job += 2) {  // jobs are even
      read(y, job + 1);
      if (a.in_place) __syncthreads();  // all four waves have read their two blocks
      write(x, job);
      if (job + 2 < jobs) read(x, job + 2);
      write(y, job + 1);
    }
    __syncthreads();
  }
}

// The same for blocks too large to be held, read again after their scale is known.
// In place a workgroup is one wave and takes a head's blocks in order, 64 units of
// a block in order: what it writes over has been read.
// Blocks of 64 tokens instead of 16 in the case above: 134 us a call, in place 349.
__global__ void __launch_bounds__(kThreads) evict_move_large_kernel(EvictArgs a, int groups) {
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
  for (int j = g * waves + wave; j < blocks; j += groups * waves) {
    const int units = min(d.bs, k - j * d.bs) * du;
    float m = 0.f, x;
    for (int u = l; u < units; u += 64) {
      const u32x4 c = read(j, u, &x);
      m = amax_of(c, x, m);
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    const int64_t blk = d.bt ? d.bt[(int64_t)sb * d.max_blocks + j] : j;
    if (d.bt && (uint64_t)blk >= (uint64_t)d.num_blocks) continue;
    const float p = scale_for(m), inv = inverse(p);
    u32x4* out = (u32x4*)(to + blk * d.s_blk);
    for (int u = l; u < units; u += 64) {
      const u32x4 c = read(j, u, &x);
      out[u] = again(c, x * inv);
    }
    if (l == 0) to_scale[blk * d.c_blk] = p;
  }
}

}  // namespace

hipError_t launch_evict_select(const EvictArgs& a, hipStream_t s) {
  // As few weights to a lane as hold the longest sequence.
  const int lanes = evict_select_lanes(a.most);
  const void* fn = lanes == 1024      ? (const void*)&evict_select_kernel<1024, 16>
                   : a.most > 4 * 256 ? (const void*)&evict_select_kernel<256, 16>
                                      : (const void*)&evict_select_kernel<256, 4>;
  void* args[] = {const_cast<EvictArgs*>(&a)};
  return hipLaunchKernel(fn, dim3((uint32_t)a.nseq * a.s.heads, a.nl), dim3(lanes), args, 0, s);
}

bool evict_blocks_held(int64_t bs, int64_t D) { return bs * D <= kHeld * 1024; }

hipError_t launch_evict_move(const EvictArgs& a, hipStream_t s) {
  EvictArgs x = a;
  if (evict_blocks_held(a.d.bs, a.s.D)) {
    void* args[] = {&x};
    return hipLaunchKernel((const void*)&evict_move_kernel, dim3((uint32_t)a.items, a.nl),
                           dim3(kThreads), args, (size_t)a.group * a.d.bs * 12, s);
  }
  const int waves = a.in_place ? 1 : 4;
  int groups = a.in_place ? 1 : (a.blocks + waves - 1) / waves;
  void* args[] = {&x, &groups};
  return hipLaunchKernel((const void*)&evict_move_large_kernel,
                         dim3((uint32_t)a.nseq * a.s.heads * groups, 2 * a.nl), dim3(waves * 64),
                         args, 0, s);
}

}  // namespace dv
