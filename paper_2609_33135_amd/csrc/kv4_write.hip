// kv4_write.hip -- K and V into the 4-bit cache for gfx950: on a sequence's first call
// its statistics (K means, tensor scales), then NVFP4 rows of both.
//
// Every rounding is fixed, so a call's codes are bit-reproducible.  The means come from FP64
// sums: bf16 tokens add exactly in 53 bits, in any order, where the exponents of a channel span
// at most 45 - log2(tokens); beyond that the order counts, which is fixed for a call but goes by
// the call's token counts (how many tokens make a partial, who adds the partials).  Centering is
// one FP32 subtraction, and x -> fl(x - mean) is monotone, so the largest |K - mean| is reached
// at a channel's maximum or minimum and the tokens are read once for it.
#include "kv4_device.h"

#pragma clang fp contract(off)

namespace mpfa {

namespace {

constexpr int64_t kLastLevelCache = (int64_t)256 << 20;
// Where every workgroup of the write pass reads the partials of its sequence itself: up to so
// many of them, and so many reads of one by all workgroups (2 KB each, from L2).  One launch
// less.  8 heads: 777 tokens 12.4 us, 15.1 not; 4000 17.6 and 19.5; eight of 2000, 64000 reads,
// 44.5 and 48.7; but 6000, 47 partials, 26.4 and 23.7; four of 4000, 128000 reads, 50.3 and
// 49.5; eight, 256000, 104 and 92.
constexpr int kFusedPartials = 32;
constexpr int64_t kFusedReads = 100000;
// Tokens per workgroup of the write pass: eight per wave, eight lanes (groups of 16) each.  In
// both passes the KV heads of the same tokens are neighbours in the grid: their rows lie side
// by side in memory (8 heads: 33000 tokens 100 us, 104 head by head; four prompts, 4048 tokens
// together, 18.1 and 19.4; but eight of 4000 92 and 90).
constexpr int kWriteTokens = kKv4WriteTokens;

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

__device__ __forceinline__ u32x4 load16(const uint16_t* src, bool stream) {
  const u32x4* at = reinterpret_cast<const u32x4*>(src);
  return stream ? __builtin_nontemporal_load(at) : *at;
}

// Statistics partial of block blk of sequence b (the blocks of a batch are numbered so
// that no two sequences share one: floor(t0 / tokens) + b, since ceil(n / tokens) more of
// them end at or before the next sequence's first).
__device__ __forceinline__ uint8_t* stat_block(const Kv4WriteParams& p, int64_t t0, int b, int blk, int hk) {
  return p.ws + ((t0 / p.stat_tokens + b + blk) * p.h_kv + hk) * kKv4StatBytes;
}

struct StatPtrs {
  double* sum;
  float *mx, *mn, *v;
};
__device__ __forceinline__ StatPtrs stat_ptrs(uint8_t* s) {
  return {reinterpret_cast<double*>(s), reinterpret_cast<float*>(s + kD * 8), reinterpret_cast<float*>(s + kD * 12),
          reinterpret_cast<float*>(s + kD * 16)};
}

// One workgroup per (stat_tokens tokens, KV head): 16 lanes per token row, 128 rows at a time.
// STREAM: the rows are read past the caches' ordinary replacement.  What does not fit the
// last-level cache is lost to the write pass anyway: 65536 tokens, 8 heads, 182 us of the
// whole call so, 195 not; 16384 tokens, which fit, 52.9 and 51.2.
template <bool STREAM>
__global__ __launch_bounds__(256) void kv4_stats_kernel(Kv4WriteParams p) {
  __shared__ double s_sum[4][kD];
  __shared__ float s_mx[4][kD], s_mn[4][kD], s_v[4];
  const int b = blockIdx.y, hk = blockIdx.x % p.h_kv, blk = blockIdx.x / p.h_kv;
  const int64_t t0 = p.cu_seqlens[b];
  const int n = p.cu_seqlens[b + 1] - (int)t0;
  const int begin = blk * p.stat_tokens, te = min(n, begin + p.stat_tokens);
  if (begin >= n) return;
  const int c = threadIdx.x & 15, row = threadIdx.x >> 4, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double sum[8];
  float mx[8], mn[8], va = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    sum[e] = 0.0;
    mx[e] = -INFINITY;
    mn[e] = INFINITY;
  }
  // eight rows of K and V in flight; rows past the end repeat the last one, whose values
  // change no extreme, and are left out of the sums
  constexpr int kRows = kKv4StatTokens / 16;
  for (int tb = begin; tb < te; tb += kKv4StatTokens) {
    u32x4 kw[kRows], vw[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int64_t t = t0 + min(tb + 16 * i + row, te - 1);
      kw[i] = load16(p.k + t * p.k_stride + hk * kD + 8 * c, STREAM);
      vw[i] = load16(p.v + t * p.v_stride + hk * kD + 8 * c, STREAM);
    }
    auto take = [&](bool whole) {
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const bool mine = whole || tb + 16 * i + row < te;
        va = fmaxf(va, q_amax(vw[i]));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = e & 1 ? bf_hi(kw[i][e >> 1]) : bf_lo(kw[i][e >> 1]);
          sum[e] += mine ? (double)x : 0.0;
          mx[e] = fmaxf(mx[e], x);
          mn[e] = fminf(mn[e], x);
        }
      }
    };
    if (tb + kKv4StatTokens <= te) take(true);   // uniform: no selects
    else take(false);
  }
  // the four rows of a wave, then the four waves
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    for (int off = 16; off <= 32; off <<= 1) {
      sum[e] += __shfl_xor(sum[e], off);
      mx[e] = fmaxf(mx[e], __shfl_xor(mx[e], off));
      mn[e] = fminf(mn[e], __shfl_xor(mn[e], off));
    }
  }
  for (int off = 32; off >= 1; off >>= 1) va = fmaxf(va, __shfl_xor(va, off));
  if (lane < 16) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s_sum[wave][8 * c + e] = sum[e];
      s_mx[wave][8 * c + e] = mx[e];
      s_mn[wave][8 * c + e] = mn[e];
    }
  }
  if (lane == 0) s_v[wave] = va;
  __syncthreads();
  const int t = threadIdx.x;
  const StatPtrs o = stat_ptrs(stat_block(p, t0, b, blk, hk));
  if (t < kD) {
    o.sum[t] = (s_sum[0][t] + s_sum[1][t]) + (s_sum[2][t] + s_sum[3][t]);
    o.mx[t] = fmaxf(fmaxf(s_mx[0][t], s_mx[1][t]), fmaxf(s_mx[2][t], s_mx[3][t]));
    o.mn[t] = fminf(fminf(s_mn[0][t], s_mn[1][t]), fminf(s_mn[2][t], s_mn[3][t]));
  }
  if (t == 0) o.v[0] = fmaxf(fmaxf(s_v[0], s_v[1]), fmaxf(s_v[2], s_v[3]));
}

// What the partials of a (sequence, KV head) come to: the means (BF16, in LDS) and the
// tensor scales, by a workgroup of PARTS x 128 threads: 128 lanes hold the channels, PARTS of
// them share the blocks.
template <int PARTS>
struct StatSmem {
  double sum[PARTS][kD];
  float mx[PARTS][kD], mn[PARTS][kD], v[2 * PARTS], k[2], scale[2];
  __attribute__((aligned(16))) uint16_t mean[kD];
};

template <int PARTS>
__device__ __forceinline__ void finish_stats(const Kv4WriteParams& p, StatSmem<PARTS>& sm, int b, int hk, int64_t t0, int n) {
  const int c = threadIdx.x & (kD - 1), part = threadIdx.x >> 7;
  const int nblk = (n + p.stat_tokens - 1) / p.stat_tokens;
  constexpr int kAhead = 8;
  double sum = 0.0;
  float mx = -INFINITY, mn = INFINITY;
  auto v_of = [&](int blk) { return stat_ptrs(stat_block(p, t0, b, blk, hk)).v[0]; };
  float va = v_of(min((int)threadIdx.x, nblk - 1));   // in flight beside the loads below
  for (int blk0 = part; blk0 < nblk; blk0 += PARTS * kAhead) {   // past the last block it again, without its sum
    double sums[kAhead];
    float mxs[kAhead], mns[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const StatPtrs s = stat_ptrs(stat_block(p, t0, b, min(blk0 + PARTS * i, nblk - 1), hk));
      sums[i] = s.sum[c];
      mxs[i] = s.mx[c];
      mns[i] = s.mn[c];
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      sum += blk0 + PARTS * i < nblk ? sums[i] : 0.0;
      mx = fmaxf(mx, mxs[i]);
      mn = fminf(mn, mns[i]);
    }
  }
  for (int blk = threadIdx.x + PARTS * kD; blk < nblk; blk += PARTS * kD) va = fmaxf(va, v_of(blk));
  for (int off = 32; off >= 1; off >>= 1) va = fmaxf(va, __shfl_xor(va, off));
  sm.sum[part][c] = sum;
  sm.mx[part][c] = mx;
  sm.mn[part][c] = mn;
  if ((threadIdx.x & 63) == 0) sm.v[threadIdx.x >> 6] = va;
  __syncthreads();
  if (threadIdx.x < kD) {
    for (int i = 1; i < PARTS; ++i) {
      sum += sm.sum[i][c];
      mx = fmaxf(mx, sm.mx[i][c]);
      mn = fminf(mn, sm.mn[i][c]);
    }
    sm.mean[c] = p.smooth ? bf16_rne((float)(sum / (double)n)) : 0;
    const float mean = bf16_to_f32(sm.mean[c]);
    float a = fmaxf(__builtin_fabsf(mx - mean), __builtin_fabsf(mn - mean));
    for (int off = 32; off >= 1; off >>= 1) a = fmaxf(a, __shfl_xor(a, off));
    if ((threadIdx.x & 63) == 0) sm.k[threadIdx.x >> 6] = a;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2 * PARTS; ++i) va = fmaxf(va, sm.v[i]);
    sm.scale[0] = tensor_scale(fmaxf(sm.k[0], sm.k[1]));
    sm.scale[1] = tensor_scale(va);
  }
  __syncthreads();
}

template <int PARTS>
__device__ __forceinline__ void store_stats(const Kv4WriteParams& p, const StatSmem<PARTS>& sm, int b, int hk) {
  const int at = b * p.h_kv + hk;
  if (threadIdx.x < kD) p.k_mean[(int64_t)at * kD + threadIdx.x] = sm.mean[threadIdx.x];
  if (threadIdx.x == 0) {
    p.k_tscale[at] = sm.scale[0];
    p.v_tscale[at] = sm.scale[1];
  }
}

// Sequences without tokens keep their statistics.
__global__ __launch_bounds__(1024) void kv4_stats_final_kernel(Kv4WriteParams p) {
  __shared__ StatSmem<8> sm;
  const int b = blockIdx.y, hk = blockIdx.x;
  const int64_t t0 = p.cu_seqlens[b];
  const int n = p.cu_seqlens[b + 1] - (int)t0;
  if (n <= 0) return;
  finish_stats(p, sm, b, hk, t0, n);
  store_stats(p, sm, b, hk);
}

// One group of 16 values: codes of channels 0..7 and 8..15, and the scale byte.
struct Group {
  uint32_t lo, hi, sc;
  float step;   // t * scale
};

// x: the values divided by the tensor scale (exact, a power of two).  Values past the
// format's largest (2688 of them; a frozen tensor scale and a later, larger token)
// saturate, so they are cut at 8192 first and no quotient overflows.  div_by_scale is
// the correctly rounded quotient; its rounding never moves a value onto or over a
// boundary between codes, as a boundary times a scale has 7 bits.
__device__ __forceinline__ Group quantize_group(const float* x, float t) {
  float y[16], a = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    y[i] = fminf(fmaxf(x[i], -8192.0f), 8192.0f);
    a = fmaxf(a, __builtin_fabsf(y[i]));
  }
  Group g;
  g.sc = fp8_sat_pair(0u, div_by_scale(a, 6.0f, kRcp6), 0.0f, false) & 0xFFu;
  const float sd = e4m3_value(g.sc);
  g.step = t * sd;
  g.lo = g.hi = 0u;
  if (g.sc != 0u) {
    const float r = __fdiv_rn(1.0f, sd);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      g.lo = fp4_pair(g.lo, div_by_scale(y[2 * j], sd, r), div_by_scale(y[2 * j + 1], sd, r), 1.0f, j);
      g.hi = fp4_pair(g.hi, div_by_scale(y[8 + 2 * j], sd, r), div_by_scale(y[9 + 2 * j], sd, r), 1.0f, j);
    }
  } else {   // no scale, no value: sign-only codes
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      g.lo |= ((__float_as_uint(y[i]) >> 28) & 8u) << (4 * i);
      g.hi |= ((__float_as_uint(y[8 + i]) >> 28) & 8u) << (4 * i);
    }
  }
  return g;
}

// The values that a group's codes stand for, as bf16 (exact: six bits).  Nothing here reads
// them again: stored past the caches they leave K and V there (16384 tokens, 8 heads, 31
// us, 37 not).
__device__ __forceinline__ void store_values(uint16_t* out, const Group& g) {
  u32x4 w[2];
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const uint32_t c = half ? g.hi : g.lo;
    const f32x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3)};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[half][j] = (__float_as_uint(v[j][0] * g.step) >> 16) | (__float_as_uint(v[j][1] * g.step) & 0xFFFF0000u);
  }
  __builtin_nontemporal_store(w[0], reinterpret_cast<u32x4*>(out));
  __builtin_nontemporal_store(w[1], reinterpret_cast<u32x4*>(out) + 1);
}

__device__ __forceinline__ void load_group(const uint16_t* src, float* x) {
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const u32x4 w = reinterpret_cast<const u32x4*>(src)[half];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[8 * half + 2 * j] = bf_lo(w[j]);
      x[8 * half + 2 * j + 1] = bf_hi(w[j]);
    }
  }
}

// FUSED: every workgroup finishes the statistics itself (see kFusedPartials) and the first of
// each (sequence, KV head) stores them.  Five waves fit a SIMD (four prompts, 4048 tokens
// together, 8 heads: 19.4 us; 21.3 with four, 21.2 with six, which spill; 18.1 with the heads
// side by side).
template <bool FUSED>
__global__ __launch_bounds__(256, FUSED ? 5 : 1) void kv4_write_kernel(Kv4WriteParams p) {
  const int b = blockIdx.y, hk = blockIdx.x % p.h_kv, first = blockIdx.x / p.h_kv * kWriteTokens;
  const int64_t t0 = p.cu_seqlens[b];
  const int n = p.cu_seqlens[b + 1] - (int)t0;
  if (first >= n) return;
  const int g = threadIdx.x & 7, i = first + (threadIdx.x >> 3);
  const int64_t t = t0 + min(i, n - 1);
  const int64_t slot = p.slot_mapping[t];
  float k[16], v[16], m[16], tk, tv;
  load_group(p.k + t * p.k_stride + hk * kD + 16 * g, k);
  load_group(p.v + t * p.v_stride + hk * kD + 16 * g, v);
  if (FUSED) {
    __shared__ StatSmem<2> sm;
    finish_stats(p, sm, b, hk, t0, n);
    if (first == 0) store_stats(p, sm, b, hk);
    load_group(sm.mean + 16 * g, m);
    tk = sm.scale[0];
    tv = sm.scale[1];
  } else {
    if (p.smooth) load_group(p.k_mean + ((int64_t)b * p.h_kv + hk) * kD + 16 * g, m);
    tk = p.k_tscale[b * p.h_kv + hk];
    tv = p.v_tscale[b * p.h_kv + hk];
  }
  if (i >= n) return;
  const int ek = -ilog2f(tk), ev = -ilog2f(tv);
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    if (p.smooth) k[e] -= m[e];
    k[e] = __builtin_ldexpf(k[e], ek);
    v[e] = __builtin_ldexpf(v[e], ev);
  }
  const Group gk = quantize_group(k, tk), gv = quantize_group(v, tv);
  if (slot >= 0 && slot < p.num_pages * kPage) {   // else a padded token: nothing to keep
    const int o = (int)(slot & (kPage - 1));
    const int64_t row = kv4_row(slot / kPage, p.h_kv, hk);
    *reinterpret_cast<uint2*>(p.cache.k_codes + (row * kPage + o) * 64 + 8 * g) = make_uint2(gk.lo, gk.hi);
    p.cache.k_scales[(row * kPage + o) * 8 + g] = (uint8_t)gk.sc;
    uint32_t* vq = reinterpret_cast<uint32_t*>(p.cache.v_codes + (row * 16 + (o >> 2)) * 256) + 8 * g + (o & 3);
    vq[0] = gv.lo;
    vq[4] = gv.hi;
    p.cache.v_scales[(row * 8 + g) * kPage + o] = (uint8_t)gv.sc;
    if (p.cache.weights && g == 0) p.cache.weights[row * kPage + o] = 0.0f;
  }
  const int64_t out = (t * p.h_kv + hk) * kD + 16 * g;
  if (p.k_out) store_values(p.k_out + out, gk);
  if (p.v_out) store_values(p.v_out + out, gv);
}

}  // namespace

hipError_t launch_kv4_write(const Kv4WriteParams& p, hipStream_t stream) {
  if (p.total_tokens == 0 || p.max_seqlen == 0) return hipSuccess;
  const dim3 chunks((p.max_seqlen + kWriteTokens - 1u) / kWriteTokens * p.h_kv, p.batch);
  if (!p.compute_stats) {
    kv4_write_kernel<false><<<chunks, 256, 0, stream>>>(p);
    return hipGetLastError();
  }
  const int blocks = (p.max_seqlen + p.stat_tokens - 1) / p.stat_tokens;
  const dim3 grid((unsigned)blocks * p.h_kv, p.batch);
  if ((int64_t)p.total_tokens * p.h_kv * kD * 4 >= kLastLevelCache) kv4_stats_kernel<true><<<grid, 256, 0, stream>>>(p);
  else kv4_stats_kernel<false><<<grid, 256, 0, stream>>>(p);
  const int64_t reads = (int64_t)p.total_tokens / kWriteTokens * p.h_kv * blocks;
  if (blocks <= kFusedPartials && reads <= kFusedReads) {
    kv4_write_kernel<true><<<chunks, 256, 0, stream>>>(p);
  } else {
    kv4_stats_final_kernel<<<dim3(p.h_kv, p.batch), 1024, 0, stream>>>(p);
    kv4_write_kernel<false><<<chunks, 256, 0, stream>>>(p);
  }
  return hipGetLastError();
}

}  // namespace mpfa
