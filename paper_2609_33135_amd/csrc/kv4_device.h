// kv4_device.h -- device helpers of the 4-bit cache's kernels: addresses of its planes
// and the dequantization of V, whose codes pair channels where the matrix instructions
// want pairs of keys.
#pragma once
#include "kv4_internal.h"
#include "mpfa_device.h"

namespace mpfa {

namespace {

// log2 of the factor P carries into its FP16 rounding.  P is at most 1: with 2^15 it
// stays below the FP16 maximum and keeps its 11 bits down to 2^-29 (2^-14 without),
// where a row of 128K equal keys still sums them exactly enough.
constexpr float kLog2P = 15.0f;
// P is 2^(s lam + bias), bias = 15 - m lam rounded once: off by a factor of up to 2^(2^-24 |bias|),
// which would pass the FP16 maximum and then all bounds as scores grow.  Columns whose bias is
// larger than this (2^-16 of P) take the difference s - m first, which is exact at the maximum
// and finite for all finite inputs, and the bias 15.  For a wave without such a column that is
// one branch a step: 777 tokens 21.6 us, 21.1 without it; 64 contexts of four rows and 2048 keys
// 43.4 and 43.1; 8192 tokens, 32 contexts of 16K to 64K the same.
constexpr float kPlainBias = 256.0f;

// (page, KV head) row of a plane
__device__ __forceinline__ int64_t kv4_row(int64_t page, int h_kv, int hk) { return page * h_kv + hk; }

// Bytes j of the results: channel 2j (even) / 2j + 1 (odd) of the octet, the first key in
// the low nibble, the second in the high one.  a, b: an octet's codes of two keys.
__device__ __forceinline__ uint32_t keys_even(uint32_t a, uint32_t b) { return (a & 0x0F0F0F0Fu) | ((b << 4) & 0xF0F0F0F0u); }
__device__ __forceinline__ uint32_t keys_odd(uint32_t a, uint32_t b) { return ((a >> 4) & 0x0F0F0F0Fu) | (b & 0xF0F0F0F0u); }

// Byte SEL of w: two E2M1 codes as FP16, times m.
template <int SEL>
__device__ __forceinline__ f16x2 fp4_pair_f16(uint32_t w, f16x2 m) {
  return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, SEL) * m;
}

// Exponent shift of a query row whose largest magnitude is a, for keys in units of the tensor
// scale: the row times 2^shift is below 2^15, so its bf16 values are exact in FP16 (11 bits)
// wherever they are above 2^-28 of the largest, and off by at most 2^-39 of it elsewhere.  The
// shift stops where score_scale's factor would leave the normal numbers, 2^(scale's exponent -
// shift) = 2^-123: rows that small have scores below 2^-90.
__device__ __forceinline__ int q_shift(float a, float k_tscale) {
  return a > 0.0f ? min(14 - ilog2f(a), 123 + ilog2f(k_tscale)) : 0;
}
// log2(e) / sqrt(128) for scores in units of the K tensor scale and the row's shift.  The
// exponent stays where the factor is a normal number (2^-126 .. ): 0 times a masked
// score's -inf would be NaN.  Scores are below 2^34 units (2^15 * 2688 * 128): with an exponent
// of at most 90 their scaled values are finite; unequal ones differ by 2^-34 at least, so from
// there on the softmax is the same for every larger factor.
__device__ __forceinline__ float score_scale(float lam, float k_tscale, int shift) {
  return __builtin_ldexpf(lam, min(ilog2f(k_tscale) - shift, 90));
}

// Eight bf16 values times 2^shift as FP16.
__device__ __forceinline__ f16x8 q_operand(u32x4 w, int shift) {
  f16x8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[2 * i] = (_Float16)__builtin_ldexpf(__uint_as_float(w[i] << 16), shift);
    r[2 * i + 1] = (_Float16)__builtin_ldexpf(__uint_as_float(w[i] & 0xFFFF0000u), shift);
  }
  return r;
}
__device__ __forceinline__ float q_amax(u32x4 w) {
  float a = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    a = fmaxf(a, fmaxf(__builtin_fabsf(__uint_as_float(w[i] << 16)), __builtin_fabsf(__uint_as_float(w[i] & 0xFFFF0000u))));
  return a;
}

// Channels 2l and 2l + 1 of a row of the output: O / L * tv, or 0 where nothing was visible.
__device__ __forceinline__ void kv4_store_row(uint16_t* out, float L, float o0, float o1, float tv) {
  const float inv = L > 0.0f ? __frcp_rn(L) : 0.0f;
  const uint32_t lo = bf16_rne(o0 * inv * tv), hi = bf16_rne(o1 * inv * tv);
  *reinterpret_cast<uint32_t*>(out + 2 * (threadIdx.x & 63)) = lo | (hi << 16);
}

// Merge of the partition states of one row (query token and head), `stride` floats apart,
// by WAVES waves: M is the largest m, L = sum f l, O = sum f O with f = 2^(m - M); wave w
// sums partitions w, w + WAVES, .. in order, the waves' sums add in order.  Lane l owns channels 2l and 2l + 1.
template <int WAVES>
__device__ __forceinline__ void kv4_merge_row(const float* st, int64_t stride, int np, float tv, uint16_t* out) {
  __shared__ float part[WAVES][kKv4State];
  const int lane = threadIdx.x & 63, wave = WAVES > 1 ? threadIdx.x >> 6 : 0;
  constexpr int kAhead = 8;
  float2 ml[kAhead], o[kAhead];
  auto load = [&](int q0) {   // partitions q0, q0 + WAVES, ..; past the last it again (not used)
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const float* s = st + min(q0 + j * WAVES, np - 1) * stride;
      ml[j] = *reinterpret_cast<const float2*>(s);
      o[j] = *reinterpret_cast<const float2*>(s + 2 + 2 * lane);
    }
  };
  float M = -INFINITY, L = 0.0f, o0 = 0.0f, o1 = 0.0f;
  if (np > 0) {
    load(wave);   // the first ones beside the maxima
    for (int q = lane; q < np; q += 64) M = fmaxf(M, st[q * stride]);
    for (int off = 32; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor(M, off));
  }
  if (M > -INFINITY) {
    for (int q0 = wave; q0 < np; q0 += kAhead * WAVES) {
      if (q0 > wave) load(q0);
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const float f = q0 + j * WAVES < np ? __builtin_amdgcn_exp2f(ml[j].x - M) : 0.0f;
        L = __builtin_fmaf(f, ml[j].y, L);
        o0 = __builtin_fmaf(f, o[j].x, o0);
        o1 = __builtin_fmaf(f, o[j].y, o1);
      }
    }
  }
  if (WAVES > 1) {
    if (lane == 0) part[wave][0] = L;
    part[wave][2 + 2 * lane] = o0;
    part[wave][3 + 2 * lane] = o1;
    __syncthreads();
    if (wave != 0) return;
    L = o0 = o1 = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      L += part[w][0];
      o0 += part[w][2 + 2 * lane];
      o1 += part[w][3 + 2 * lane];
    }
  }
  kv4_store_row(out, L, o0, o1, tv);
}

}  // namespace

}  // namespace mpfa
