// linear_decode.hip -- linear attention with a decay, one or a few new tokens per sequence, for gfx950.
//
// S_t = a_t S_{t-1} + k_t v_t^T, o_t = scale q_t^T S_t in FP32.  Bound by the state's 64 KB per KV head, read
// and written once: the rows of a call are taken one after the other with the state in registers.  128 sequences of
// 32:32 heads, a row each, take 105 us (537 MB, 5.1 TB/s, a large copy's rate), 64 of 40:8 heads 13.6 (67 MB, 4.9)
// and with four rows each 19.4 to 20.2, since 20 dot products a column and the staging of rows are vector and LDS work
// that the state's loads and stores do not hide in full (22.2 over twelve sets of inputs, none of which stays in the
// cache; within it a copy of as many bytes reaches 8 TB/s).  32 columns a workgroup: 256 threads hold them in 16
// registers each, and one sequence of eight KV heads has 32 workgroups.
#include "linear_internal.h"
#include "mpfa_device.h"

namespace mpfa {

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kCols = 32;              // columns of the state per workgroup: four workgroups a state
constexpr int kLanes = kCols / 4;      // lanes side by side on a row of it
constexpr int kRows = 256 / kLanes;    // rows at a time
constexpr int kEach = kD / kRows;      // a thread's, one after the other
static_assert(kEach == 4, "one vector of k, of q");
// Rows of queries (token and head) between two barriers, and with their keys: what leaves LDS for eight workgroups
// a unit (32 staged rows leave it for five: 64 sequences of 40:8 heads 15.6 us instead of 13.7, with four rows each
// 25.0 instead of 23.0; 18 are as fast but for 16 rows of four heads, 14.1 instead of 13.0).
constexpr int kPairs = 16;
constexpr int kStaged = 20;
constexpr int kTokens = kStaged / 2;   // at most

// Eight BF16 as FP32.
__device__ __forceinline__ void widen(const u32x4& w, float* to) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
    reinterpret_cast<f32x4*>(to)[i] = (f32x4){__uint_as_float(w[2 * i] << 16), __uint_as_float(w[2 * i] & 0xFFFF0000u),
                                              __uint_as_float(w[2 * i + 1] << 16), __uint_as_float(w[2 * i + 1] & 0xFFFF0000u)};
}

// Sums over the eight lanes of a wave that hold the same four columns: column 2 (lane / 16 % 2) + lane / 32 of the
// four.  A swap of two registers' halves (or rows of 16 lanes) leaves in each half one column's values of both, so
// every step also halves the values that are left.
static_assert(kLanes == 8, "rows of a wave");
__device__ __forceinline__ float rows_sum(const f32x4& x) {
  float y[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[2 * i]), __float_as_uint(x[2 * i + 1]), false, false);
    y[i] = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(y[0]), __float_as_uint(y[1]), false, false);
  const float z = __uint_as_float(b[0]) + __uint_as_float(b[1]);
  return z + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(z), 0x128, 0xF, 0xF, false));   // 8 lanes on in 16
}

// One workgroup per (sequence, KV head, kCols columns of the state).
__global__ __launch_bounds__(256) void linear_decode_kernel(LinearParams p) {
  __shared__ float s_row[kStaged][kD], s_v[kTokens][kCols], s_a[kTokens];   // queries, then keys
  __shared__ float s_sum[4][kPairs][kCols];
  constexpr int kParts = kD / kCols;
  const int part = blockIdx.x % kParts, hk = blockIdx.x / kParts % p.h_kv, b = blockIdx.x / kParts / p.h_kv;
  const int tid = threadIdx.x, c = tid % kLanes, row = tid / kLanes, lane = tid & 63, wave = tid >> 6;
  const int grp = p.h_q / p.h_kv, heads = min(grp, kPairs), tokens = min(kPairs / heads, kStaged / (heads + 1));
  float (*const s_k)[kD] = &s_row[tokens * heads];
  const int64_t t0 = (int64_t)b * p.q_tokens;
  const int src = p.state_src[b], dst = p.state_dst[b];
  f32x4 st[kEach];
  if (src >= 0) {
    const float* from = p.states + ((int64_t)src * p.h_kv + hk) * kLinState + part * kCols + 4 * c;
#pragma unroll
    for (int i = 0; i < kEach; ++i) st[i] = *reinterpret_cast<const f32x4*>(from + (kEach * row + i) * kD);
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i) st[i] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
  }
  for (int r0 = 0; r0 < p.q_tokens; r0 += tokens) {
    const int nr = min(tokens, p.q_tokens - r0);
    for (int h0 = 0; h0 < grp; h0 += heads) {   // more than one turn: a token at a time
      const int nh = min(heads, grp - h0);
      __syncthreads();
      {   // 16 threads a row
        const int i = tid >> 4, at = 8 * (tid & 15);
        if (i < nr * nh) {
          const uint16_t* q = p.q + (t0 + r0 + i / nh) * p.q_stride + (hk * grp + h0 + i % nh) * kD;
          widen(*reinterpret_cast<const u32x4*>(q + at), &s_row[i][at]);
        }
        if (h0 == 0 && i < nr) {
          const int64_t t = t0 + r0 + i;
          widen(*reinterpret_cast<const u32x4*>(p.k + t * p.k_stride + hk * kD + at), &s_k[i][at]);
          if (at < kCols) widen(*reinterpret_cast<const u32x4*>(p.v + t * p.v_stride + hk * kD + part * kCols + at), &s_v[i][at]);
          if (at == kCols) s_a[i] = expf(fminf(fmaxf(p.log_decay[t * p.decay_stride + hk], kLinLeastDecay), 0.0f));
        }
      }
      __syncthreads();
      for (int r = 0; r < nr; ++r) {
        if (h0 == 0) {
          const float a = s_a[r];
          const f32x4 v = *reinterpret_cast<const f32x4*>(&s_v[r][4 * c]), k = *reinterpret_cast<const f32x4*>(&s_k[r][kEach * row]);
#pragma unroll
          for (int i = 0; i < kEach; ++i) st[i] = st[i] * a + v * k[i];
        }
        for (int h = 0; h < nh; ++h) {
          const f32x4 q = *reinterpret_cast<const f32x4*>(&s_row[r * nh + h][kEach * row]);
          f32x4 o = st[0] * q[0];
#pragma unroll
          for (int i = 1; i < kEach; ++i) o += st[i] * q[i];
          const float sum = rows_sum(o);
          if (!(lane & 8)) s_sum[wave][r * nh + h][4 * c + 2 * (lane >> 4 & 1) + (lane >> 5)] = sum;
        }
      }
      __syncthreads();
      if (tid < nr * nh * kLanes) {
        const int i = tid / kLanes, x = tid % kLanes;
        f32x4 w[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) w[n] = *reinterpret_cast<const f32x4*>(&s_sum[n][i][4 * x]);
        const f32x4 o = ((w[0] + w[1]) + (w[2] + w[3])) * p.scale;
        uint16_t* to = p.out + ((t0 + r0 + i / nh) * p.h_q + hk * grp + h0 + i % nh) * kD + part * kCols + 4 * x;
        *reinterpret_cast<u32x2*>(to) = (u32x2){bf16_rne(o[0]) | (uint32_t)bf16_rne(o[1]) << 16, bf16_rne(o[2]) | (uint32_t)bf16_rne(o[3]) << 16};
      }
    }
  }
  if (dst >= 0) {   // read again a step of the whole model later: streamed past the cache (23.0 -> 21.6 us, 109 -> 105)
    float* to = p.states + ((int64_t)dst * p.h_kv + hk) * kLinState + part * kCols + 4 * c;
#pragma unroll
    for (int i = 0; i < kEach; ++i) __builtin_nontemporal_store(st[i], reinterpret_cast<f32x4*>(to + (kEach * row + i) * kD));
  }
}

}  // namespace

hipError_t launch_linear_decode(const LinearParams& p, hipStream_t stream) {
  const int64_t heads = (int64_t)p.batch * p.h_kv;
  linear_decode_kernel<<<dim3((unsigned)(heads * (kD / kCols))), dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace mpfa
