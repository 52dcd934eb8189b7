// linear_decode.hip -- linear attention with a decay, one or a few new tokens per sequence, for gfx950.
//
// S_t = a_t S_{t-1} + k_t v_t^T, o_t = scale q_t^T S_t in FP32.  Bound by the state's 64 KB per KV head, read
// and written once: the rows of a call are taken one after the other with the state in registers.
#include "linear_internal.h"
#include "mpfa_device.h"

namespace mpfa {

namespace {

constexpr int kHeads = 8;   // query heads whose sums are joined together

// One workgroup of 256 threads per (sequence, KV head, kCols columns of the state): kCols / 4 lanes side by
// side on a row, 1024 / kCols rows at a time.
template <int kCols>
__global__ __launch_bounds__(256) void linear_decode_kernel(LinearParams p) {
  constexpr int kLanes = kCols / 4, kRows = 256 / kLanes, kEach = kD / kRows, kParts = kD / kCols;
  __shared__ float s_k[kD], s_q[kHeads][kD];
  __shared__ f32x4 s_sum[4][kHeads][kLanes];
  const int part = blockIdx.x % kParts, hk = blockIdx.x / kParts % p.h_kv, b = blockIdx.x / kParts / p.h_kv;
  const int tid = threadIdx.x, c = tid % kLanes, row = tid / kLanes, lane = tid & 63, wave = tid >> 6;
  const int grp = p.h_q / p.h_kv, col = part * kCols + 4 * c;
  const int src = p.state_src[b], dst = p.state_dst[b];
  f32x4 st[kEach];
  if (src >= 0) {
    const float* from = p.states + ((int64_t)src * p.h_kv + hk) * kLinState + col;
#pragma unroll
    for (int i = 0; i < kEach; ++i) st[i] = *reinterpret_cast<const f32x4*>(from + (row + kRows * i) * kD);
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i) st[i] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
  }
  for (int r = 0; r < p.q_tokens; ++r) {
    const int64_t t = (int64_t)b * p.q_tokens + r;
    const float g = fminf(fmaxf(p.log_decay[t * p.decay_stride + hk], kLinLeastDecay), 0.0f), a = expf(g);
    const uint32_t* vw = reinterpret_cast<const uint32_t*>(p.v + t * p.v_stride + hk * kD + col);
    const f32x4 v = {__uint_as_float(vw[0] << 16), __uint_as_float(vw[0] & 0xFFFF0000u), __uint_as_float(vw[1] << 16),
                     __uint_as_float(vw[1] & 0xFFFF0000u)};
    for (int h0 = 0; h0 < grp; h0 += kHeads) {
      const int heads = min(kHeads, grp - h0);
      __syncthreads();
      if (h0 == 0 && tid < kD) s_k[tid] = bf16_to_f32(p.k[t * p.k_stride + hk * kD + tid]);
      for (int i = tid; i < heads * kD; i += 256) s_q[i / kD][i % kD] = bf16_to_f32(p.q[t * p.q_stride + (hk * grp + h0) * kD + i]);
      __syncthreads();
      if (h0 == 0)
#pragma unroll
        for (int i = 0; i < kEach; ++i) st[i] = st[i] * a + v * s_k[row + kRows * i];
      for (int h = 0; h < heads; ++h) {
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < kEach; ++i) o += st[i] * s_q[h][row + kRows * i];
#pragma unroll
        for (int off = kLanes; off < 64; off <<= 1)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], off);
        if (lane < kLanes) s_sum[wave][h][lane] = o;
      }
      __syncthreads();
      for (int i = tid; i < heads * kLanes; i += 256) {
        const int h = i / kLanes, x = i % kLanes;
        const f32x4 o = ((s_sum[0][h][x] + s_sum[1][h][x]) + (s_sum[2][h][x] + s_sum[3][h][x])) * p.scale;
        uint16_t* to = p.out + (t * p.h_q + hk * grp + h0 + h) * kD + part * kCols + 4 * x;
#pragma unroll
        for (int e = 0; e < 4; ++e) to[e] = bf16_rne(o[e]);
      }
    }
  }
  if (dst >= 0) {
    float* to = p.states + ((int64_t)dst * p.h_kv + hk) * kLinState + col;
#pragma unroll
    for (int i = 0; i < kEach; ++i) *reinterpret_cast<f32x4*>(to + (row + kRows * i) * kD) = st[i];
  }
}

}  // namespace

hipError_t launch_linear_decode(const LinearParams& p, hipStream_t stream) {
  const int64_t heads = (int64_t)p.batch * p.h_kv;
  linear_decode_kernel<32><<<dim3((unsigned)(heads * 4)), dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace mpfa
