// rms_norm.hip -- root-mean-square norm of rows for gfx950, with the residual's addition and E4M3 codes.
//
// r = bf16(x + residual), y = r w / sqrt(mean r^2 + eps).  Codes of a group of channels: with m the largest
// |r w| of the group the scale is m / (448 sqrt(..)), in which y / scale = 448 (r w) / m: the root cancels,
// r w is exact in FP32 (eight bits times eight), and its one correctly rounded quotient by m cannot lie on a
// border of E4M3 that the true one does not lie on (16 + 5 bits), so codes are exact.
//
// Bound by memory: a row is read once, into registers, and every output written once.  16384 rows of 5120 channels
// with a residual and a scale per 128 channels 116 us (590 MB, 5.1 TB/s, a large copy's rate); 161920 rows of 128
// channels to BF16 18.7 us where no input is left in the cache from calls before (83 MB, 4.4 TB/s) and 15.3 over three
// sets of inputs, most of which are; 32 rows of 4096 4.6 us, a launch and two trips to memory.
#include "linear_internal.h"
#include "mpfa_device.h"

namespace mpfa {

namespace {

__device__ __forceinline__ float bits_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bits_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 r = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, r);
}

// Sum or maximum over `lanes` (a power of two) neighbouring lanes.
__device__ __forceinline__ float lanes_sum(float x, int lanes) {
  for (int off = 1; off < lanes; off <<= 1) x += __shfl_xor(x, off);
  return x;
}
__device__ __forceinline__ float lanes_max(float x, int lanes) {
  for (int off = 1; off < lanes; off <<= 1) x = fmaxf(x, __shfl_xor(x, off));
  return x;
}

// Eight channels of a row.
struct Octet {
  float r[8];
};

__device__ __forceinline__ void octet_sum(const NormParams& p, int64_t row, int c, u32x4 x, Octet* o) {
  if (p.residual) {
    const u32x4 y = *reinterpret_cast<const u32x4*>(p.residual + row * p.width + 8 * c);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = pack_bf16(bits_lo(x[i]) + bits_lo(y[i]), bits_hi(x[i]) + bits_hi(y[i]));
    // read again layers of kernels later: streamed past the cache (16384 rows of 5120 channels 128 -> 125 us)
    __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(p.residual_out + row * p.width + 8 * c));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o->r[2 * i] = bits_lo(x[i]);
    o->r[2 * i + 1] = bits_hi(x[i]);
  }
}

__device__ __forceinline__ void octet_weigh(const NormParams& p, int c, Octet* o) {
  if (!p.weight) return;
  const u32x4 w = *reinterpret_cast<const u32x4*>(p.weight + 8 * c);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o->r[2 * i] *= bits_lo(w[i]);
    o->r[2 * i + 1] *= bits_hi(w[i]);
  }
}

__device__ __forceinline__ void octet_bf16(const NormParams& p, int64_t row, int c, const Octet& o, float rstd) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_bf16(o.r[2 * i] * rstd, o.r[2 * i + 1] * rstd);
  *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p.out) + row * p.width + 8 * c) = w;
}

__device__ __forceinline__ float octet_max(const Octet& o) {
  float m = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(o.r[e]));
  return m;
}

__device__ __forceinline__ void octet_codes(const NormParams& p, int64_t row, int c, const Octet& o, float m) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  float q[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = m > 0.0f ? __fdiv_rn(o.r[e] * 0.875f, m) * 512.0f : 0.0f;   // 448 = 0.875 * 512
  *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(p.out) + row * p.width + 8 * c) =
      (u32x2){fp8_sat_pair(fp8_sat_pair(0, q[0], q[1], false), q[2], q[3], true),
              fp8_sat_pair(fp8_sat_pair(0, q[4], q[5], false), q[6], q[7], true)};
}

// 1 for a group of zeros, unless a NaN in its row has made rstd one.
__device__ __forceinline__ float group_scale(float m, float rstd) { return m > 0.0f || rstd != rstd ? m * rstd / 448.0f : 1.0f; }

// Rows of up to 512 channels: kLanes lanes a row, an octet each, so that no row needs a barrier and no lane idles at
// the heads' 128 channels.
template <int kLanes>
__global__ __launch_bounds__(256) void norm_rows_kernel(NormParams p) {
  const int c = threadIdx.x % kLanes, groups = (p.width + p.group - 1) / p.group;
  const int64_t row = (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  const bool mine = row < p.rows && 8 * c < p.width;
  Octet o = {};
  if (mine) octet_sum(p, row, c, *reinterpret_cast<const u32x4*>(p.x + row * p.x_stride + 8 * c), &o);
  float sum = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) sum += o.r[e] * o.r[e];
  const float rstd = 1.0f / sqrtf(lanes_sum(sum, kLanes) / p.width + p.eps);
  if (mine) octet_weigh(p, c, &o);
  if (!p.scales) {
    if (mine) octet_bf16(p, row, c, o, rstd);
    return;
  }
  const float m = lanes_max(octet_max(o), min(kLanes, groups == 1 ? kLanes : p.group / 8));
  if (!mine) return;
  octet_codes(p, row, c, o, m);
  if (8 * c % p.group == 0) p.scales[row * groups + 8 * c / p.group] = group_scale(m, rstd);
}

// A workgroup per row: kVecs octets a thread, those of a wave side by side.  Sum and maximum meet in one barrier; a
// group's own maximum stays within a wave.
template <int kVecs>
__global__ __launch_bounds__(1024) void norm_row_kernel(NormParams p) {
  __shared__ float s_sum[16], s_max[16];
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6, octets = p.width / 8;
  const int groups = (p.width + p.group - 1) / p.group;
  Octet o[kVecs] = {};
  u32x4 x[kVecs];
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int c = tid + i * blockDim.x;
    if (c < octets) x[i] = *reinterpret_cast<const u32x4*>(p.x + row * p.x_stride + 8 * c);
  }
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int c = tid + i * blockDim.x;
    if (c < octets) octet_sum(p, row, c, x[i], &o[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += o[i].r[e] * o[i].r[e];
  }
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int c = tid + i * blockDim.x;
    if (c < octets) octet_weigh(p, c, &o[i]);
    m = fmaxf(m, octet_max(o[i]));
  }
  sum = lanes_sum(sum, 64);
  m = lanes_max(m, 64);
  if (lane == 0) {
    s_sum[wave] = sum;
    s_max[wave] = m;
  }
  __syncthreads();
  sum = m = 0.0f;
  for (int i = 0; i < waves; ++i) {
    sum += s_sum[i];
    m = fmaxf(m, s_max[i]);
  }
  const float rstd = 1.0f / sqrtf(sum / p.width + p.eps);
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int c = tid + i * blockDim.x;
    if (!p.scales) {
      if (c < octets) octet_bf16(p, row, c, o[i], rstd);
      continue;
    }
    const float top = groups == 1 ? m : lanes_max(octet_max(o[i]), p.group / 8);
    if (c >= octets) continue;
    octet_codes(p, row, c, o[i], top);
    if (8 * c % p.group == 0) p.scales[row * groups + 8 * c / p.group] = group_scale(top, rstd);
  }
}

template <int kLanes>
void launch_rows(const NormParams& p, hipStream_t stream) {
  constexpr int kEach = 256 / kLanes;
  norm_rows_kernel<kLanes><<<dim3((unsigned)(((int64_t)p.rows + kEach - 1) / kEach)), dim3(256), 0, stream>>>(p);
}

}  // namespace

hipError_t launch_rms_norm(const NormParams& p, hipStream_t stream) {
  if (p.width <= 64) {
    launch_rows<8>(p, stream);
  } else if (p.width <= 128) {
    launch_rows<16>(p, stream);
  } else if (p.width <= 256) {
    launch_rows<32>(p, stream);
  } else if (p.width <= 512) {
    launch_rows<64>(p, stream);
  } else {
    const dim3 grid(p.rows), threads(norm_threads(p.width));
    if (norm_octets(p.width) == 2) norm_row_kernel<2><<<grid, threads, 0, stream>>>(p);
    else norm_row_kernel<4><<<grid, threads, 0, stream>>>(p);
  }
  return hipGetLastError();
}

}  // namespace mpfa
