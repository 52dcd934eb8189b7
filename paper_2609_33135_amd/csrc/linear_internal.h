// linear_internal.h -- launch parameter blocks of linear attention (linear_*.hip) and of the norm
// (rms_norm.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "linear_cut.h"

namespace mpfa {

constexpr int kLinJoin = 4;                    // places that a wave of `join` has at once
constexpr int kLinJoinWaves = 16;              // at most
constexpr float kLinLeastDecay = -200.0f;      // exp of it times any FP32 number is 0

struct LinearParams {
  int batch, h_q, h_kv;
  int q_tokens;                  // decode: rows per sequence
  int segment;                   // prefill: tokens per segment, a multiple of kLinChunk
  int split;                     // prefill: some sequence may have several segments
  int parts, heads;              // prefill: parts of a KV head's query heads, of so many each
  int items;                     // prefill: workgroups, a segment and KV head each
  int join_waves;                // prefill: waves of a workgroup that joins states
  float scale;
  int64_t q_stride, k_stride, v_stride, decay_stride;
  const int32_t* cu_seqlens;     // prefill
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const float* log_decay;
  const int32_t* state_src;
  const int32_t* state_dst;
  float* states;                 // [slot][h_kv][128][128]
  uint16_t* out;
  float* starts;                 // prefill: [segment id][h_kv][kLinState], see linear_prefill.hip
  float* decays;                 // prefill: [segment id][h_kv]
};

struct NormParams {
  int rows, width, group;        // group: channels per scale, width for one per row
  float eps;
  int64_t x_stride;
  const uint16_t* x;
  const uint16_t* weight;        // or null
  const uint16_t* residual;      // or null
  uint16_t* residual_out;
  void* out;                     // bf16, or E4M3 where scales are given
  float* scales;                 // or null
};

// Threads for a row: for more than 512 channels a workgroup, of norm_octets(width) octets a thread.
constexpr int kNormWidth = 32768;
inline int norm_octets(int width) { return width <= 16384 ? 2 : 4; }
inline int norm_threads(int width) {
  if (width <= 512) return width <= 64 ? 8 : width <= 128 ? 16 : width <= 256 ? 32 : 64;
  const int wave = 64 * 8 * norm_octets(width);
  return (width + wave - 1) / wave * 64;
}

hipError_t launch_linear_prefill(const LinearParams& p, hipStream_t stream);
hipError_t launch_linear_decode(const LinearParams& p, hipStream_t stream);
hipError_t launch_rms_norm(const NormParams& p, hipStream_t stream);
// whether any log decay [tokens][heads] is NaN or above 0 (debug library)
hipError_t launch_scan_decay(const float* x, int64_t tokens, int heads, int64_t stride, int* flag, hipStream_t stream);

}  // namespace mpfa
