// kv4_internal.h -- launch parameter blocks and the visible-tile arithmetic shared
// by the host layer (kv4_api.cpp) and the kernels of the 4-bit cache (kv4_*.hip).
// Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mpfa.h"

namespace mpfa {

constexpr int kKv4StatTokens = 128;   // fewest tokens per statistics partial
// per partial of one KV head: FP64 sums, FP32 maxima and minima of K per channel, and
// the largest |V| (padded to 16 bytes)
constexpr int kKv4StatBytes = 128 * (8 + 4 + 4) + 16;
constexpr int kKv4WriteTokens = 32;   // tokens per workgroup of 256 threads of the write pass
constexpr int kKv4Rows = 256;         // most query rows (tokens x heads of one KV head) of a prefill item
constexpr int kKv4WeightKeys = 1024;  // keys of a KV head whose weights a workgroup adds, four per thread
constexpr int kKv4State = 130;        // floats of a partition state: m, l, O[128]

// Planes of the cache; page pg, KV head h, slot o.
struct Kv4Cache {
  uint8_t* k_codes;   // [P][H][64][64]: token rows, channel 2i in the low nibble of byte i
  uint8_t* k_scales;  // [P][H][64][8]
  uint8_t* v_codes;   // [P][H][16][16][4][4]: quad o / 4, octet of channels c / 8, o % 4, the octet's 4 bytes
  uint8_t* v_scales;  // [P][H][8][64]: group c / 16, slot
  float* weights;     // [P][H][64] or null
};

struct Kv4WriteParams {
  int batch, total_tokens, max_seqlen, h_kv;
  int smooth, compute_stats;
  int stat_tokens;                    // tokens per statistics partial, a multiple of kKv4StatTokens
  int64_t num_pages, k_stride, v_stride;
  const int32_t* cu_seqlens;
  const uint16_t* k;
  const uint16_t* v;
  const int64_t* slot_mapping;
  uint16_t* k_mean;
  float* k_tscale;
  float* v_tscale;
  Kv4Cache cache;
  uint16_t* k_out;
  uint16_t* v_out;
  uint8_t* ws;
};

struct Kv4AttnParams {
  int batch, h_q, h_kv, max_pages;
  int q_tokens;                          // decode: rows per sequence
  int max_seqlen_q;                      // prefill
  int partition_tiles, max_partitions;   // decode
  int n_items, n_merges, half;           // prefill by a plan: its items (half: of 128 rows)
  int window, sinks;
  float lam;                             // log2(e) / sqrt(128)
  int64_t q_stride;
  const int32_t* cu_seqlens_q;           // prefill
  const int32_t* q_start;                // prefill
  const int32_t* kv_len;
  const int32_t* page_table;
  const uint16_t* q;
  Kv4Cache cache;
  const float* k_tscale;
  const float* v_tscale;
  uint16_t* out;
  const mpfa_kv4_item* items;            // prefill: the plan, or null
  float* states;                         // decode [row][h_q][max_partitions][130], prefill [state][h_kv][rows][130]
  float* scores;                         // weights: [b][h_kv][q_tokens * G][max_partitions * partition tokens]
};

struct Kv4EvictParams {
  int batch, h_kv, max_pages, dst_max_pages;
  int budget, sinks, recent, in_place;
  const int32_t* kv_len;
  const int32_t* page_table;
  const int32_t* dst_page_table;
  Kv4Cache cache;
  int32_t* kept;                         // [b][h_kv][budget]
  int32_t* new_len;                      // [b]
};

// The 128-key tiles that rows at positions first .. last (first may be negative: such
// rows see nothing) look at: tiles 0 .. ns - 1 (first tokens that stay visible), then
// tiles jl .. (the window and the rows themselves); nt in all.  Visible tile v is tile v
// below ns and jl + v - ns from there.
struct Kv4Tiles {
  int ns, jl, nt;
  __host__ __device__ int tile(int v) const { return v < ns ? v : jl + v - ns; }
};

__host__ __device__ inline Kv4Tiles kv4_tiles(int first, int last, int window, int sinks) {
  Kv4Tiles t = {0, 0, 0};
  if (last < 0) return t;
  const int f = first > 0 ? first : 0;
  t.jl = window > 0 && f >= window ? (f - window + 1) >> 7 : 0;
  const int ends = sinks < last + 1 ? sinks : last + 1;   // keys below it are sinks
  const int st = (ends + 127) >> 7;
  t.ns = st < t.jl ? st : t.jl;
  t.nt = t.ns + (last >> 7) - t.jl + 1;
  return t;
}

// Whether decode waves take 32 columns (rows times heads of a KV head) each, or 16.
__host__ __device__ inline bool kv4_wide_columns(int64_t cols) { return cols > 16; }

// Whether the four waves of a decode workgroup have all partitions of their rows (in `chunks`
// parts of 16 or 32 columns), and write the output themselves.
constexpr int kKv4DecodeWaves = 4;
__host__ __device__ inline bool kv4_direct(int64_t chunks, int64_t max_partitions, bool weights) {
  return kKv4DecodeWaves % chunks == 0 && max_partitions <= kKv4DecodeWaves / chunks && !weights;
}

hipError_t launch_kv4_write(const Kv4WriteParams& p, hipStream_t stream);
hipError_t launch_kv4_prefill(const Kv4AttnParams& p, hipStream_t stream);
hipError_t launch_kv4_decode(const Kv4AttnParams& p, hipStream_t stream);
hipError_t launch_kv4_evict(const Kv4EvictParams& p, hipStream_t stream);

}  // namespace mpfa
