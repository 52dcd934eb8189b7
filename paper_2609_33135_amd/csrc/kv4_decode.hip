// kv4_decode.hip -- split-KV attention of a few bf16 query rows per sequence over the
// 4-bit cache for gfx950, the merge of its partitions, and the accumulation of the
// attention weights.
//
// One wave takes one (sequence, KV head, 16 or 32 columns, partition of the visible tiles).
// A column is a query row: (token, query head of the KV head).  Keys are centered by their
// sequence's mean when they are written; the term q . mean is the same for every key of a
// row, so the softmax does not see it and bf16 queries need no compensation.
//
//   S^T = K Q^T      16x16x32 FP16 MFMA, K dequantized exactly (6 bits), Q exact (q_shift)
//   P = 2^(S - m)    FP32 statistics, P rounded to FP16 (at most 2^-11 of each P, an
//                    eighth of the bf16 output's own 2^-8; FP8 would be 2^-4)
//   O^T += V^T P^T   16x16x32 FP16 MFMA
//
// K and V go from memory to registers, 16 bytes per lane and load, no LDS, a page of 64 keys
// per step, whose address is in scalar registers.  MFMA row r of key block mb is key
// 16 (r/4) + 4 mb + r%4, so lane group g (lanes 16g .. +15) ends up with the scores of keys
// 16g .. 16g+15 of its column, and these are the keys it supplies to the PV product.  For V
// a lane holds the octet of channels 8 lr .. +7 of those keys: all its values share one
// scale group, and MFMA row lr of channel block db is channel 8 lr + db.
//
// What bounds it: HBM reads, 144 bytes per (token, KV head).
#include "kv4_device.h"

#include <type_traits>

namespace mpfa {

namespace {

constexpr int kDecodeWaves = kKv4DecodeWaves;

__device__ __forceinline__ int partitions_of(const Kv4AttnParams& p, const Kv4Tiles& tiles) {
  return min((tiles.nt + p.partition_tiles - 1) / p.partition_tiles, p.max_partitions);
}

// The waves of a workgroup that have partitions of the same rows can join them in LDS.  They
// do where that
//  - leaves the output itself (the workgroup has all partitions of its rows), with no launch
//    to merge them: 64 contexts of four rows and 2048 keys, 40:8 heads, 43 us, 54 with it; 64
//    of 2100, 32:8, 32.3 and 38.7, with 40 columns (40:8, eight rows) 62 and 73; or
//  - a fourth of many states: one context of 64K keys, 40:8, 19.6 us, 21.1 not.  (In between
//    the waves that wait for the others cost more: 4 of 32K, 32:8, 35.4 us, 33.8 not.)
constexpr int kJoinPartitions = 64;
__host__ __device__ inline bool direct(const Kv4AttnParams& p, int chunks) {
  return kv4_direct(chunks, p.max_partitions, p.scores != nullptr);
}
__host__ __device__ inline bool joined(const Kv4AttnParams& p, int chunks) {
  return direct(p, chunks) || (chunks == 1 && !p.scores && p.max_partitions > kJoinPartitions);
}
// States per row
__device__ __forceinline__ int states_of(const Kv4AttnParams& p, const Kv4Tiles& tiles, int chunks) {
  const int parts = partitions_of(p, tiles);
  return joined(p, chunks) ? (parts + kDecodeWaves - 1) / kDecodeWaves : parts;
}

// Workgroups of a sequence of kvl keys for one KV head: partitions times column chunks,
// four waves each; one for the zeros of a sequence without keys where nothing follows.
__device__ __forceinline__ int groups_of(const Kv4AttnParams& p, int kvl, int chunks) {
  const int parts = partitions_of(p, kv4_tiles(kvl - p.q_tokens, kvl - 1, p.window, p.sinks));
  return max((parts * chunks + kDecodeWaves - 1) / kDecodeWaves, direct(p, chunks) ? 1 : 0);
}

// Sequence and workgroup of position `pos` in a grid whose first workgroups are the ones
// with work, sequence by sequence; false past them.  Spread over a grid by sequence, the
// empty workgroups of the shorter ones take places on the card, and others get two: 16
// contexts of 10K to 32K keys, 8:2 heads, 23.1 us so, 30.3 before; 32 of 16K to 64K, 32:8,
// 210 us, 222 before.
__device__ __forceinline__ bool find_group(const Kv4AttnParams& p, int pos, int chunks, int& b, int& group) {
  const int lane = threadIdx.x & 63;
  for (int base = 0; base < p.batch; base += 64) {
    const int mine = base + lane < p.batch ? groups_of(p, p.kv_len[base + lane], chunks) : 0;
    int incl = mine;
    for (int d = 1; d < 64; d <<= 1) {
      const int up = __shfl_up(incl, d);
      if (lane >= d) incl += up;
    }
    const uint64_t past = __ballot(incl > pos);
    if (past) {
      const int at = __ffsll((unsigned long long)past) - 1;
      b = base + at;
      group = pos - (__builtin_amdgcn_readlane(incl, at) - __builtin_amdgcn_readlane(mine, at));
      return true;
    }
    pos -= __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// PACKED: one grid dimension, see find_group; else sequences on z (a batch whose lengths
// would take long to scan; a single sequence, which needs none: 1 us less).
constexpr int kPackedBatch = 512;

// COLS: columns per wave, 16 or 32 (two MFMA column blocks that share the dequantized K and
// V).  In steps of one page three waves of 16 columns fit a SIMD, or two of 32; with tiles of
// two pages two of 16, and 32 spilled (one context of 64K keys, 40:8 heads, 20.8 us, 21.8 so;
// 16 contexts of 10K to 32K, 8:2 heads, 21.4 and 22.8).
template <int COLS, bool JOIN, bool WEIGHTS, bool PACKED>
__global__ __launch_bounds__(64 * kDecodeWaves, COLS == 16 ? 3 : 2) void kv4_decode_kernel(Kv4AttnParams p) {
  constexpr int kN = COLS / 16;
  const int lane = threadIdx.x & 63, g = lane >> 4, lr = lane & 15;
  const int grp = p.h_q / p.h_kv, cols = p.q_tokens * grp;
  const int chunks = (cols + COLS - 1) / COLS;
  int b = blockIdx.z, hk = blockIdx.y, group = blockIdx.x;
  if (PACKED) {
    hk = blockIdx.x % p.h_kv;
    if (!find_group(p, blockIdx.x / p.h_kv, chunks, b, group)) return;
  }
  // the waves that take the column chunks of one partition are neighbours: they read the
  // same tiles at about the same time
  const int item = __builtin_amdgcn_readfirstlane(group * kDecodeWaves + (threadIdx.x >> 6));
  const int part = item / chunks, chunk = item - part * chunks;
  const int kvl = p.kv_len[b];
  const Kv4Tiles tiles = kv4_tiles(kvl - p.q_tokens, kvl - 1, p.window, p.sinks);
  const int v0 = part * p.partition_tiles, v1 = part < p.max_partitions ? min(tiles.nt, v0 + p.partition_tiles) : 0;
  const bool idle = v0 >= v1;
  if (!JOIN && idle) return;

  const int32_t* pt = p.page_table + (int64_t)b * p.max_pages;
  const int npg = (kvl + 63) >> 6;
  // the pages of 32 visible tiles, one per lane, read back with v_readlane: the loop has
  // no page-table loads, whose results would drain the loads in flight
  int win = 0, win_base = 0;
  auto load_window = [&](int v) {
    win_base = v;
    const int x = v + (lane >> 1);
    win = pt[min(2 * tiles.tile(min(x, tiles.nt - 1)) + (lane & 1), npg - 1)];
  };
  int64_t c;   // (page, KV head) row of a step
  auto step_page = [&](int u) {   // step u: page u of the visible tiles
    if ((u >> 1) - win_base >= 32) load_window(u >> 1);
    c = kv4_row(__builtin_amdgcn_readlane(win, u - 2 * win_base), p.h_kv, hk);
  };

  // offsets of the lane's bytes in a page: the rest is scalar or constant
  const uint32_t krow = 16 * (lr >> 2) + (lr & 3);   // + 4 mb: key of MFMA row lr
  const uint32_t k_off = krow * 64 + 16 * g, ks_off = krow * 8 + 2 * g;
  const uint32_t v_off = g * 1024 + lr * 16, vs_off = (lr >> 1) * 64 + 16 * g;
  u32x4 kc[4];
  uint32_t ksc[4];
  auto load_k = [&]() {
    const uint8_t *codes = p.cache.k_codes + c * 4096, *scales = p.cache.k_scales + c * 512;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      ksc[i] = *reinterpret_cast<const uint16_t*>(scales + ks_off + 32 * i);
      kc[i] = *reinterpret_cast<const u32x4*>(codes + k_off + 256 * i);
    }
  };
  u32x4 vc[4], vsc;
  auto load_v = [&]() {
    const uint8_t *codes = p.cache.v_codes + c * 4096, *scales = p.cache.v_scales + c * 512;
#pragma unroll
    for (int i = 0; i < 4; ++i) vc[i] = *reinterpret_cast<const u32x4*>(codes + v_off + 256 * i);
    vsc = *reinterpret_cast<const u32x4*>(scales + vs_off);
  };

  // the last tile's second page is left out where the sequence ends before it
  const int u0 = 2 * v0, u1 = 2 * v1 - (tiles.tile(v1 - 1) * kTile + kPage >= kvl ? 1 : 0);
  if (!idle) {
    load_window(v0);
    step_page(u0);
    load_k();
  }

  // ---- Q: channels 32g .. +31 of the lane's columns, and what they see
  f16x8 qop[kN][4];
  float lam[kN], m[kN], l[kN];   // m in accumulator units (times lam: log2)
  int pos[kN];                   // last visible key; negative: none
  f32x4 o[kN][8];
  auto col_of = [&](int n) { return chunk * COLS + 16 * n + lr; };
  const float tk = p.k_tscale[b * p.h_kv + hk];
#pragma unroll
  for (int n = 0; n < kN; ++n) {
    const int col = min(col_of(n), cols - 1), tok = col / grp;
    pos[n] = kvl - p.q_tokens + tok;
    const u32x4* src = reinterpret_cast<const u32x4*>(p.q + ((int64_t)b * p.q_tokens + tok) * p.q_stride +
                                                      (hk * grp + col - tok * grp) * kD + 32 * g);
    u32x4 w[4];
    float a = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = src[i];
      a = fmaxf(a, q_amax(w[i]));
    }
    const int shift = q_shift(wave_max16(a), tk);
#pragma unroll
    for (int i = 0; i < 4; ++i) qop[n][i] = q_operand(w[i], shift);
    lam[n] = score_scale(p.lam, tk, shift);
    m[n] = -INFINITY;
    l[n] = 0.0f;
#pragma unroll
    for (int db = 0; db < 8; ++db) o[n][db] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }

  for (int u = u0; u < u1; ++u) {
    const int key0 = tiles.tile(u >> 1) * kTile + kPage * (u & 1);
    load_v();
    __builtin_amdgcn_sched_barrier(0);   // the waits for K below leave V in flight
    f32x4 s[kN][4];
#pragma unroll
    for (int mb = 0; mb < 4; ++mb) {
      const f16x2 sc = e4m3_pair_f16(ksc[mb]);
      const f16x8 k[4] = {dequant8h(kc[mb][0], sc[0]), dequant8h(kc[mb][1], sc[0]), dequant8h(kc[mb][2], sc[1]),
                          dequant8h(kc[mb][3], sc[1])};
#pragma unroll
      for (int n = 0; n < kN; ++n) {
        s[n][mb] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][mb] = mfma_f16(k[i], qop[n][i], s[n][mb]);
      }
    }
    step_page(min(u + 1, u1 - 1));
    load_k();                            // past the last step: it again
    const int k0 = key0 + 16 * g;
    f16x8 pb[kN][2];
#pragma unroll
    for (int n = 0; n < kN; ++n) {
      // ---- masked scores (which may come from stale bytes) by selection
      if (key0 + kPage - 1 > kvl - p.q_tokens || (p.window > 0 && key0 < kvl - p.window)) {   // uniform
        // keys below it are outside the window (unless they are sinks)
        const int low = p.window > 0 ? max(pos[n] - p.window + 1, 0) : 0;
#pragma unroll
        for (int mb = 0; mb < 4; ++mb)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = k0 + 4 * mb + i;
            const bool seen = key <= pos[n] && (key >= low || key < p.sinks);
            s[n][mb][i] = seen ? s[n][mb][i] : -INFINITY;
          }
      }
      if (WEIGHTS) {
        if (col_of(n) < cols) {
          float* dst = p.scores +
                       (((int64_t)b * p.h_kv + hk) * cols + col_of(n)) * ((int64_t)p.max_partitions * p.partition_tiles * kTile) +
                       (int64_t)u * kPage + 16 * g;
#pragma unroll
          for (int mb = 0; mb < 4; ++mb) *reinterpret_cast<f32x4*>(dst + 4 * mb) = s[n][mb] * lam[n];
        }
      }
      float mxa = -INFINITY, mxb = -INFINITY;
#pragma unroll
      for (int mb = 0; mb < 4; mb += 2) {
        mxa = fmaxf(fmaxf(mxa, s[n][mb][0]), s[n][mb][1]);
        mxa = fmaxf(fmaxf(mxa, s[n][mb][2]), s[n][mb][3]);
        mxb = fmaxf(fmaxf(mxb, s[n][mb + 1][0]), s[n][mb + 1][1]);
        mxb = fmaxf(fmaxf(mxb, s[n][mb + 1][2]), s[n][mb + 1][3]);
      }
      const float mnew = fmaxf(m[n], wave_max16(fmaxf(mxa, mxb)));
      const float muse = mnew == -INFINITY ? 0.0f : mnew;
      const float alpha = m[n] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m[n] - muse) * lam[n]);
      m[n] = mnew;
      float bias = __builtin_fmaf(-muse, lam[n], kLog2P);
      const bool far = __builtin_fabsf(bias) > kPlainBias;
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(far) != 0, 0)) {
        const float d = far ? muse : 0.0f;
#pragma unroll
        for (int mb = 0; mb < 4; ++mb) s[n][mb] -= d;
        bias = far ? kLog2P : bias;
      }
      float ps = 0.0f;
#pragma unroll
      for (int mb = 0; mb < 4; ++mb) {
        float e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][mb][i], lam[n], bias));
          pb[n][mb >> 1][4 * (mb & 1) + i] = (_Float16)e[i];
        }
        ps += (e[0] + e[1]) + (e[2] + e[3]);
      }
      l[n] = alpha * l[n] + ps;
      if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
        for (int db = 0; db < 8; ++db) o[n][db] *= alpha;
      }
    }
    // ---- V: keys past the end hold stale bytes, P = 0 there: their scales are cleared so
    // that 0 * NaN cannot occur
    if (key0 + kPage > kvl) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int keep = kvl - k0 - 4 * i;
        vsc[i] &= keep >= 4 ? 0xFFFFFFFFu : (keep <= 0 ? 0u : ((1u << (8 * keep)) - 1u));
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {        // keys 16g + 8t .. +7
      uint32_t ev[4], od[4];
      f16x2 sc[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t a = vc[2 * t + (i >> 1)][2 * (i & 1)], c = vc[2 * t + (i >> 1)][2 * (i & 1) + 1];
        ev[i] = keys_even(a, c);
        od[i] = keys_odd(a, c);
        const uint32_t w = vsc[2 * t + (i >> 1)];
        sc[i] = e4m3_pair_f16((i & 1) ? w >> 16 : w);
      }
      auto pv = [&](const uint32_t (&w)[4], auto sel, int db) {
        constexpr int S = decltype(sel)::value;
        const f16x2 x0 = fp4_pair_f16<S>(w[0], sc[0]), x1 = fp4_pair_f16<S>(w[1], sc[1]);
        const f16x2 x2 = fp4_pair_f16<S>(w[2], sc[2]), x3 = fp4_pair_f16<S>(w[3], sc[3]);
        const f16x8 x = {x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]};
#pragma unroll
        for (int n = 0; n < kN; ++n) o[n][db] = mfma_f16(x, pb[n][t], o[n][db]);
      };
      pv(ev, std::integral_constant<int, 0>{}, 0);
      pv(od, std::integral_constant<int, 0>{}, 1);
      pv(ev, std::integral_constant<int, 1>{}, 2);
      pv(od, std::integral_constant<int, 1>{}, 3);
      pv(ev, std::integral_constant<int, 2>{}, 4);
      pv(od, std::integral_constant<int, 2>{}, 5);
      pv(ev, std::integral_constant<int, 3>{}, 6);
      pv(od, std::integral_constant<int, 3>{}, 7);
    }
  }
  // where a column's state goes: to LDS, or to the workspace
  __shared__ float joint[JOIN ? kDecodeWaves : 1][JOIN ? COLS : 1][kKv4State];   // [wave][column of its chunk]
  const int64_t row0 = (int64_t)b * p.q_tokens * p.h_q + hk * grp;
  auto row_of = [&](int col) { return row0 + (int64_t)(col / grp) * p.h_q + col % grp; };
  auto state_of = [&](int col, int at) { return p.states + (row_of(col) * p.max_partitions + at) * kKv4State; };
  if (!idle) {
#pragma unroll
    for (int n = 0; n < kN; ++n) {
      // keep the products in full-wave control flow (the store below is under a branch)
#pragma unroll
      for (int db = 0; db < 8; ++db) asm volatile("" : "+v"(o[n][db]));
      const float lt = wave_sum16(l[n]);
      const int col = col_of(n);
      if (col < cols) {
        float* st = JOIN ? joint[threadIdx.x >> 6][16 * n + lr] : state_of(col, part);
        if (g == 0) *reinterpret_cast<float2*>(st) = make_float2(m[n] * lam[n], lt);
        // accumulator row 4g + i of block db is channel 8 (4g + i) + db
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int db = 0; db < 8; db += 2)
            *reinterpret_cast<float2*>(st + 2 + 32 * g + 8 * i + db) = make_float2(o[n][db][i], o[n][db + 1][i]);
      }
    }
  }
  if constexpr (JOIN) {
    __syncthreads();
    const int own = kDecodeWaves / chunks;   // partitions of the workgroup
    const int live = max(min(partitions_of(p, tiles) - group * own, own), 0);
    const float tv = p.v_tscale[b * p.h_kv + hk];
    for (int col = threadIdx.x >> 6; col < cols; col += kDecodeWaves) {
      const float(*st0)[COLS][kKv4State] = joint + col / COLS;   // of the workgroup's first partition
      const int at = col % COLS;
      float M = -INFINITY, L = 0.0f, o0 = 0.0f, o1 = 0.0f;
      for (int q = 0; q < live; ++q) M = fmaxf(M, st0[q * chunks][at][0]);
      if (M > -INFINITY)
        for (int q = 0; q < live; ++q) {
          const float* st = st0[q * chunks][at];
          const float2 ml = *reinterpret_cast<const float2*>(st), x = *reinterpret_cast<const float2*>(st + 2 + 2 * lane);
          const float f = __builtin_amdgcn_exp2f(ml.x - M);
          L = __builtin_fmaf(f, ml.y, L);
          o0 = __builtin_fmaf(f, x.x, o0);
          o1 = __builtin_fmaf(f, x.y, o1);
        }
      if (direct(p, chunks)) {
        kv4_store_row(p.out + row_of(col) * kD, L, o0, o1, tv);
      } else {
        float* st = state_of(col, group);
        if (lane == 0) *reinterpret_cast<float2*>(st) = make_float2(M, L);
        *reinterpret_cast<float2*>(st + 2 + 2 * lane) = make_float2(o0, o1);
      }
    }
  }
}

// ---- after the partitions: the rows' merge and, with weights, the keys' shares.  One launch
// for both: the shares' workgroups derive the merged maximum and sum of every row from the
// partitions themselves (a launch of their own after the merge took 4 us more).

// Rows (token, query head): a wave each, four to a workgroup, or a workgroup of four waves
// each where there are many states (a wave keeps eight in flight).
constexpr int kManyStates = 16;
constexpr int kWeightKeys = kKv4WeightKeys;
constexpr int kWeightRows = 64;     // whose maxima and sums are held at a time

template <int WAVES>
__device__ __forceinline__ void merge_rows(const Kv4AttnParams& p, int b, int block, const Kv4Tiles& tiles, int chunks) {
  const int rows = p.q_tokens * p.h_q;
  const int i = WAVES > 1 ? block : __builtin_amdgcn_readfirstlane(block * 4 + (threadIdx.x >> 6));
  if (i >= rows) return;
  const int64_t r = (int64_t)b * rows + i;
  kv4_merge_row<WAVES>(p.states + r * p.max_partitions * kKv4State, kKv4State, states_of(p, tiles, chunks),
                       p.v_tscale[b * p.h_kv + i % p.h_q / (p.h_q / p.h_kv)], p.out + r * kD);
}

// Adds every visible key's share of the attention, summed over the rows of its KV head in
// order, to the cache's weights.
__device__ __forceinline__ void add_weights(const Kv4AttnParams& p, int b, int hk, int block, const Kv4Tiles& tiles,
                                            int chunks) {
  __shared__ float2 stats[kWeightRows];   // a row's maximum, and 2^15 / its sum (0: it sees nothing)
  const int kvl = p.kv_len[b], grp = p.h_q / p.h_kv, cols = p.q_tokens * grp, np = states_of(p, tiles, chunks);
  const int64_t per_col = (int64_t)p.max_partitions * p.partition_tiles * kTile;
  if ((int64_t)block * kWeightKeys >= min((int64_t)tiles.nt * kTile, per_col)) return;
  const int vk = block * kWeightKeys + threadIdx.x * 4;
  const bool mine = vk < min((int64_t)tiles.nt * kTile, per_col);
  const int key = mine ? tiles.tile(vk / kTile) * kTile + (vk & (kTile - 1)) : kvl;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  f32x4 w = {0.f, 0.f, 0.f, 0.f};
  for (int c0 = 0; c0 < cols; c0 += kWeightRows) {
    const int n = min(cols - c0, kWeightRows);
    __syncthreads();
    for (int c = wave; c < n; c += 4) {
      const int tok = (c0 + c) / grp, h = hk * grp + (c0 + c) - tok * grp;
      const float* st = p.states + (((int64_t)b * p.q_tokens + tok) * p.h_q + h) * p.max_partitions * kKv4State;
      float M = -INFINITY, L = 0.0f;
      for (int q = lane; q < np; q += 64) M = fmaxf(M, st[(int64_t)q * kKv4State]);
      for (int off = 32; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor(M, off));
      if (M > -INFINITY)
        for (int q = lane; q < np; q += 64) {
          const float2 ml = *reinterpret_cast<const float2*>(st + (int64_t)q * kKv4State);
          L = __builtin_fmaf(__builtin_amdgcn_exp2f(ml.x - M), ml.y, L);
        }
      for (int off = 32; off >= 1; off >>= 1) L += __shfl_xor(L, off);
      if (lane == 0) stats[c] = make_float2(M, L > 0.0f ? __fdiv_rn(0x1p15f, L) : 0.0f);
    }
    __syncthreads();
    if (key < kvl) {
      const float* src = p.scores + (((int64_t)b * p.h_kv + hk) * cols + c0) * per_col + vk;
      for (int c = 0; c < n; ++c) {
        const float2 st = stats[c];
        if (!(st.y > 0.0f)) continue;
        const f32x4 s = *reinterpret_cast<const f32x4*>(src + c * per_col);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_fmaf(__builtin_amdgcn_exp2f(s[i] - st.x), st.y, w[i]);
      }
    }
  }
  if (key >= kvl) return;
  const int32_t pg = p.page_table[(int64_t)b * p.max_pages + (key >> 6)];
  float* dst = p.cache.weights + kv4_row(pg, p.h_kv, hk) * kPage + (key & (kPage - 1));
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (key + i < kvl) dst[i] += w[i];
}

// Grid x: the blocks of rows, then with weights those of keys per KV head; y: sequences.
template <int WAVES, bool WEIGHTS>
__global__ __launch_bounds__(256) void kv4_decode_finish_kernel(Kv4AttnParams p, int chunks) {
  const int b = blockIdx.y, kvl = p.kv_len[b];
  const int rows = p.q_tokens * p.h_q, blocks = WAVES > 1 ? rows : (rows + 3) / 4;
  const Kv4Tiles tiles = kv4_tiles(kvl - p.q_tokens, kvl - 1, p.window, p.sinks);
  const int x = blockIdx.x;
  if (!WEIGHTS || x < blocks) merge_rows<WAVES>(p, b, x, tiles, chunks);
  else add_weights(p, b, (x - blocks) % p.h_kv, (x - blocks) / p.h_kv, tiles, chunks);
}

template <int COLS, bool JOIN, bool WEIGHTS>
void launch_partitions(const Kv4AttnParams& p, int chunks, hipStream_t stream) {
  const int64_t groups = ((int64_t)p.max_partitions * chunks + kDecodeWaves - 1) / kDecodeWaves;
  const int64_t all = groups * p.h_kv * p.batch;
  if (p.batch > 1 && p.batch <= kPackedBatch && all * 64 * kDecodeWaves <= UINT32_MAX)
    kv4_decode_kernel<COLS, JOIN, WEIGHTS, true><<<dim3((unsigned)all), 64 * kDecodeWaves, 0, stream>>>(p);
  else
    kv4_decode_kernel<COLS, JOIN, WEIGHTS, false><<<dim3((unsigned)groups, p.h_kv, p.batch), 64 * kDecodeWaves, 0, stream>>>(p);
}

template <int COLS>
void launch_columns(const Kv4AttnParams& p, int chunks, hipStream_t stream) {
  if (p.scores) launch_partitions<COLS, false, true>(p, chunks, stream);
  else if (joined(p, chunks)) launch_partitions<COLS, true, false>(p, chunks, stream);
  else launch_partitions<COLS, false, false>(p, chunks, stream);
}

}  // namespace

hipError_t launch_kv4_decode(const Kv4AttnParams& p, hipStream_t stream) {
  const int cols = p.q_tokens * (p.h_q / p.h_kv);
  const bool wide = kv4_wide_columns(cols);
  const int chunks = wide ? (cols + 31) / 32 : 1;
  wide ? launch_columns<32>(p, chunks, stream) : launch_columns<16>(p, chunks, stream);
  if (direct(p, chunks)) return hipGetLastError();
  const int states = joined(p, chunks) ? (p.max_partitions + kDecodeWaves - 1) / kDecodeWaves : p.max_partitions;
  const bool many = states > kManyStates;
  const int64_t rows = (int64_t)p.q_tokens * p.h_q, keys = (int64_t)p.max_partitions * p.partition_tiles * kTile;
  const int64_t blocks = (many ? rows : (rows + 3) / 4) + (p.scores ? (keys + kWeightKeys - 1) / kWeightKeys * p.h_kv : 0);
  const dim3 grid((unsigned)blocks, p.batch);
  if (p.scores && many) kv4_decode_finish_kernel<4, true><<<grid, 256, 0, stream>>>(p, chunks);
  else if (p.scores) kv4_decode_finish_kernel<1, true><<<grid, 256, 0, stream>>>(p, chunks);
  else if (many) kv4_decode_finish_kernel<4, false><<<grid, 256, 0, stream>>>(p, chunks);
  else kv4_decode_finish_kernel<1, false><<<grid, 256, 0, stream>>>(p, chunks);
  return hipGetLastError();
}

}  // namespace mpfa
