// kv4_prefill.hip -- causal attention of many bf16 query rows over the 4-bit cache for
// gfx950, with a sliding window and first tokens that stay visible.
//
// One workgroup of eight waves takes 256 rows of one KV head: TM = 256 / G tokens times
// the G query heads that share it, 32 rows per wave, one per lane pair.  Packing the heads
// of a KV head makes the item short in tokens: fewer keys outside the diagonal and the
// window, more items for short prompts, and one dequantization of K and V for all of them.
// A plan (made on the host, where the lengths are known) orders the items by length, cuts
// some of them along the keys, whose parts are merged, and may halve the items: of 128
// rows, the waves of either half of the workgroup take the same rows and half of every
// tile's keys, and join at the end.
//
// Per 128-key tile K and V are loaded as codes a tile ahead, dequantized exactly to FP16
// (6 bits) on their way into LDS, and multiplied on the 32x32x16 FP16 MFMA:
//   S^T = K Q^T, online softmax in FP32, P rounded to FP16 (see kv4_decode.hip),
//   O^T += V^T P^T.
// The step is software pipelined as the 8-bit prefill's: the QK products of the next tile
// take the score registers block by block as the exponentials of this one free them.
//
// What bounds it: the matrix pipe (512 flop per visible pair) and the vector work of the
// softmax and the dequantization, which overlap in part: for 8192 tokens, 32:8 heads, the pipe is
// busy 46 % of the cycles, 44 % of these with vector instructions beside it, which issue in about
// as many cycles themselves.
#include "kv4_device.h"

namespace mpfa {

namespace {

constexpr int kStride = 256 + 16;   // bytes of an LDS row: 128 FP16 values, padded so that operand reads spread over the banks

struct Kv4Smem {
  // K rows in MFMA order: key 32 kb + kappa of the tile is row 32 kb + k_row(kappa), so that
  // accumulator register r of lane half hf is key 16 (r/8) + 8 hf + r%8 of its block
  uint8_t k[2][kTile * kStride];
  // V rows [channel][key], channel c in row 16 (c%8) + c/8: lanes that hold the octets of
  // one quad of keys store to 16 consecutive rows, on distinct banks
  uint8_t v[2][kD * kStride];
};

__device__ __forceinline__ int k_row(int kappa) {
  return 8 * (2 * (kappa >> 4) + ((kappa >> 2) & 1)) + 4 * ((kappa >> 3) & 1) + (kappa & 3);
}

// One thread's share of a tile: 16 bytes of K codes (32 channels of a key) and of V codes
// (an octet of channels of four keys) and their scales.
struct Kv4Regs {
  u32x4 k, v;
  uint32_t ks, vs;
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t plane_rsrc(const void* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, 0x00027000);
}

// u: unit of the page (0 .. 255)
__device__ __forceinline__ void fetch_k(Kv4Regs& r, const Kv4AttnParams& p, int pg, int hk, uint32_t u) {
  const int64_t row = kv4_row(pg, p.h_kv, hk);
  r.k = __builtin_amdgcn_raw_buffer_load_b128(plane_rsrc(p.cache.k_codes + row * 4096, 4096), u * 16u, 0, 0);
  r.ks = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(plane_rsrc(p.cache.k_scales + row * 512, 512), u * 2u, 0, 0);
}
__device__ __forceinline__ void fetch_v(Kv4Regs& r, const Kv4AttnParams& p, int pg, int hk, uint32_t u) {
  const int64_t row = kv4_row(pg, p.h_kv, hk);
  r.v = __builtin_amdgcn_raw_buffer_load_b128(plane_rsrc(p.cache.v_codes + row * 4096, 4096), u * 16u, 0, 0);
  // octet u % 16 (group u % 16 / 2), tokens 4 (u / 16) .. +3
  r.vs = __builtin_amdgcn_raw_buffer_load_b32(plane_rsrc(p.cache.v_scales + row * 512, 512), ((u & 15u) >> 1) * 64u + (u >> 4) * 4u, 0, 0);
}
__device__ __forceinline__ void store_k(Kv4Smem& sm, int buf, const Kv4Regs& r, int half, int u) {
  const int key = 64 * half + (u >> 2), qt = u & 3;
  uint8_t* dst = sm.k[buf] + ((key & ~31) + k_row(key & 31)) * kStride + qt * 64;
  const f16x2 s = e4m3_pair_f16(r.ks);
#pragma unroll
  for (int w = 0; w < 4; ++w) *reinterpret_cast<f16x8*>(dst + 16 * w) = dequant8h(r.k[w], s[w >> 1]);
}
// nvalid: keys of the tile before kv_len; past them the scales are cleared (stale bytes
// may be NaN, and 0 * NaN must not occur)
__device__ __forceinline__ void store_v(Kv4Smem& sm, int buf, const Kv4Regs& r, int half, int u, int nvalid) {
  const int key = 64 * half + 4 * (u >> 4), oct = u & 15;
  uint32_t vs = r.vs;
  if (nvalid < kTile) {
    const int keep = nvalid - key;
    vs &= keep >= 4 ? 0xFFFFFFFFu : (keep <= 0 ? 0u : ((1u << (8 * keep)) - 1u));
  }
  const f16x2 s0 = e4m3_pair_f16(vs), s1 = e4m3_pair_f16(vs >> 16);
  const uint32_t e0 = keys_even(r.v[0], r.v[1]), e1 = keys_even(r.v[2], r.v[3]);
  const uint32_t o0 = keys_odd(r.v[0], r.v[1]), o1 = keys_odd(r.v[2], r.v[3]);
  uint8_t* dst = sm.v[buf] + oct * kStride + key * 2;
  typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
  auto put = [&](int c, f16x2 a, f16x2 b) { *reinterpret_cast<f16x4*>(dst + 16 * c * kStride) = (f16x4){a[0], a[1], b[0], b[1]}; };
  put(0, fp4_pair_f16<0>(e0, s0), fp4_pair_f16<0>(e1, s1));
  put(1, fp4_pair_f16<0>(o0, s0), fp4_pair_f16<0>(o1, s1));
  put(2, fp4_pair_f16<1>(e0, s0), fp4_pair_f16<1>(e1, s1));
  put(3, fp4_pair_f16<1>(o0, s0), fp4_pair_f16<1>(o1, s1));
  put(4, fp4_pair_f16<2>(e0, s0), fp4_pair_f16<2>(e1, s1));
  put(5, fp4_pair_f16<2>(o0, s0), fp4_pair_f16<2>(o1, s1));
  put(6, fp4_pair_f16<3>(e0, s0), fp4_pair_f16<3>(e1, s1));
  put(7, fp4_pair_f16<3>(o0, s0), fp4_pair_f16<3>(o1, s1));
}

// What a wave keeps of its item.
struct Kv4Item {
  int lane, hf, lc;
  int pos, low, sinks;      // the lane's row sees keys <= pos that are >= low or < sinks
  int wpos_min, wlow_max;   // smallest pos and largest low of the wave's rows
  int kb0;                  // first of the wave's 32-key blocks in a tile
  float lam;
  f16x8 q[8];               // channels 16 ks + 8 hf .. +7
};

// 32-key blocks of a tile per wave
template <bool HALF>
constexpr int kBlocks = HALF ? 2 : 4;

__device__ __forceinline__ void qk_block(f32x16& s, int kb, const Kv4Smem& sm, int buf, const Kv4Item& it) {
  const uint8_t* kp = sm.k[buf] + (32 * (it.kb0 + kb) + it.lc) * kStride + 16 * it.hf;
  s = (f32x16){};
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) s = mfma32_f16(*reinterpret_cast<const f16x8*>(kp + 32 * ks), it.q[ks], s);
}

template <int NB>
__device__ __forceinline__ void mask_tile(f32x16 (&s)[NB], int key0, const Kv4Item& it) {
  const int k0 = key0 + 32 * it.kb0 + 8 * it.hf;
#pragma unroll
  for (int kb = 0; kb < NB; ++kb) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = k0 + 32 * kb + 16 * (q >> 1) + 4 * (q & 1) + i;
        const bool seen = key <= it.pos && (key >= it.low || key < it.sinks);
        s[kb][4 * q + i] = seen ? s[kb][4 * q + i] : -INFINITY;
      }
      __builtin_amdgcn_sched_barrier(0);   // compare next to select: 64 masks at once exhaust the scalar registers
    }
  }
}

struct Kv4Soft {
  float m, l, bias;   // running maximum (accumulator units), row sum, exponent bias
};

// Running maximum and bias of the tile's exponentials (s: the scores, or their distance from the
// maximum where that is needed, see kPlainBias); returns the factor of what was summed before.
template <int NB>
__device__ __forceinline__ float max_tile(f32x16 (&s)[NB], const Kv4Item& it, Kv4Soft& ss) {
  float mxa = -INFINITY, mxb = -INFINITY;
#pragma unroll
  for (int kb = 0; kb < NB; kb += 2) {
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      mxa = fmaxf(fmaxf(mxa, s[kb][r]), s[kb][r + 1]);
      mxb = fmaxf(fmaxf(mxb, s[kb + 1][r]), s[kb + 1][r + 1]);
    }
  }
  const float mnew = fmaxf(ss.m, wave_max32(fmaxf(mxa, mxb)));
  const float muse = mnew == -INFINITY ? 0.0f : mnew;
  const float alpha = ss.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((ss.m - muse) * it.lam);
  ss.m = mnew;
  ss.bias = __builtin_fmaf(-muse, it.lam, kLog2P);
  const bool far = __builtin_fabsf(ss.bias) > kPlainBias;
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(far) != 0, 0)) {
    const float d = far ? muse : 0.0f;
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) s[kb] -= d;
    ss.bias = far ? kLog2P : ss.bias;
  }
  return alpha;
}

// P of one 32-key block: ph[2 kb + t] are keys 32 (kb0 + kb) + 16 t + 8 hf .. +7
template <int NP>
__device__ __forceinline__ float exp_block(const f32x16& s, int kb, const Kv4Item& it, const Kv4Soft& ss, f16x8 (&ph)[NP]) {
  float ps = 0.0f;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    float e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * t + i], it.lam, ss.bias));
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f16x2 x = {(_Float16)e[2 * i], (_Float16)e[2 * i + 1]};
      w[i] = __builtin_bit_cast(uint32_t, x);
    }
    ps += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
    // keeps the exponentials here: the compiler would sink them to the PV product
    asm volatile("" : "+v"(w), "+v"(ps));
    ph[2 * kb + t] = __builtin_bit_cast(f16x8, w);
  }
  return ps;
}

__device__ __forceinline__ void rescale(f32x16 (&o)[4], float alpha) {
  if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
    for (int db = 0; db < 4; ++db) o[db] *= alpha;
  }
}

template <int NP>
__device__ __forceinline__ void pv_tile(const Kv4Smem& sm, int buf, const f16x8 (&ph)[NP], f32x16 (&o)[4], const Kv4Item& it) {
  const uint8_t* vp = sm.v[buf] + it.lc * kStride + 16 * it.hf + 64 * it.kb0;
#pragma unroll
  for (int t = 0; t < NP; ++t)
#pragma unroll
    for (int db = 0; db < 4; ++db)
      o[db] = mfma32_f16(*reinterpret_cast<const f16x8*>(vp + 32 * db * kStride + 32 * t), ph[t], o[db]);
}

// Joins the halves of an item of 128 rows: the waves of the second half leave their states
// in LDS, those of the first add them to their own.
__device__ __forceinline__ bool join_halves(Kv4Smem& sm, int wave, const Kv4Item& it, Kv4Soft& ss, f32x16 (&o)[4]) {
  static_assert(4 * 66 * 64 * sizeof(float) <= sizeof(Kv4Smem), "states of four waves");
  float* st = reinterpret_cast<float*>(&sm) + (wave & 3) * 66 * 64 + it.lane;
  __syncthreads();   // the tiles are read
  if (wave >= 4) {
    st[0] = ss.m;
    st[64] = ss.l;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) st[64 * (2 + 16 * db + r)] = o[db][r];
  }
  __syncthreads();
  if (wave >= 4) return false;
  const float m1 = st[0], l1 = st[64], M = fmaxf(ss.m, m1), use = M == -INFINITY ? 0.0f : M;
  const float f0 = __builtin_amdgcn_exp2f((ss.m - use) * it.lam), f1 = __builtin_amdgcn_exp2f((m1 - use) * it.lam);
  ss.m = M;
  ss.l = f0 * ss.l + f1 * l1;
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[db][r] = f0 * o[db][r] + f1 * st[64 * (2 + 16 * db + r)];
  return true;
}

// Tokens tok0 .. of sequence b, KV head hk, visible tiles v0 .. v1 - 1 of the item; state:
// where the item's parts leave their states for the merge, or null: the output.
template <bool HALF>
__device__ __forceinline__ void prefill_item(const Kv4AttnParams& p, Kv4Smem& sm, int b, int hk, int tok0, int tm, int nq, int q0,
                                             const Kv4Tiles& tiles, int v0, int v1, float* state) {
  constexpr int kNb = kBlocks<HALF>;
  const int grp = p.h_q / p.h_kv;
  Kv4Item it;
  it.lane = threadIdx.x & 63;
  it.hf = it.lane >> 5;
  it.lc = it.lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wrow = 32 * (HALF ? wave & 3 : wave);    // the wave's first row
  it.kb0 = HALF ? 2 * (wave >> 2) : 0;
  const int last = min(tok0 + tm, nq) - 1;           // last token of the item
  const int qs = p.q_start[b], kvl = p.kv_len[b];
  const int row = wrow + it.lc;
  const int tok = min(tok0 + row / grp, last);       // rows past the item repeat its last token
  const bool active = wrow < (last + 1 - tok0) * grp;
  it.pos = qs + tok;
  it.low = p.window > 0 ? max(it.pos - p.window + 1, 0) : 0;
  it.sinks = p.sinks;
  it.wpos_min = qs + min(tok0 + wrow / grp, last);
  it.wlow_max = p.window > 0 ? max(qs + min(tok0 + (wrow + 31) / grp, last) - p.window + 1, 0) : 0;
  {
    const u32x4* src = reinterpret_cast<const u32x4*>(p.q + (int64_t)(q0 + tok) * p.q_stride + (hk * grp + row % grp) * kD);
    u32x4 w[8];
    float a = 0.0f;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      w[ks] = src[2 * ks + it.hf];
      a = fmaxf(a, q_amax(w[ks]));
    }
    const float tk = p.k_tscale[b * p.h_kv + hk];
    const int shift = q_shift(wave_max32(a), tk);
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) it.q[ks] = q_operand(w[ks], shift);
    it.lam = score_scale(p.lam, tk, shift);
  }

  Kv4Soft ss = {-INFINITY, 0.0f, 0.0f};
  f32x16 o[4];
#pragma unroll
  for (int db = 0; db < 4; ++db) o[db] = (f32x16){};

  const int32_t* pt = p.page_table + (int64_t)b * p.max_pages;
  const int npg = (kvl + 63) >> 6;
  const int half = wave >> 2, u = threadIdx.x & 255;
  auto page = [&](int v) { return pt[min(2 * tiles.tile(max(v, 0)) + half, npg - 1)]; };
  Kv4Regs kr;
  int pgk, pgv, pgn;
  auto next_pages = [&](int v) {
    pgv = pgk;
    pgk = __builtin_amdgcn_readfirstlane(pgn);
    pgn = page(v);
  };
  // step v (last to first): K of tile v - 1 and V of tile v are read; K of v - 2 and V of
  // v - 1 are stored over buffers that the next step reads
  const int vh = v1 - 1;
  auto put_v = [&](int v) { store_v(sm, v & 1, kr, half, u, kvl - tiles.tile(v) * kTile); };
  pgk = __builtin_amdgcn_readfirstlane(page(vh));
  pgn = page(vh - 1);
  fetch_k(kr, p, pgk, hk, u);
  fetch_v(kr, p, pgk, hk, u);
  store_k(sm, vh & 1, kr, half, u);
  next_pages(vh - 2);
  if (vh > v0) fetch_k(kr, p, pgk, hk, u);
  put_v(vh);
  if (vh > v0) store_k(sm, (vh - 1) & 1, kr, half, u);
  __syncthreads();
  if (!active) {   // a wave without rows moves its share of the tiles
    if (vh > v0) __syncthreads();
    for (int v = vh; v > v0; --v) {
      next_pages(v - 3);
      fetch_k(kr, p, pgk, hk, u);
      fetch_v(kr, p, pgv, hk, u);
      store_k(sm, v & 1, kr, half, u);
      put_v(v - 1);
      __syncthreads();
    }
    if (HALF) {   // the barriers of join_halves
      __syncthreads();
      __syncthreads();
    }
    return;
  }

  f32x16 s[kNb];
  f16x8 ph[2 * kNb];
#pragma unroll
  for (int kb = 0; kb < kNb; ++kb) qk_block(s[kb], kb, sm, vh & 1, it);
  if (vh > v0) __syncthreads();
  auto mask = [&](int v) {
    const int key0 = tiles.tile(v) * kTile;
    if (key0 + kTile - 1 > it.wpos_min || key0 < it.wlow_max) mask_tile(s, key0, it);
  };
  mask(vh);
  float alpha = max_tile(s, it, ss);
  float ps = exp_block(s[0], 0, it, ss, ph);
  for (int v = vh; v > v0; --v) {
    next_pages(v - 3);
    fetch_k(kr, p, pgk, hk, u);   // tile v - 2
    fetch_v(kr, p, pgv, hk, u);   // tile v - 1
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kb = 0; kb < kNb - 1; ++kb) {
      qk_block(s[kb], kb, sm, (v - 1) & 1, it);
      ps += exp_block(s[kb + 1], kb + 1, it, ss, ph);
      __builtin_amdgcn_sched_barrier(0);
    }
    ss.l = __builtin_fmaf(alpha, ss.l, ps);
    qk_block(s[kNb - 1], kNb - 1, sm, (v - 1) & 1, it);
    store_k(sm, v & 1, kr, half, u);
    put_v(v - 1);
    __builtin_amdgcn_sched_barrier(0);
    mask(v - 1);
    const float next = max_tile(s, it, ss);   // ahead of the PV products: its branch leaves them beside the exponentials
    rescale(o, alpha);
    pv_tile(sm, v & 1, ph, o, it);
    alpha = next;
    ps = exp_block(s[0], 0, it, ss, ph);
    __syncthreads();
  }
#pragma unroll
  for (int kb = 1; kb < kNb; ++kb) ps += exp_block(s[kb], kb, it, ss, ph);
  ss.l = __builtin_fmaf(alpha, ss.l, ps);
  rescale(o, alpha);
  pv_tile(sm, v0 & 1, ph, o, it);
#pragma unroll
  for (int db = 0; db < 4; ++db) asm volatile("" : "+v"(o[db]));
  if (HALF && !join_halves(sm, wave, it, ss, o)) return;
  const float lt = ss.l + __shfl_xor(ss.l, 32);
  // the lane's row once more: kept over the loop it would take registers that the loop needs
  const int lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)), hf = lane >> 5, r = wrow + (lane & 31);
  if (r >= (last + 1 - tok0) * grp) return;
  const int t = it.pos - qs;   // its token
  // accumulator register 4a + i of block db is channel 64 (a%2) + 32 hf + 8 i + 2 db + a/2
  if (state) {
    float* st = state + (int64_t)r * kKv4State;
    if (hf == 0) *reinterpret_cast<float2*>(st) = make_float2(ss.m * it.lam, lt);
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int db = 0; db < 4; ++db)
          *reinterpret_cast<float2*>(st + 2 + 64 * a + 32 * hf + 8 * i + 2 * db) =
              make_float2(o[db][4 * a + i], o[db][8 + 4 * a + i]);
  } else {
    const float inv = lt > 0.0f ? __frcp_rn(lt) * p.v_tscale[b * p.h_kv + hk] : 0.0f;
    uint16_t* dst = p.out + ((int64_t)(q0 + t) * p.h_q + hk * grp + r - (t - tok0) * grp) * kD + 32 * hf;
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u32x4 w;
#pragma unroll
        for (int db = 0; db < 4; ++db)
          w[db] = (uint32_t)bf16_rne(o[db][4 * a + i] * inv) | ((uint32_t)bf16_rne(o[db][8 + 4 * a + i] * inv) << 16);
        *reinterpret_cast<u32x4*>(dst + 64 * a + 8 * i) = w;
      }
  }
}

// floats of the states of one part of an item, for one KV head
__device__ __forceinline__ int64_t state_floats(bool half) { return (half ? kKv4Rows / 2 : kKv4Rows) * kKv4State; }

// Items of a plan, in its order.
template <bool HALF>
__global__ __launch_bounds__(512, 2) void kv4_prefill_plan_kernel(Kv4AttnParams p) {
  __shared__ Kv4Smem sm;
  const int tm = (HALF ? kKv4Rows / 2 : kKv4Rows) / (p.h_q / p.h_kv);
  const int hk = blockIdx.x % p.h_kv;
  const mpfa_kv4_item x = p.items[blockIdx.x / p.h_kv];
  const int q0 = p.cu_seqlens_q[x.seq], nq = p.cu_seqlens_q[x.seq + 1] - q0, qs = p.q_start[x.seq];
  if (x.row >= nq) return;
  const Kv4Tiles tiles = kv4_tiles(qs + x.row, qs + min(x.row + tm, nq) - 1, p.window, p.sinks);
  const int v1 = min(x.last, tiles.nt);
  float* state = x.state < 0 ? nullptr : p.states + ((int64_t)x.state * p.h_kv + hk) * state_floats(HALF);
  if (x.first >= v1) {   // a plan of a longer prompt: a part without tiles adds nothing to its block
    if (state)
      for (int i = threadIdx.x; i < state_floats(HALF); i += 512) state[i] = i % kKv4State == 0 ? -INFINITY : 0.0f;
    return;
  }
  prefill_item<HALF>(p, sm, x.seq, hk, x.row, tm, nq, q0, tiles, x.first, v1, state);
}

// Without one: items of 256 rows, the later (longer) ones first.  Blocks are dealt
// round-robin to the 8 XCDs: with a multiple of 8 KV heads each XCD gets the items of its
// own heads, whose tiles share that XCD's L2.
__global__ __launch_bounds__(512, 2) void kv4_prefill_kernel(Kv4AttnParams p) {
  __shared__ Kv4Smem sm;
  const int tm = kKv4Rows / (p.h_q / p.h_kv);
  const int n_items = (p.max_seqlen_q + tm - 1) / tm;
  int x = blockIdx.x;
  const int hk = x % p.h_kv;
  x /= p.h_kv;
  const int b = x % p.batch, tok0 = (n_items - 1 - x / p.batch) * tm;
  const int q0 = p.cu_seqlens_q[b], nq = p.cu_seqlens_q[b + 1] - q0;
  if (tok0 >= nq) return;
  const int qs = p.q_start[b];
  const Kv4Tiles tiles = kv4_tiles(qs + tok0, qs + min(tok0 + tm, nq) - 1, p.window, p.sinks);
  prefill_item<false>(p, sm, b, hk, tok0, tm, nq, q0, tiles, 0, tiles.nt, nullptr);
}

// Items that the plan cut: four rows per workgroup, one per wave.
__global__ __launch_bounds__(256) void kv4_prefill_merge_kernel(Kv4AttnParams p) {
  const int hk = blockIdx.y, grp = p.h_q / p.h_kv;
  const mpfa_kv4_item x = p.items[p.n_items + blockIdx.z];
  const int r = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), tok = x.row + r / grp;
  const int tm = (p.half ? kKv4Rows / 2 : kKv4Rows) / grp;
  const int q0 = p.cu_seqlens_q[x.seq], nq = p.cu_seqlens_q[x.seq + 1] - q0;
  if (r >= tm * grp || tok >= nq) return;
  const int64_t one = state_floats(p.half);
  kv4_merge_row<1>(p.states + ((int64_t)x.state * p.h_kv + hk) * one + (int64_t)r * kKv4State, one * p.h_kv, x.parts,
                   p.v_tscale[x.seq * p.h_kv + hk], p.out + ((int64_t)(q0 + tok) * p.h_q + hk * grp + r % grp) * kD);
}

}  // namespace

hipError_t launch_kv4_prefill(const Kv4AttnParams& p, hipStream_t stream) {
  if (p.items) {
    const unsigned blocks = (unsigned)p.n_items * p.h_kv;
    if (p.half) kv4_prefill_plan_kernel<true><<<dim3(blocks), 512, 0, stream>>>(p);
    else kv4_prefill_plan_kernel<false><<<dim3(blocks), 512, 0, stream>>>(p);
    if (p.n_merges) {
      const int rows = p.half ? kKv4Rows / 2 : kKv4Rows;
      kv4_prefill_merge_kernel<<<dim3(rows / 4, p.h_kv, p.n_merges), 256, 0, stream>>>(p);
    }
  } else if (p.max_seqlen_q > 0) {
    const int tm = kKv4Rows / (p.h_q / p.h_kv);
    const int64_t items = (int64_t)((p.max_seqlen_q + tm - 1) / tm) * p.h_kv * p.batch;
    kv4_prefill_kernel<<<dim3((unsigned)items), 512, 0, stream>>>(p);
  }
  return hipGetLastError();
}

}  // namespace mpfa
