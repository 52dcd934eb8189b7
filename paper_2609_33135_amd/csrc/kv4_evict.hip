// kv4_evict.hip -- eviction from the 4-bit cache by accumulated attention weight for
// gfx950: which tokens of each (sequence, KV head) stay, and their move to the front of
// the destination pages.
//
// Choice (kv4_select_kernel, one workgroup per (sequence, KV head)): the first `sinks` and
// the last `recent` tokens stay; of the others those of the largest weights, ties to the
// lower index.  Weights become 32-bit images in the same order, tokens that stay the
// largest image, so the threshold is simply the budget-th largest.  It is found by a radix
// selection, 8 bits a pass, over histograms with 16 columns that lanes take in turn (most
// weights share their leading byte and would meet on one counter).  Once at most 256 images
// share the leading bytes (usually after two passes), each is compared with all of them.
// Then two sweeps count and write the indices in order, each wave over a segment of its own.
// The images stay in LDS, 32768 of them; what a longer sequence has more is read again each
// sweep, a page at a time (65536 tokens 91 us, 131072 230).
// What bounds it: one compute unit, of whose 37000 cycles for 32768 tokens a third
// are the read of the weights (beside it the first histogram), a quarter the other sweep for
// the threshold with the comparisons, a quarter the two sweeps for the indices; each spends
// 10 to 20 instructions on 64 tokens.  32768 tokens to 4096, 8 heads: 17.5 to 20 us over cards
// (76 with a histogram per wave and the weights read each sweep; 32 with the images in
// registers; 23 with a sweep more for the first histogram and the places counted in vector
// registers).
//
// Move (kv4_move_kernel): destination place i takes source token kept[i] >= i.  With
// separate pages the places are shared among workgroups; in place, a workgroup per half of
// the planes, or per quarter of either's codes where there are few, goes through them in
// order, reading a chunk before it writes it: a later chunk's sources lie at or after its own
// places, so no write reaches a token that is still to be read.  (The whole call in place,
// by halves and by quarters: 32768 tokens to 4096, 8 heads, 117 and 51 us; 24 sequences to
// 2048, 104 and 112, as the quarters read every line more than once.  Of it the move takes 27
// by quarters and 84 by halves.)
// What bounds it: memory lines.  A kept token's V codes are 4-byte words of two lines; where one
// in four stays up to 330 bytes are read for its 148 (FETCH_SIZE).  24 sequences to 2048 tokens, 8
// heads: 47 to 49 us for up to 124 MB read and 56 written.
#include "kv4_device.h"

namespace mpfa {

namespace {

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
constexpr int kHeld = 32;        // pages per wave whose images stay in LDS (128 KB, 32768 tokens)
constexpr int kLoads = 16;       // pages in flight when they are filled
constexpr int kAhead = 4;        // pages per step of a sweep
constexpr int kListed = 256;     // images compared with each other (each thread one)
constexpr int kColumns = 16;     // histogram columns
constexpr int kManyHeads = 64;   // (sequence, KV head) pairs from which halves of the planes fill the card
constexpr int kMoveTokens = 4;   // tokens per thread and step of the move
static_assert(256 * kColumns == 4 * kSelectThreads, "one 16-byte word of the histogram per thread");
static_assert(kHeld % kLoads == 0 && kHeld % kAhead == 0 && kHeld <= 64, "whole reads of held pages");

// FP32 order as unsigned order; -0 as +0; NaN above everything.
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w + 0.0f);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0xFFFFFFFEu;
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

constexpr uint32_t kStays = 0xFFFFFFFFu, kNone = 0u;   // images of a token that stays anyway, and of no token

__global__ __launch_bounds__(kSelectThreads) void kv4_select_kernel(Kv4EvictParams p) {
  __shared__ __attribute__((aligned(16))) uint32_t hist[256 * kColumns];   // [bin][column]
  __shared__ uint32_t images[kSelectWaves * kHeld * 64];
  __shared__ uint32_t total[256];
  __shared__ uint32_t s_prefix, s_need, s_count, s_listed;
  __shared__ int above[kSelectWaves], equal[kSelectWaves];
  const int hk = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = max(p.kv_len[b], 0);
  int32_t* kept = p.kept + ((int64_t)b * p.h_kv + hk) * p.budget;
  if (n <= p.budget) {   // everything stays
    for (int i = tid; i < p.budget; i += kSelectThreads) kept[i] = i < n ? i : -1;
    return;
  }
  const int32_t* pt = p.page_table + (int64_t)b * p.max_pages;
  const int lo = p.sinks, hi = n - p.recent;   // tokens that compete: lo .. hi - 1
  // waves own segments of whole pages, in order
  const int pages = (n + 63) >> 6, seg = (pages + kSelectWaves - 1) / kSelectWaves;
  const int g0 = wave * seg, mine = max(0, min(pages - g0, seg));
  auto image_of = [&](int i, float w) {
    return i >= n ? kNone : (i < lo || i >= hi ? kStays : weight_key(w));
  };
  auto clear = [&] { reinterpret_cast<u32x4*>(hist)[tid] = (u32x4){0u, 0u, 0u, 0u}; };
  auto count_in = [&](uint32_t k, int shift) {
    atomicAdd(&hist[((k >> shift) & 255u) * kColumns + (lane & (kColumns - 1))], 1u);
  };
  clear();
  if (tid == 0) {
    s_prefix = s_listed = 0u;
    s_need = (uint32_t)p.budget;
  }
  __syncthreads();
  // The images, and beside the loads the histogram of their first byte.  Sixteen lanes read a
  // page, four tokens each.
  uint32_t* own = images + wave * kHeld * 64;   // the wave's images, one page per 64
  const int my_page = mine > 0 ? pt[g0 + min(lane & (kHeld - 1), mine - 1)] : 0;
  for (int j0 = 0; j0 < min(mine, kHeld); j0 += kLoads) {
    f32x4 w[kLoads / 4];
#pragma unroll
    for (int j = 0; j < kLoads / 4; ++j)
      w[j] = reinterpret_cast<const f32x4*>(
          p.cache.weights + kv4_row(__shfl(my_page, j0 + 4 * j + (lane >> 4)), p.h_kv, hk) * kPage)[lane & 15];
#pragma unroll
    for (int j = 0; j < kLoads / 4; ++j) {
      const int pg = j0 + 4 * j + (lane >> 4), i = (g0 + pg) * 64 + 4 * (lane & 15);
      u32x4 k;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        k[e] = pg < mine ? image_of(i + e, w[j][e]) : kNone;
        if (pg < mine) count_in(k[e], 24);
      }
      reinterpret_cast<u32x4*>(own)[(j0 / 4 + j) * 64 + lane] = k;
    }
  }
  auto rest = [&](auto&& f) {   // what is not held
    for (int j = kHeld; j < mine; ++j)
      f(j, image_of((g0 + j) * 64 + lane, p.cache.weights[kv4_row(pt[g0 + j], p.h_kv, hk) * kPage + lane]));
  };
  rest([&](int, uint32_t k) { count_in(k, 24); });
  __syncthreads();
  // f(j, image) for the wave's pages in order
  auto sweep = [&](auto&& f) {
    for (int j0 = 0; j0 < min(mine, kHeld); j0 += kAhead) {   // past `mine` no token's image
      uint32_t k[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) k[j] = own[(j0 + j) * 64 + lane];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) f(j0 + j, k[j]);
    }
    rest(f);
  };

  // ---- threshold: the budget-th largest image
  for (int shift = 24;; shift -= 8) {
    const uint32_t base = s_prefix, left = s_need;
    {   // four threads per bin, a quarter of its columns each
      const u32x4 w = reinterpret_cast<const u32x4*>(hist)[tid];
      uint32_t t = (w[0] + w[1]) + (w[2] + w[3]);
      t += __shfl_xor(t, 1);
      t += __shfl_xor(t, 2);
      if ((tid & 3) == 0) total[tid >> 2] = t;
    }
    __syncthreads();
    if (wave == 0) {   // lane l holds bins 4l .. 4l + 3
      uint32_t c[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        c[i] = total[4 * lane + i];
        sum += c[i];
      }
      uint32_t up = sum;   // inclusive suffix sum over the lanes
      for (int off = 1; off < 64; off <<= 1) {
        const uint32_t o = __shfl_down(up, off);
        if (lane + off < 64) up += o;
      }
      uint32_t over = up - sum;   // images in bins of higher lanes
#pragma unroll
      for (int i = 3; i >= 0; --i) {
        if (over < left && left <= over + c[i]) {
          s_prefix = base | ((uint32_t)(4 * lane + i) << shift);
          s_need = left - over;
          s_count = c[i];
        }
        over += c[i];
      }
    }
    __syncthreads();
    if (shift == 0) break;
    const uint32_t found = s_prefix, count = s_count;
    auto inside = [&](uint32_t k) { return (k >> shift) == (found >> shift); };
    clear();
    __syncthreads();
    if (count <= kListed) {   // few enough: each image against all of them
      const uint32_t need = s_need;
      uint32_t* list = hist;         // its first words are zero: no image
      sweep([&](int, uint32_t k) {
        if (k != kNone && inside(k)) list[atomicAdd(&s_listed, 1u)] = k;
      });
      __syncthreads();
      {   // four threads per image, every fourth four of the others each
        const uint32_t k = list[tid >> 2];
        uint32_t gt = 0, ge = 0;
#pragma unroll 1
        for (uint32_t i = 4 * (tid & 3); i < count; i += 16) {
          const u32x4 o = reinterpret_cast<const u32x4*>(list)[i >> 2];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            gt += o[e] > k;
            ge += o[e] >= k;
          }
        }
        for (int off = 1; off <= 2; off <<= 1) {
          gt += __shfl_xor(gt, off);
          ge += __shfl_xor(ge, off);
        }
        if (k != kNone && gt < need && need <= ge) {   // the equal ones all write the same
          s_prefix = k;
          s_need = need - gt;
        }
      }
      __syncthreads();
      break;
    }
    sweep([&](int, uint32_t k) {
      if (inside(k)) count_in(k, shift - 8);
    });
    __syncthreads();
  }
  const uint32_t prefix = s_prefix;
  const int need = (int)s_need;   // of the images equal to the threshold, the first `need` stay

  // ---- counts per wave, then places
  int na = 0, ne = 0;
  sweep([&](int, uint32_t k) {
    na += __popcll(__ballot(k > prefix));
    ne += __popcll(__ballot(k == prefix));
  });
  if (lane == 0) {
    above[wave] = na;
    equal[wave] = ne;
  }
  __syncthreads();
  int place = 0, eq = 0;   // places taken and equal images met before this wave's segment
  for (int w = 0; w < wave; ++w) {
    place += above[w] + min(equal[w], max(0, need - eq));
    eq += equal[w];
  }
  // base + the number of lower lanes in m
  auto rank = [](uint64_t m, int base) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, base));
  };
  place = __builtin_amdgcn_readfirstlane(place);
  eq = __builtin_amdgcn_readfirstlane(eq);
  auto choose = [&](uint32_t k) {
    uint64_t am = __ballot(k > prefix);
    const uint64_t em = __ballot(k == prefix);
    if (em) {
      am |= __ballot(k == prefix && rank(em, eq) < need);
      eq += __popcll(em);
    }
    return am;
  };
  sweep([&](int j, uint32_t k) {
    const uint64_t am = choose(k);
    if (__builtin_amdgcn_inverse_ballot_w64(am)) kept[(uint32_t)rank(am, place)] = (g0 + j) * 64 + lane;
    place += __popcll(am);
  });
}

// What a thread moves of a token: a 4-byte piece of K's codes, of V's, or both, with some
// threads SCALES group scales, and with one the weight.
template <int SCALES>
struct Moved {
  uint32_t k, v, w;
  uint8_t sk[SCALES], sv[SCALES];
};

// Grid x: the workgroups that share the places, or in place one; y: the KV head and, in
// place, the part of the planes, whose workgroups do not depend on each other: K's or V's
// half (PARTS 2), or a quarter of either's codes (8).  PARTS 1: not in place.
template <int PARTS>
__global__ __launch_bounds__(1024) void kv4_move_kernel(Kv4EvictParams p) {
  constexpr bool IN_PLACE = PARTS > 1;
  constexpr int kPieces = PARTS == 8 ? 4 : 16, kSlots = 1024 / kPieces, kChunk = kSlots * kMoveTokens;
  constexpr int kScales = PARTS == 8 ? 2 : 1;
  const int b = blockIdx.z, hk = blockIdx.y / PARTS, part = blockIdx.y % PARTS;
  const int quarter = PARTS == 8 ? part & 3 : 0;
  const int local = threadIdx.x & (kPieces - 1), piece = local + kPieces * quarter, slot = threadIdx.x / kPieces;
  const bool do_k = PARTS == 1 || part < PARTS / 2, do_v = PARTS == 1 || part >= PARTS / 2;
  const bool scales = PARTS == 8 ? quarter == 0 : local < 8;
  const bool weight = PARTS == 8 ? part == 0 && local == 0 : local == 8;
  const int n = min(max(p.kv_len[b], 0), p.budget);
  const int32_t* kept = p.kept + ((int64_t)b * p.h_kv + hk) * p.budget;
  const int32_t* src_pt = p.page_table + (int64_t)b * p.max_pages;
  const int32_t* dst_pt = p.dst_page_table + (int64_t)b * p.dst_max_pages;
  const int steps = (n + kChunk - 1) / kChunk;
  for (int c = blockIdx.x; c < steps; c += gridDim.x) {
    Moved<kScales> m[kMoveTokens] = {};
    bool have[kMoveTokens];
#pragma unroll
    for (int t = 0; t < kMoveTokens; ++t) {
      const int i = c * kChunk + t * kSlots + slot;
      have[t] = i < n;
      const int s = have[t] ? kept[i] : 0;
      if (IN_PLACE && s == i) have[t] = false;   // it stays where it is
      if (!have[t]) continue;
      const int o = s & (kPage - 1);
      const int64_t row = kv4_row(src_pt[s >> 6], p.h_kv, hk);
      if (do_k) {
        m[t].k = reinterpret_cast<const uint32_t*>(p.cache.k_codes + (row * kPage + o) * 64)[piece];
        if (scales) {
#pragma unroll
          for (int g = 0; g < kScales; ++g) m[t].sk[g] = p.cache.k_scales[(row * kPage + o) * 8 + kScales * local + g];
        }
        if (weight) m[t].w = __float_as_uint(p.cache.weights[row * kPage + o]);
      }
      if (do_v) {
        m[t].v = reinterpret_cast<const uint32_t*>(p.cache.v_codes + (row * 16 + (o >> 2)) * 256)[piece * 4 + (o & 3)];
        if (scales) {
#pragma unroll
          for (int g = 0; g < kScales; ++g) m[t].sv[g] = p.cache.v_scales[(row * 8 + kScales * local + g) * kPage + o];
        }
      }
    }
    if (IN_PLACE) __syncthreads();   // the chunk is read before any of it is written
#pragma unroll
    for (int t = 0; t < kMoveTokens; ++t) {
      if (!have[t]) continue;
      const int i = c * kChunk + t * kSlots + slot, o = i & (kPage - 1);
      const int64_t row = kv4_row(dst_pt[i >> 6], p.h_kv, hk);
      if (do_k) {
        reinterpret_cast<uint32_t*>(p.cache.k_codes + (row * kPage + o) * 64)[piece] = m[t].k;
        if (scales) {
#pragma unroll
          for (int g = 0; g < kScales; ++g) p.cache.k_scales[(row * kPage + o) * 8 + kScales * local + g] = m[t].sk[g];
        }
        if (weight) p.cache.weights[row * kPage + o] = __uint_as_float(m[t].w);
      }
      if (do_v) {
        reinterpret_cast<uint32_t*>(p.cache.v_codes + (row * 16 + (o >> 2)) * 256)[piece * 4 + (o & 3)] = m[t].v;
        if (scales) {
#pragma unroll
          for (int g = 0; g < kScales; ++g) p.cache.v_scales[(row * 8 + kScales * local + g) * kPage + o] = m[t].sv[g];
        }
      }
    }
    if (IN_PLACE) __syncthreads();
  }
  // new_len may be kv_len: this kernel gets the same n from either value, and the choice has
  // read the lengths before it
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) p.new_len[b] = n;
}

}  // namespace

hipError_t launch_kv4_evict(const Kv4EvictParams& p, hipStream_t stream) {
  kv4_select_kernel<<<dim3(p.h_kv, p.batch), kSelectThreads, 0, stream>>>(p);
  constexpr int kChunk = 64 * kMoveTokens;   // places per step, 16 threads each
  const int steps = (int)(((int64_t)p.budget + kChunk - 1) / kChunk);
  if (!p.in_place) kv4_move_kernel<1><<<dim3(min(steps, 4096), p.h_kv, p.batch), 1024, 0, stream>>>(p);
  else if (p.h_kv * p.batch >= kManyHeads) kv4_move_kernel<2><<<dim3(1, 2 * p.h_kv, p.batch), 1024, 0, stream>>>(p);
  else kv4_move_kernel<8><<<dim3(1, 8 * p.h_kv, p.batch), 1024, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace mpfa
