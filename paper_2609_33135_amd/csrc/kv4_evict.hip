// kv4_evict.hip -- eviction from the 4-bit cache by accumulated attention weight for
// gfx950: which tokens of each (sequence, KV head) stay, and their move to the front of
// the destination pages.
//
// Choice (kv4_select_kernel, one workgroup per (sequence, KV head)): the first `sinks` and
// the last `recent` tokens stay; of the others those of the largest weights, ties to the
// lower index.  The threshold is found by a radix selection over order-preserving 32-bit
// images of the weights (8 bits a pass, one histogram per wave so that weights with the
// same leading byte do not meet on one counter), then two sweeps count and write the
// indices in order, each wave over a segment of its own.  What bounds it: six sweeps over
// 4 bytes per token, from L2 after the first.
//
// Move (kv4_move_kernel): destination place i takes source token kept[i] >= i.  With
// separate pages the places are shared among workgroups; in place, one workgroup per plane
// goes through them in order, reading a chunk before it writes it: a later chunk's sources
// lie at or after its own places, so no write reaches a token that is still to be read.
#include "kv4_device.h"

namespace mpfa {

namespace {

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
constexpr int kMoveChunk = 64;   // places per step of the move: 16 threads each (1024)

// FP32 order as unsigned order; -0 as +0; NaN above everything.
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w + 0.0f);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0xFFFFFFFEu;
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kSelectThreads) void kv4_select_kernel(Kv4EvictParams p) {
  __shared__ uint32_t hist[kSelectWaves][256];
  __shared__ uint32_t total[256];
  __shared__ uint32_t s_prefix, s_need;
  __shared__ int above[kSelectWaves], equal[kSelectWaves];
  const int hk = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = max(p.kv_len[b], 0);
  int32_t* kept = p.kept + ((int64_t)b * p.h_kv + hk) * p.budget;
  if (tid == 0 && hk == 0) p.new_len[b] = min(n, p.budget);
  if (n <= p.budget) {   // everything stays
    for (int i = tid; i < p.budget; i += kSelectThreads) kept[i] = i < n ? i : -1;
    return;
  }
  const int32_t* pt = p.page_table + (int64_t)b * p.max_pages;
  const int lo = p.sinks, hi = n - p.recent;             // tokens that compete: lo .. hi - 1
  const int want = p.budget - p.sinks - p.recent;        // of them stay (>= 0, < hi - lo since n > budget)
  auto key_of = [&](int i) {
    return weight_key(p.cache.weights[kv4_row(pt[i >> 6], p.h_kv, hk) * kPage + (i & (kPage - 1))]);
  };
  // waves own segments of whole pages, in order
  const int pages = (n + 63) >> 6, seg = (pages + kSelectWaves - 1) / kSelectWaves;
  const int g0 = wave * seg, g1 = min(pages, g0 + seg);

  // ---- threshold: the want-th largest key (want == 0: above every key)
  uint32_t prefix = 0xFFFFFFFFu, need = 0;
  if (want > 0) {
    if (tid == 0) {
      s_prefix = 0u;
      s_need = (uint32_t)want;
    }
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < kSelectWaves * 256; i += kSelectThreads) hist[0][i] = 0u;
      __syncthreads();
      const uint32_t base = s_prefix, left = s_need;
      for (int g = g0; g < g1; ++g) {
        const int i = g * 64 + lane;
        if (i >= lo && i < hi) {
          const uint32_t k = key_of(i);
          if (shift == 24 || (k >> (shift + 8)) == (base >> (shift + 8))) atomicAdd(&hist[wave][(k >> shift) & 255u], 1u);
        }
      }
      __syncthreads();
      if (tid < 256) {
        uint32_t t = 0;
        for (int w = 0; w < kSelectWaves; ++w) t += hist[w][tid];
        total[tid] = t;
      }
      __syncthreads();
      if (wave == 0) {   // lane l holds bins 4l .. 4l + 3; counts of the bins above
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
        uint32_t over = up - sum;   // keys in bins of higher lanes
#pragma unroll
        for (int i = 3; i >= 0; --i) {
          if (over < left && left <= over + c[i]) {
            s_prefix = base | ((uint32_t)(4 * lane + i) << shift);
            s_need = left - over;
          }
          over += c[i];
        }
      }
      __syncthreads();
    }
    prefix = s_prefix;
    need = s_need;   // of the keys equal to the threshold, the first `need` stay
  }

  // ---- counts per wave, then places
  int na = 0, ne = 0;
  for (int g = g0; g < g1; ++g) {
    const int i = g * 64 + lane;
    bool a = i < n && (i < lo || i >= hi), e = false;
    if (want > 0 && i >= lo && i < hi) {
      const uint32_t k = key_of(i);
      a = k > prefix;
      e = k == prefix;
    }
    na += __popcll(__ballot(a));
    ne += __popcll(__ballot(e));
  }
  if (lane == 0) {
    above[wave] = na;
    equal[wave] = ne;
  }
  __syncthreads();
  int place = 0, eq = 0;   // places taken and equal keys met before this wave's segment
  for (int w = 0; w < wave; ++w) {
    const int take = min(equal[w], max(0, (int)need - eq));
    place += above[w] + take;
    eq += equal[w];
  }
  for (int g = g0; g < g1; ++g) {
    const int i = g * 64 + lane;
    bool a = i < n && (i < lo || i >= hi), e = false;
    if (want > 0 && i >= lo && i < hi) {
      const uint32_t k = key_of(i);
      a = k > prefix;
      e = k == prefix;
    }
    const uint64_t below = (1ull << lane) - 1ull, em = __ballot(e);
    if (e && eq + __popcll(em & below) < (int)need) a = true;
    const uint64_t am = __ballot(a);
    if (a) kept[place + __popcll(am & below)] = i;
    place += __popcll(am);
    eq += __popcll(em);
  }
}

// A thread's part of a token: of every plane the piece that `piece` (0 .. 15) names.
struct Moved {
  uint32_t k, v, w;
  uint8_t sk, sv;
};

__global__ __launch_bounds__(1024) void kv4_move_kernel(Kv4EvictParams p) {
  const int hk = blockIdx.y, b = blockIdx.z, piece = threadIdx.x & 15, slot = threadIdx.x >> 4;
  const int n = min(max(p.kv_len[b], 0), p.budget);
  const int32_t* kept = p.kept + ((int64_t)b * p.h_kv + hk) * p.budget;
  const int32_t* src_pt = p.page_table + (int64_t)b * p.max_pages;
  const int32_t* dst_pt = p.dst_page_table + (int64_t)b * p.dst_max_pages;
  const int steps = (n + kMoveChunk - 1) / kMoveChunk;
  for (int c = blockIdx.x; c < steps; c += gridDim.x) {
    const int i = c * kMoveChunk + slot;
    const bool have = i < n;
    Moved m = {};
    if (have) {
      const int s = kept[i], o = s & (kPage - 1);
      const int64_t row = kv4_row(src_pt[s >> 6], p.h_kv, hk);
      m.k = reinterpret_cast<const uint32_t*>(p.cache.k_codes + (row * kPage + o) * 64)[piece];
      m.v = reinterpret_cast<const uint32_t*>(p.cache.v_codes + (row * 16 + (o >> 2)) * 256)[piece * 4 + (o & 3)];
      if (piece < 8) {
        m.sk = p.cache.k_scales[(row * kPage + o) * 8 + piece];
        m.sv = p.cache.v_scales[(row * 8 + piece) * kPage + o];
      }
      if (piece == 8) m.w = __float_as_uint(p.cache.weights[row * kPage + o]);
    }
    if (p.in_place) __syncthreads();   // the chunk is read before any of it is written
    if (have) {
      const int o = i & (kPage - 1);
      const int64_t row = kv4_row(dst_pt[i >> 6], p.h_kv, hk);
      reinterpret_cast<uint32_t*>(p.cache.k_codes + (row * kPage + o) * 64)[piece] = m.k;
      reinterpret_cast<uint32_t*>(p.cache.v_codes + (row * 16 + (o >> 2)) * 256)[piece * 4 + (o & 3)] = m.v;
      if (piece < 8) {
        p.cache.k_scales[(row * kPage + o) * 8 + piece] = m.sk;
        p.cache.v_scales[(row * 8 + piece) * kPage + o] = m.sv;
      }
      if (piece == 8) p.cache.weights[row * kPage + o] = __uint_as_float(m.w);
    }
    if (p.in_place) __syncthreads();
  }
}

}  // namespace

hipError_t launch_kv4_evict(const Kv4EvictParams& p, hipStream_t stream) {
  kv4_select_kernel<<<dim3(p.h_kv, p.batch), kSelectThreads, 0, stream>>>(p);
  const int steps = (p.budget + kMoveChunk - 1) / kMoveChunk;
  kv4_move_kernel<<<dim3(p.in_place ? 1 : steps, p.h_kv, p.batch), 1024, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace mpfa
