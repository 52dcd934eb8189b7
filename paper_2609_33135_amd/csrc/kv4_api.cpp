// kv4_api.cpp -- the C ABI of the 4-bit cache (include/mpfa.h): host-side validation (no
// HIP call before an argument set is accepted), workspace sizes and partition policies.
#include "mpfa.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "kv4_internal.h"

#ifdef MPFA_DEBUG_CHECKS
#include <vector>

#include "mpfa_internal.h"
#endif

namespace {

constexpr int kMaxKvHeads = 32;
constexpr int kFar = 1 << 30;   // windows and sinks from here on see every key there can be
constexpr float kLambda = 0.12751743074173085f;   // log2(e) / sqrt(128)
constexpr int64_t kMaxStride = (int64_t)1 << 31;  // elements between tokens

mpfa_status dim_ok(int head_dim) {
  if (head_dim == MPFA_HEAD_DIM) return MPFA_OK;
  return head_dim > 0 ? MPFA_ERR_UNSUPPORTED : MPFA_ERR_INVALID;
}

bool aligned16(const void* x) { return (reinterpret_cast<uintptr_t>(x) & 15) == 0; }

// token stride of a [T][heads][128] tensor: whole rows, 16-byte loads
bool stride_ok(int64_t stride, int heads) {
  return stride >= (int64_t)heads * MPFA_HEAD_DIM && stride % 8 == 0 && stride < kMaxStride;
}

bool kv_heads_ok(int h_kv) { return h_kv >= 1 && h_kv <= kMaxKvHeads; }

bool cache_ok(const mpfa_kv4_cache& c) {
  return c.k_codes && c.k_scales && c.v_codes && c.v_scales && c.num_pages >= 1 &&
         c.num_pages <= INT32_MAX && aligned16(c.k_codes) && aligned16(c.k_scales) && aligned16(c.v_codes) &&
         aligned16(c.v_scales) && aligned16(c.weights);
}

mpfa::Kv4Cache planes(const mpfa_kv4_cache& c) {
  return {c.k_codes, c.k_scales, c.v_codes, c.v_scales, c.weights};
}

int far(int x) { return x < kFar ? x : kFar; }

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// Bytes of the three parts of a decode workspace: partition states, then with weights the
// merged statistics and the scores.  False where a size does not fit.
struct DecodeSpace {
  size_t states, stats, scores;
};
bool decode_space(int batch, int h_q, int q_tokens, int partition_tokens, int max_partitions, bool weights, DecodeSpace* s) {
  const double rows = (double)batch * q_tokens * h_q;
  const double keys = (double)max_partitions * partition_tokens;
  if (rows * max_partitions * mpfa::kKv4State * 4 + (weights ? rows * (8 + keys * 4) : 0) > 9e18) return false;
  const size_t r = (size_t)batch * q_tokens * h_q;
  s->states = align256(r * max_partitions * mpfa::kKv4State * sizeof(float));
  s->stats = weights ? align256(r * 2 * sizeof(float)) : 0;
  s->scores = weights ? r * (size_t)max_partitions * partition_tokens * sizeof(float) : 0;
  return true;
}

// What prefill and decode share.
mpfa_status attn_params(const mpfa_kv4_attn_args* a, mpfa::Kv4AttnParams& p) {
  if (!a) return MPFA_ERR_INVALID;
  if (const mpfa_status st = dim_ok(a->head_dim)) return st;
  if (a->batch < 1 || a->batch > 65535 || a->max_pages < 1) return MPFA_ERR_INVALID;
  if (a->max_pages > INT32_MAX / MPFA_PAGE_TOKENS) return MPFA_ERR_INVALID;
  if (!kv_heads_ok(a->h_kv) || a->h_q < 1 || a->h_q > MPFA_MAX_HEADS || a->h_q % a->h_kv) return MPFA_ERR_INVALID;
  if (a->window < 0 || a->sinks < 0) return MPFA_ERR_INVALID;
  if (a->partition_tokens < 0 || a->partition_tokens % MPFA_KV_TILE || a->max_partitions < 0) return MPFA_ERR_INVALID;
  p = mpfa::Kv4AttnParams{};
  if (a->q_tokens == 0 && a->total_tokens == 0) return MPFA_OK;   // a prefill without rows
  if (!cache_ok(a->cache) || !stride_ok(a->q_stride, a->h_q) || !aligned16(a->q) || !aligned16(a->out)) return MPFA_ERR_INVALID;
  if (!a->kv_len || !a->page_table || !a->q || !a->k_tscale || !a->v_tscale || !a->out) return MPFA_ERR_INVALID;
  p.batch = a->batch;
  p.h_q = a->h_q;
  p.h_kv = a->h_kv;
  p.max_pages = a->max_pages;
  p.partition_tiles = a->partition_tokens / MPFA_KV_TILE;
  p.max_partitions = a->max_partitions;
  p.window = far(a->window);
  p.sinks = far(a->sinks);
  p.xcd_remap = a->h_kv % 8 == 0;
  p.lam = kLambda;
  p.q_stride = a->q_stride;
  p.cu_seqlens_q = a->cu_seqlens_q;
  p.q_start = a->q_start;
  p.kv_len = a->kv_len;
  p.page_table = a->page_table;
  p.q = static_cast<const uint16_t*>(a->q);
  p.cache = planes(a->cache);
  p.k_tscale = a->k_tscale;
  p.v_tscale = a->v_tscale;
  p.out = static_cast<uint16_t*>(a->out);
  return MPFA_OK;
}

// Tiles seen from a block of rows at positions first .. last.
int64_t seen_tiles(int64_t first, int64_t last, int window, int sinks) {
  return mpfa::kv4_tiles((int)std::max<int64_t>(first, 0), (int)last, far(window), far(sinks)).nt;
}

#ifdef MPFA_DEBUG_CHECKS
template <typename T>
bool to_host(const T* dev, size_t n, std::vector<T>& out) {
  out.resize(n);
  return n == 0 || hipMemcpy(out.data(), dev, n * sizeof(T), hipMemcpyDeviceToHost) == hipSuccess;
}

// rows [T][row] at a token stride: finite values?
mpfa_status scan_rows(const void* x, int64_t tokens, int64_t row, int64_t stride, hipStream_t s) {
  int* flag = nullptr;
  if (tokens == 0) return MPFA_OK;
  if (hipMalloc(&flag, sizeof(int)) != hipSuccess) return MPFA_ERR_HIP;
  int h = 0;
  bool ok = hipMemsetAsync(flag, 0, sizeof(int), s) == hipSuccess;
  if (stride == row) {
    ok = ok && mpfa::launch_scan_nonfinite(static_cast<const uint16_t*>(x), tokens * row, flag, s) == hipSuccess;
  } else {
    for (int64_t t = 0; t < tokens; ++t)
      ok = ok && mpfa::launch_scan_nonfinite(static_cast<const uint16_t*>(x) + t * stride, row, flag, s) == hipSuccess;
  }
  ok = ok && hipMemcpyAsync(&h, flag, sizeof(int), hipMemcpyDeviceToHost, s) == hipSuccess && hipStreamSynchronize(s) == hipSuccess;
  (void)hipFree(flag);
  if (!ok) return MPFA_ERR_HIP;
  return h ? MPFA_ERR_DATA : MPFA_OK;
}

// the first `pages` entries of row b
bool row_pages_ok(const std::vector<int32_t>& pt, int b, int max_pages, int64_t pages, int64_t num_pages) {
  if (pages > max_pages) return false;
  for (int64_t i = 0; i < pages; ++i) {
    const int32_t e = pt[(size_t)b * max_pages + i];
    if (e < 0 || e >= num_pages) return false;
  }
  return true;
}

mpfa_status check_write(const mpfa_kv4_write_args* a, hipStream_t s) {
  if (hipStreamSynchronize(s) != hipSuccess) return MPFA_ERR_HIP;
  std::vector<int32_t> cu;
  std::vector<int64_t> slots;
  if (!to_host(a->cu_seqlens, (size_t)a->batch + 1, cu) || !to_host(a->slot_mapping, (size_t)a->total_tokens, slots))
    return MPFA_ERR_HIP;
  if (cu[0] != 0 || cu[a->batch] != a->total_tokens) return MPFA_ERR_DATA;
  for (int b = 0; b < a->batch; ++b)
    if (cu[b + 1] < cu[b] || cu[b + 1] - cu[b] > a->max_seqlen) return MPFA_ERR_DATA;
  std::sort(slots.begin(), slots.end());
  for (size_t i = 0; i < slots.size(); ++i)   // negative: padding
    if (slots[i] >= 64 * a->cache.num_pages || (i > 0 && slots[i] >= 0 && slots[i] == slots[i - 1])) return MPFA_ERR_DATA;
  mpfa_status st = scan_rows(a->k, a->total_tokens, (int64_t)a->h_kv * MPFA_HEAD_DIM, a->k_stride, s);
  if (st == MPFA_OK) st = scan_rows(a->v, a->total_tokens, (int64_t)a->h_kv * MPFA_HEAD_DIM, a->v_stride, s);
  return st;
}

mpfa_status check_attn(const mpfa_kv4_attn_args* a, bool decode, hipStream_t s) {
  if (hipStreamSynchronize(s) != hipSuccess) return MPFA_ERR_HIP;
  std::vector<int32_t> cu, qs, kv, pt;
  if (!to_host(a->kv_len, (size_t)a->batch, kv) || !to_host(a->page_table, (size_t)a->batch * a->max_pages, pt)) return MPFA_ERR_HIP;
  if (!decode && (!to_host(a->cu_seqlens_q, (size_t)a->batch + 1, cu) || !to_host(a->q_start, (size_t)a->batch, qs)))
    return MPFA_ERR_HIP;
  const int tm = mpfa::kKv4Rows / (a->h_q / a->h_kv);
  for (int b = 0; b < a->batch; ++b) {
    if (kv[b] < 0 || !row_pages_ok(pt, b, a->max_pages, ((int64_t)kv[b] + 63) / 64, a->cache.num_pages)) return MPFA_ERR_DATA;
    const int64_t room = (int64_t)a->max_partitions * (a->partition_tokens / MPFA_KV_TILE);
    if (decode) {
      if (seen_tiles((int64_t)kv[b] - a->q_tokens, kv[b] - 1, a->window, a->sinks) > room) return MPFA_ERR_DATA;
      continue;
    }
    const int n = cu[b + 1] - cu[b];
    if (n < 0 || n > a->max_seqlen_q || qs[b] < 0 || (int64_t)qs[b] + n > kv[b]) return MPFA_ERR_DATA;
    for (int t = 0; a->partition_tokens > 0 && t < n; t += tm)
      if (seen_tiles(qs[b] + t, qs[b] + std::min(t + tm, n) - 1, a->window, a->sinks) > room) return MPFA_ERR_DATA;
  }
  if (!decode && cu[0] != 0) return MPFA_ERR_DATA;
  const int64_t rows = decode ? (int64_t)a->batch * a->q_tokens : cu[a->batch];
  return scan_rows(a->q, rows, (int64_t)a->h_q * MPFA_HEAD_DIM, a->q_stride, s);
}

mpfa_status check_evict(const mpfa_kv4_evict_args* a, hipStream_t s) {
  if (hipStreamSynchronize(s) != hipSuccess) return MPFA_ERR_HIP;
  std::vector<int32_t> kv, pt, dt;
  if (!to_host(a->kv_len, (size_t)a->batch, kv) || !to_host(a->page_table, (size_t)a->batch * a->max_pages, pt) ||
      !to_host(a->dst_page_table, (size_t)a->batch * a->dst_max_pages, dt))
    return MPFA_ERR_HIP;
  std::vector<uint8_t> read((size_t)a->cache.num_pages, 0), written((size_t)a->cache.num_pages, 0);
  const bool in_place = a->flags & MPFA_KV4_IN_PLACE;
  for (int b = 0; b < a->batch; ++b) {
    const int64_t src = ((int64_t)kv[b] + 63) / 64, dst = ((int64_t)std::min(kv[b], a->budget) + 63) / 64;
    if (kv[b] < 0 || !row_pages_ok(pt, b, a->max_pages, src, a->cache.num_pages) ||
        !row_pages_ok(dt, b, a->dst_max_pages, dst, a->cache.num_pages))
      return MPFA_ERR_DATA;
    for (int64_t i = 0; i < src; ++i) {
      uint8_t& r = read[pt[(size_t)b * a->max_pages + i]];
      if (in_place && r) return MPFA_ERR_DATA;   // a page that another sequence reads
      r = 1;
    }
  }
  for (int b = 0; b < a->batch; ++b)
    for (int64_t i = 0; i < ((int64_t)std::min(kv[b], a->budget) + 63) / 64; ++i) {
      const int32_t e = dt[(size_t)b * a->dst_max_pages + i];
      if (written[e] || (in_place ? e != pt[(size_t)b * a->max_pages + i] : read[e] != 0)) return MPFA_ERR_DATA;
      written[e] = 1;
    }
  return MPFA_OK;
}
#endif

mpfa_status done(hipError_t e) { return e == hipSuccess ? MPFA_OK : MPFA_ERR_HIP; }

}  // namespace

extern "C" {

mpfa_status mpfa_kv4_write_workspace_size(int32_t batch, int32_t total_tokens, int32_t h_kv, size_t* bytes) {
  if (!bytes || batch < 1 || total_tokens < 0 || !kv_heads_ok(h_kv)) return MPFA_ERR_INVALID;
  *bytes = ((size_t)total_tokens / mpfa::kKv4StatTokens + batch) * h_kv * mpfa::kKv4StatBytes;
  return MPFA_OK;
}

mpfa_status mpfa_kv4_write(const mpfa_kv4_write_args* a, void* workspace, size_t workspace_bytes, mpfa_stream_t stream) {
  if (!a) return MPFA_ERR_INVALID;
  if (const mpfa_status st = dim_ok(a->head_dim)) return st;
  if (a->batch < 1 || a->total_tokens < 0 || a->max_seqlen < 0) return MPFA_ERR_INVALID;
  if (!kv_heads_ok(a->h_kv) || (a->flags & ~(MPFA_SMOOTH | MPFA_COMPUTE_STATS))) return MPFA_ERR_INVALID;
  if (a->total_tokens == 0) return MPFA_OK;
  const bool stats = a->flags & MPFA_COMPUTE_STATS, smooth = a->flags & MPFA_SMOOTH;
  if (!cache_ok(a->cache) || !stride_ok(a->k_stride, a->h_kv) || !stride_ok(a->v_stride, a->h_kv)) return MPFA_ERR_INVALID;
  if (!a->cu_seqlens || !a->k || !a->v || !a->slot_mapping || !a->k_tscale || !a->v_tscale || ((stats || smooth) && !a->k_mean))
    return MPFA_ERR_INVALID;
  if (!aligned16(a->k) || !aligned16(a->v) || !aligned16(a->k_mean) || !aligned16(a->k_out) || !aligned16(a->v_out))
    return MPFA_ERR_INVALID;
  if (a->batch > 65535) return MPFA_ERR_UNSUPPORTED;
  if (stats) {
    size_t need = 0;
    if (mpfa_kv4_write_workspace_size(a->batch, a->total_tokens, a->h_kv, &need) != MPFA_OK) return MPFA_ERR_INVALID;
    if (!workspace || workspace_bytes < need || !aligned16(workspace)) return MPFA_ERR_WORKSPACE;
  }
  mpfa::Kv4WriteParams p{};
  p.batch = a->batch;
  p.total_tokens = a->total_tokens;
  p.max_seqlen = a->max_seqlen;
  p.h_kv = a->h_kv;
  p.smooth = smooth;
  p.compute_stats = stats;
  p.num_pages = a->cache.num_pages;
  p.k_stride = a->k_stride;
  p.v_stride = a->v_stride;
  p.cu_seqlens = a->cu_seqlens;
  p.k = static_cast<const uint16_t*>(a->k);
  p.v = static_cast<const uint16_t*>(a->v);
  p.slot_mapping = a->slot_mapping;
  p.k_mean = static_cast<uint16_t*>(a->k_mean);
  p.k_tscale = a->k_tscale;
  p.v_tscale = a->v_tscale;
  p.cache = planes(a->cache);
  p.k_out = static_cast<uint16_t*>(a->k_out);
  p.v_out = static_cast<uint16_t*>(a->v_out);
  p.ws = static_cast<uint8_t*>(workspace);
#ifdef MPFA_DEBUG_CHECKS
  if (const mpfa_status st = check_write(a, reinterpret_cast<hipStream_t>(stream))) return st;
#endif
  return done(mpfa::launch_kv4_write(p, reinterpret_cast<hipStream_t>(stream)));
}

mpfa_status mpfa_kv4_prefill_plan(int32_t batch, const int32_t* rows_host, const int32_t* kv_len_host, int32_t h_q, int32_t h_kv,
                                  int32_t window, int32_t sinks, int32_t num_cus, int32_t* partition_tokens,
                                  int32_t* max_partitions, size_t* workspace_bytes) {
  if (batch < 1 || batch > 65535 || !rows_host || !kv_len_host || !kv_heads_ok(h_kv) || h_q < 1 || h_q > MPFA_MAX_HEADS || h_q % h_kv ||
      window < 0 || sinks < 0 || num_cus < 1 || !partition_tokens || !max_partitions || !workspace_bytes)
    return MPFA_ERR_INVALID;
  const int tm = mpfa::kKv4Rows / (h_q / h_kv);
  int64_t items = 0, tiles = 0, most = 0, total_rows = 0, max_rows = 0;
  for (int b = 0; b < batch; ++b) {
    if (rows_host[b] < 0 || rows_host[b] > kv_len_host[b]) return MPFA_ERR_INVALID;
    const int64_t n = rows_host[b], start = (int64_t)kv_len_host[b] - n;
    total_rows += n;
    max_rows = std::max(max_rows, n);
    for (int64_t t = 0; t < n; t += tm) {
      const int64_t nt = seen_tiles(start + t, start + std::min(t + tm, n) - 1, window, sinks);
      items += h_kv;
      tiles += nt * h_kv;
      most = std::max(most, nt);
    }
  }
  *partition_tokens = *max_partitions = 0;
  *workspace_bytes = 0;
  // One workgroup fills a compute unit.  Items are split where they leave units idle
  // and the longest of them is much longer than a unit's share of all tiles.
  const int64_t share = (tiles + num_cus - 1) / num_cus;
  if (items == 0 || max_rows > 65535 || 2 * share + 2 >= most) return MPFA_OK;
  const int64_t part = std::max<int64_t>(share, 4);
  const int64_t parts = (most + part - 1) / part;
  *partition_tokens = (int32_t)(part * MPFA_KV_TILE);
  *max_partitions = (int32_t)parts;
  *workspace_bytes = (size_t)total_rows * h_q * parts * mpfa::kKv4State * sizeof(float);
  return MPFA_OK;
}

mpfa_status mpfa_kv4_prefill(const mpfa_kv4_attn_args* a, void* workspace, size_t workspace_bytes, mpfa_stream_t stream) {
  mpfa::Kv4AttnParams p;
  if (const mpfa_status st = attn_params(a, p)) return st;
  if (a->q_tokens != 0 || a->max_seqlen_q < 0 || a->total_tokens < 0 || a->flags) return MPFA_ERR_INVALID;
  if (a->total_tokens == 0) return MPFA_OK;
  if (!a->cu_seqlens_q || !a->q_start) return MPFA_ERR_INVALID;
  p.max_seqlen_q = a->max_seqlen_q;
  const int tm = mpfa::kKv4Rows / (a->h_q / a->h_kv);
  const int64_t items = ((int64_t)a->max_seqlen_q + tm - 1) / tm * a->h_kv * a->batch;
  if (p.partition_tiles) {
    if (a->max_partitions < 1) return MPFA_ERR_INVALID;
    if (a->max_seqlen_q > 65535) return MPFA_ERR_UNSUPPORTED;
    const double need = (double)a->total_tokens * a->h_q * a->max_partitions * mpfa::kKv4State * sizeof(float);
    if (!workspace || (double)workspace_bytes < need || !aligned16(workspace)) return MPFA_ERR_WORKSPACE;
    p.states = static_cast<float*>(workspace);
  }
  if (items * (p.partition_tiles ? a->max_partitions : 1) > (int64_t)UINT32_MAX / 512) return MPFA_ERR_UNSUPPORTED;
#ifdef MPFA_DEBUG_CHECKS
  if (const mpfa_status st = check_attn(a, false, reinterpret_cast<hipStream_t>(stream))) return st;
#endif
  return done(mpfa::launch_kv4_prefill(p, reinterpret_cast<hipStream_t>(stream)));
}

mpfa_status mpfa_kv4_decode_plan(int32_t batch, const int32_t* kv_len_host, int32_t h_q, int32_t h_kv, int32_t q_tokens,
                                 int32_t window, int32_t sinks, uint32_t flags, int32_t num_cus, int32_t* partition_tokens,
                                 int32_t* max_partitions, size_t* workspace_bytes) {
  if (batch < 1 || batch > 65535 || !kv_len_host || !kv_heads_ok(h_kv) || h_q < 1 || h_q > MPFA_MAX_HEADS || h_q % h_kv || q_tokens < 1 ||
      window < 0 || sinks < 0 || (flags & ~MPFA_KV4_WEIGHTS) || num_cus < 1 || !partition_tokens || !max_partitions ||
      !workspace_bytes)
    return MPFA_ERR_INVALID;
  const int64_t chunks = ((int64_t)q_tokens * (h_q / h_kv) + 15) / 16;
  auto seen = [&](int b) {
    return seen_tiles((int64_t)kv_len_host[b] - q_tokens, (int64_t)kv_len_host[b] - 1, window, sinks);
  };
  int64_t most = 1;
  for (int b = 0; b < batch; ++b) {
    if (kv_len_host[b] < 0) return MPFA_ERR_INVALID;
    most = std::max(most, seen(b));
  }
  // A workgroup holds four partitions (waves) of a KV head.  The units of the card take
  // equally many workgroups, rounded up, of `part` tiles and about one tile's time to start
  // and store each: the smallest such sum wins.  (32 contexts of 16K to 64K keys, 32:8 heads:
  // 10 tiles 222 us, 12 tiles, with a last round of few, 260; 4 of 32K: 8 tiles 35 us, 5
  // tiles 40, 2 tiles 46; one of 64K, 40:8: 4 tiles 25.5, 3 tiles 32; 64 of 2100: 5 tiles
  // 38.8, 10 tiles 41.9.)
  int64_t part = 1, best = INT64_MAX;
  for (int64_t t = 1; t <= 128; ++t) {
    int64_t groups = 0;
    for (int b = 0; b < batch; ++b) groups += ((seen(b) + t - 1) / t * chunks + 3) / 4 * h_kv;
    const int64_t cost = (groups + num_cus - 1) / num_cus * (t + 1);
    if (cost < best) {
      best = cost;
      part = t;
    }
    if (t >= most) break;   // one partition each: longer ones change nothing
  }
  const int64_t parts = (most + part - 1) / part;
  DecodeSpace s;
  if (!decode_space(batch, h_q, q_tokens, (int)part * MPFA_KV_TILE, (int)parts, flags & MPFA_KV4_WEIGHTS, &s)) return MPFA_ERR_INVALID;
  *partition_tokens = (int32_t)(part * MPFA_KV_TILE);
  *max_partitions = (int32_t)parts;
  *workspace_bytes = s.states + s.stats + s.scores;
  return MPFA_OK;
}

mpfa_status mpfa_kv4_decode(const mpfa_kv4_attn_args* a, void* workspace, size_t workspace_bytes, mpfa_stream_t stream) {
  mpfa::Kv4AttnParams p;
  if (const mpfa_status st = attn_params(a, p)) return st;
  const bool weights = a->flags & MPFA_KV4_WEIGHTS;
  if (a->flags & ~MPFA_KV4_WEIGHTS) return MPFA_ERR_INVALID;
  if (a->q_tokens < 1 || a->q_tokens > 65535 || a->partition_tokens < 1 || a->max_partitions < 1) return MPFA_ERR_INVALID;
  if (weights && !a->cache.weights) return MPFA_ERR_INVALID;
  p.q_tokens = a->q_tokens;
  const int64_t chunks = ((int64_t)a->q_tokens * (a->h_q / a->h_kv) + 15) / 16;
  if (chunks * a->h_kv > 65535) return MPFA_ERR_UNSUPPORTED;
  if ((int64_t)a->max_partitions * a->partition_tokens > ((int64_t)1 << 30)) return MPFA_ERR_UNSUPPORTED;
  DecodeSpace s;
  if (!decode_space(a->batch, a->h_q, a->q_tokens, a->partition_tokens, a->max_partitions, weights, &s)) return MPFA_ERR_INVALID;
  if (!workspace || workspace_bytes < s.states + s.stats + s.scores || !aligned16(workspace)) return MPFA_ERR_WORKSPACE;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  p.states = reinterpret_cast<float*>(ws);
  if (weights) {
    p.stats = reinterpret_cast<float*>(ws + s.states);
    p.scores = reinterpret_cast<float*>(ws + s.states + s.stats);
  }
#ifdef MPFA_DEBUG_CHECKS
  if (const mpfa_status st = check_attn(a, true, reinterpret_cast<hipStream_t>(stream))) return st;
#endif
  return done(mpfa::launch_kv4_decode(p, reinterpret_cast<hipStream_t>(stream)));
}

mpfa_status mpfa_kv4_evict(const mpfa_kv4_evict_args* a, mpfa_stream_t stream) {
  if (!a) return MPFA_ERR_INVALID;
  if (a->batch < 1 || a->max_pages < 1 || a->dst_max_pages < 1 || !kv_heads_ok(a->h_kv)) return MPFA_ERR_INVALID;
  if (a->max_pages > INT32_MAX / MPFA_PAGE_TOKENS || a->dst_max_pages > INT32_MAX / MPFA_PAGE_TOKENS) return MPFA_ERR_INVALID;
  if (a->flags & ~MPFA_KV4_IN_PLACE) return MPFA_ERR_INVALID;
  if (a->budget < 1 || a->sinks < 0 || a->recent < 0 || (int64_t)a->sinks + a->recent > a->budget) return MPFA_ERR_INVALID;
  if (!cache_ok(a->cache) || !a->cache.weights || !a->kv_len || !a->page_table || !a->dst_page_table || !a->kept || !a->new_len)
    return MPFA_ERR_INVALID;
  if (a->batch > 65535) return MPFA_ERR_UNSUPPORTED;
  mpfa::Kv4EvictParams p{};
  p.batch = a->batch;
  p.h_kv = a->h_kv;
  p.max_pages = a->max_pages;
  p.dst_max_pages = a->dst_max_pages;
  p.budget = a->budget;
  p.sinks = a->sinks;
  p.recent = a->recent;
  p.in_place = (a->flags & MPFA_KV4_IN_PLACE) != 0;
  p.kv_len = a->kv_len;
  p.page_table = a->page_table;
  p.dst_page_table = a->dst_page_table;
  p.cache = planes(a->cache);
  p.kept = a->kept;
  p.new_len = a->new_len;
#ifdef MPFA_DEBUG_CHECKS
  if (const mpfa_status st = check_evict(a, reinterpret_cast<hipStream_t>(stream))) return st;
#endif
  return done(mpfa::launch_kv4_evict(p, reinterpret_cast<hipStream_t>(stream)));
}

}  // extern "C"
