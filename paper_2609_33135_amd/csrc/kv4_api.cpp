// kv4_api.cpp -- the C ABI of the 4-bit cache (include/mpfa.h): host-side validation (no
// HIP call before an argument set is accepted), workspace sizes and partition policies.
#include "mpfa.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <new>

#include "kv4_internal.h"

#ifdef MPFA_DEBUG_CHECKS
#include <vector>

#include "mpfa_internal.h"
#endif

namespace {

constexpr int kMaxKvHeads = 32;
constexpr int kFar = 1 << 30;   // windows and sinks from here on see every key there can be
constexpr float kLambda = 0.12751743074173085f;   // log2(e) / sqrt(128)
constexpr int kMostTokens = 1 << 28;   // of one call: its grids stay below 2^32 threads
constexpr int64_t kMergeTiles = 2;   // time of a decode's second launch, in tiles
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

// Bytes of the two parts of a decode workspace: partition states, then with weights the
// scores.  False where a size does not fit.
struct DecodeSpace {
  size_t states, scores;
};
bool decode_space(int batch, int h_q, int q_tokens, int partition_tokens, int max_partitions, bool weights, DecodeSpace* s) {
  const double rows = (double)batch * q_tokens * h_q;
  const double keys = (double)max_partitions * partition_tokens;
  if (rows * max_partitions * mpfa::kKv4State * 4 + (weights ? rows * keys * 4 : 0) > 9e18) return false;
  const size_t r = (size_t)batch * q_tokens * h_q;
  s->states = align256(r * max_partitions * mpfa::kKv4State * sizeof(float));
  s->scores = weights ? r * (size_t)max_partitions * partition_tokens * sizeof(float) : 0;
  return true;
}

// Whether a decode's grids stay below 2^32 threads, and its keys within the lengths there can be:
// partitions times column chunks, and with weights a workgroup per kKv4WeightKeys keys of a KV
// head beside one per row at most.
bool decode_grids_ok(int h_q, int h_kv, int q_tokens, int64_t partition_tokens, int64_t max_partitions, bool weights) {
  const int64_t cols = (int64_t)q_tokens * (h_q / h_kv), keys = max_partitions * partition_tokens;
  if (max_partitions * ((cols + 15) / 16) > (1 << 24) || keys > ((int64_t)1 << 30)) return false;
  return !weights || (int64_t)q_tokens * h_q + (keys + mpfa::kKv4WeightKeys - 1) / mpfa::kKv4WeightKeys * h_kv <= (int64_t)UINT32_MAX / 256;
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

// Most tiles that the last `q_tokens` of any sequence of at most kv_len keys see: with a
// window a shorter sequence may lie across one tile more.
int64_t most_tiles(int64_t kv_len, int64_t q_tokens, int window, int sinks) {
  const int64_t all = (kv_len + 127) / 128;
  if (window == 0) return all;
  const int64_t span = (int64_t)far(window) + q_tokens - 1;   // keys of the window
  return std::min(all, (std::min<int64_t>(sinks, kv_len) + 127) / 128 + (span + 254) / 128);
}

// ---- prefill plans
// tokens per item of 256 rows, or of 128; 0 where a token's heads do not fit
int item_tokens(int grp, int half) { return (half ? mpfa::kKv4Rows / 2 : mpfa::kKv4Rows) / grp; }

// of one part of an item, over the KV heads
size_t state_bytes(int h_kv, int half) {
  return (size_t)(half ? mpfa::kKv4Rows / 2 : mpfa::kKv4Rows) * h_kv * mpfa::kKv4State * sizeof(float);
}

struct PlanBlock {
  int32_t seq, row, tiles;
};

// Which blocks are cut: those longer than `most` tiles into equal parts of at most that
// (0: none), and the last `tail` ones in the order into `ways` parts; with its pieces, the
// number of blocks cut, and its estimated time in tiles.
struct PlanCut {
  float cost;
  int most, tail, ways;
  int64_t pieces, cut;
};

int parts_of(int tiles, int64_t i, int64_t n, const PlanCut& c) {
  int parts = c.most > 0 ? (tiles + c.most - 1) / c.most : 1;
  if (i >= n - c.tail) parts = std::max(parts, c.ways);
  return std::max(1, std::min(parts, tiles));
}

// Estimated time of a cut, in the time of one tile of a 256-row item (3.3 us): a piece takes
// its tiles (0.55 for 128 rows) and about 1.5 to start and store; the units take the pieces
// in order as they come free; a merge adds its launch and the states' bytes, 133 KB per
// piece and KV head written and read at 5 TB/s.
void price(const PlanBlock* s, int64_t n, int64_t units, int h_kv, int half, float* ends, PlanCut* c) {
  const float tile = half ? 0.55f : 1.0f, start = 1.5f;
  std::fill(ends, ends + units, 0.0f);   // a heap, the earliest end on top
  auto later = [](float x, float y) { return x > y; };
  float last = 0.0f;
  int64_t states = 0;
  c->pieces = c->cut = 0;
  for (int64_t i = 0; i < n; ++i) {
    const int parts = parts_of(s[i].tiles, i, n, *c);
    const float len = start + tile * s[i].tiles / parts;
    for (int k = 0; k < parts; ++k) {
      std::pop_heap(ends, ends + units, later);
      last = std::max(last, ends[units - 1] += len);
      std::push_heap(ends, ends + units, later);
    }
    c->pieces += parts;
    if (parts > 1) {
      ++c->cut;
      states += parts;
    }
  }
  c->cost = last;
  if (c->cut) c->cost += 1.2f + 0.016f * (half ? 0.5f : 1.0f) * states * h_kv;
}

PlanCut choose_cut(const PlanBlock* s, int64_t n, int64_t units, int h_kv, int half, float* ends) {
  PlanCut best = {0.0f, 0, 0, 0, 0, 0};
  price(s, n, units, h_kv, half, ends, &best);
  if (n > 16 * units) return best;   // many blocks per unit balance themselves
  auto consider = [&](PlanCut c) {
    price(s, n, units, h_kv, half, ends, &c);
    if (c.cost < best.cost) best = c;
  };
  const int longest = s[0].tiles, rest = (int)(n % units);
  for (int k = 2; k <= 64 && k <= longest; k += k / 2)   // 2, 3, 4, 6, 9, 13, ..
    if (n * k <= 24 * units || n <= units) consider({0.0f, std::max(1, (longest + k - 1) / k), 0, 0, 0, 0});
  for (int ways = 2; ways <= 8 && rest > 0 && n > units; ways += ways / 2) consider({0.0f, 0, rest, ways, 0, 0});
  return best;
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
  if (!to_host(a->cu_seqlens, (size_t)a->batch + 1, cu)) return MPFA_ERR_HIP;
  if (cu[0] != 0 || cu[a->batch] > a->total_tokens) return MPFA_ERR_DATA;
  for (int b = 0; b < a->batch; ++b)
    if (cu[b + 1] < cu[b] || cu[b + 1] - cu[b] > a->max_seqlen) return MPFA_ERR_DATA;
  const int64_t tokens = cu[a->batch];   // the rest is padding
  if (!to_host(a->slot_mapping, (size_t)tokens, slots)) return MPFA_ERR_HIP;
  std::sort(slots.begin(), slots.end());
  for (size_t i = 0; i < slots.size(); ++i)   // negative: padding
    if (slots[i] >= 64 * a->cache.num_pages || (i > 0 && slots[i] >= 0 && slots[i] == slots[i - 1])) return MPFA_ERR_DATA;
  mpfa_status st = scan_rows(a->k, tokens, (int64_t)a->h_kv * MPFA_HEAD_DIM, a->k_stride, s);
  if (st == MPFA_OK) st = scan_rows(a->v, tokens, (int64_t)a->h_kv * MPFA_HEAD_DIM, a->v_stride, s);
  return st;
}

mpfa_status check_attn(const mpfa_kv4_attn_args* a, bool decode, hipStream_t s) {
  if (hipStreamSynchronize(s) != hipSuccess) return MPFA_ERR_HIP;
  std::vector<int32_t> cu, qs, kv, pt;
  std::vector<mpfa_kv4_item> items;
  if (!to_host(a->kv_len, (size_t)a->batch, kv) || !to_host(a->page_table, (size_t)a->batch * a->max_pages, pt)) return MPFA_ERR_HIP;
  if (!decode && (!to_host(a->cu_seqlens_q, (size_t)a->batch + 1, cu) || !to_host(a->q_start, (size_t)a->batch, qs) ||
                  (a->items && !to_host(a->items, (size_t)a->n_items + a->n_merges, items))))
    return MPFA_ERR_HIP;
  std::vector<uint8_t> used;   // pages whose weights the call adds to
  if (decode && (a->flags & MPFA_KV4_WEIGHTS)) used.assign((size_t)a->cache.num_pages, 0);
  for (int b = 0; b < a->batch; ++b) {
    if (kv[b] < 0 || !row_pages_ok(pt, b, a->max_pages, ((int64_t)kv[b] + 63) / 64, a->cache.num_pages)) return MPFA_ERR_DATA;
    for (int64_t i = 0; !used.empty() && i < ((int64_t)kv[b] + 63) / 64; ++i)
      if (used[pt[(size_t)b * a->max_pages + i]]++) return MPFA_ERR_DATA;
    if (decode) {
      const int64_t room = (int64_t)a->max_partitions * (a->partition_tokens / MPFA_KV_TILE);
      if (seen_tiles((int64_t)kv[b] - a->q_tokens, kv[b] - 1, a->window, a->sinks) > room) return MPFA_ERR_DATA;
      continue;
    }
    const int n = cu[b + 1] - cu[b];
    if (n < 0 || n > a->max_seqlen_q || qs[b] < 0 || (int64_t)qs[b] + n > kv[b]) return MPFA_ERR_DATA;
  }
  if (!decode && (cu[0] != 0 || cu[a->batch] > a->total_tokens)) return MPFA_ERR_DATA;
  if (!items.empty()) {   // every block once, with all the tiles that it sees, its states inside the workspace
    const int tm = item_tokens(a->h_q / a->h_kv, a->half);
    const int64_t room = a->n_states;
    int64_t seen = 0, planned = 0, blocks = 0;
    for (int b = 0; b < a->batch; ++b)
      for (int t = 0; t < cu[b + 1] - cu[b]; t += tm, ++blocks)
        seen += seen_tiles(qs[b] + t, qs[b] + std::min(t + tm, cu[b + 1] - cu[b]) - 1, a->window, a->sinks);
    for (int i = 0; i < a->n_items + a->n_merges; ++i) {
      const mpfa_kv4_item& x = items[i];
      if (x.seq < 0 || x.seq >= a->batch || x.row < 0 || x.row % tm || x.row >= cu[x.seq + 1] - cu[x.seq]) return MPFA_ERR_DATA;
      const int n = cu[x.seq + 1] - cu[x.seq], nt =
          (int)seen_tiles(qs[x.seq] + x.row, qs[x.seq] + std::min(x.row + tm, n) - 1, a->window, a->sinks);
      if (x.first < 0 || x.first >= x.last || x.last > nt || x.parts < 1) return MPFA_ERR_DATA;
      if (x.parts > 1 ? x.state < 0 || x.state + (i < a->n_items ? 1 : x.parts) > room : x.state != -1) return MPFA_ERR_DATA;
      if (i < a->n_items) {
        planned += x.last - x.first;
        blocks -= x.parts == 1;
      } else {
        --blocks;
      }
    }
    if (seen != planned || blocks != 0) return MPFA_ERR_DATA;
  }
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
  if (a->batch > 65535 || a->total_tokens > kMostTokens) return MPFA_ERR_UNSUPPORTED;
  const int64_t groups = (std::min(a->max_seqlen, a->total_tokens) + mpfa::kKv4WriteTokens - 1) / mpfa::kKv4WriteTokens;
  if (groups * a->h_kv > (int64_t)UINT32_MAX / 256) return MPFA_ERR_UNSUPPORTED;
  if (stats) {
    size_t need = 0;
    if (mpfa_kv4_write_workspace_size(a->batch, a->total_tokens, a->h_kv, &need) != MPFA_OK) return MPFA_ERR_INVALID;
    if (!workspace || workspace_bytes < need || !aligned16(workspace)) return MPFA_ERR_WORKSPACE;
  }
  mpfa::Kv4WriteParams p{};
  p.batch = a->batch;
  p.total_tokens = a->total_tokens;
  p.max_seqlen = std::min(a->max_seqlen, a->total_tokens);
  p.h_kv = a->h_kv;
  p.smooth = smooth;
  p.compute_stats = stats;
  // from 32768 tokens on 512 per partial: workgroups enough, and a quarter of the partials
  p.stat_tokens = a->total_tokens >= 32768 ? 4 * mpfa::kKv4StatTokens : mpfa::kKv4StatTokens;
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
                                  int32_t window, int32_t sinks, int32_t num_cus, mpfa_kv4_item* items, int32_t capacity,
                                  int32_t* n_items, int32_t* n_merges, int32_t* n_states, int32_t* half,
                                  size_t* workspace_bytes) {
  if (batch < 1 || batch > 65535 || !rows_host || !kv_len_host || !kv_heads_ok(h_kv) || h_q < 1 || h_q > MPFA_MAX_HEADS ||
      h_q % h_kv || window < 0 || sinks < 0 || num_cus < 1 || capacity < 0 || !n_items || !n_merges || !n_states || !half ||
      !workspace_bytes)
    return MPFA_ERR_INVALID;
  const int grp = h_q / h_kv;
  int64_t blocks[2] = {0, 0};
  for (int b = 0; b < batch; ++b) {
    if (rows_host[b] < 0 || rows_host[b] > kv_len_host[b]) return MPFA_ERR_INVALID;
    for (int h = 0; h < 2; ++h)
      if (const int tm = item_tokens(grp, h)) blocks[h] += ((int64_t)rows_host[b] + tm - 1) / tm;
  }
  *n_items = *n_merges = *n_states = *half = 0;
  *workspace_bytes = 0;
  if (blocks[0] == 0) return MPFA_OK;
  if (blocks[1] > INT32_MAX / 64) return MPFA_ERR_UNSUPPORTED;

  // Blocks of either size, longest first; per size the cut that finishes first.
  const int64_t units = std::max(1, num_cus / h_kv);   // every unit stands for the KV heads of a block
  PlanBlock* sorted[2] = {nullptr, nullptr};
  float* ends = new (std::nothrow) float[units];
  PlanCut best = {1e30f, 0, 0, 0, 0, 0};
  int best_half = 0;
  bool ok = ends != nullptr;
  for (int h = 0; h < 2 && ok; ++h) {
    const int tm = item_tokens(grp, h);
    // halves pay where the card has units for them all, or nearly
    if (tm == 0 || (h == 1 && blocks[1] > 4 * units)) continue;
    PlanBlock* s = sorted[h] = new (std::nothrow) PlanBlock[blocks[h]];
    if (!s) {
      ok = false;
      break;
    }
    int64_t n = 0;
    for (int b = 0; b < batch; ++b)
      for (int64_t t = 0; t < rows_host[b]; t += tm) {
        const int64_t start = (int64_t)kv_len_host[b] - rows_host[b];
        s[n++] = {b, (int32_t)t,
                  (int32_t)seen_tiles(start + t, start + std::min<int64_t>(t + tm, rows_host[b]) - 1, window, sinks)};
      }
    std::sort(s, s + n, [](const PlanBlock& x, const PlanBlock& y) {
      return x.tiles != y.tiles ? x.tiles > y.tiles : x.seq != y.seq ? x.seq < y.seq : x.row > y.row;
    });
    const PlanCut c = choose_cut(s, n, units, h_kv, h, ends);
    if (c.cost < best.cost) {
      best = c;
      best_half = h;
    }
  }
  mpfa_status st = ok ? MPFA_OK : MPFA_ERR_WORKSPACE;
  if (ok) {
    const PlanBlock* s = sorted[best_half];
    const int64_t n = blocks[best_half];
    *n_items = (int32_t)best.pieces;
    *n_merges = (int32_t)best.cut;
    *half = best_half;
    *n_states = (int32_t)(best.pieces - (n - best.cut));
    *workspace_bytes = *n_states * state_bytes(h_kv, best_half);
    if (items) {
      if (capacity < best.pieces + best.cut) {
        st = MPFA_ERR_WORKSPACE;
      } else {
        int64_t at = 0, state = 0, merge = best.pieces;
        for (int64_t i = 0; i < n; ++i) {
          const int parts = parts_of(s[i].tiles, i, n, best);
          if (parts > 1) items[merge++] = {s[i].seq, s[i].row, 0, s[i].tiles, (int32_t)state, parts};
          for (int k = 0; k < parts; ++k)
            items[at++] = {s[i].seq, s[i].row, (int32_t)((int64_t)s[i].tiles * k / parts),
                           (int32_t)((int64_t)s[i].tiles * (k + 1) / parts), parts > 1 ? (int32_t)(state + k) : -1, parts};
          if (parts > 1) state += parts;
        }
        // longest first: the card takes them in this order
        std::sort(items, items + best.pieces, [](const mpfa_kv4_item& x, const mpfa_kv4_item& y) {
          const int a = x.last - x.first, b = y.last - y.first;
          return a != b ? a > b : x.seq != y.seq ? x.seq < y.seq : x.row != y.row ? x.row > y.row : x.first > y.first;
        });
      }
    }
  }
  delete[] sorted[0];
  delete[] sorted[1];
  delete[] ends;
  return st;
}

mpfa_status mpfa_kv4_prefill(const mpfa_kv4_attn_args* a, void* workspace, size_t workspace_bytes, mpfa_stream_t stream) {
  mpfa::Kv4AttnParams p;
  if (const mpfa_status st = attn_params(a, p)) return st;
  if (a->q_tokens != 0 || a->max_seqlen_q < 0 || a->total_tokens < 0 || a->flags) return MPFA_ERR_INVALID;
  if (a->total_tokens == 0) return MPFA_OK;
  if (!a->cu_seqlens_q || !a->q_start) return MPFA_ERR_INVALID;
  if (a->total_tokens > kMostTokens) return MPFA_ERR_UNSUPPORTED;
  p.max_seqlen_q = std::min(a->max_seqlen_q, a->total_tokens);
  if (a->items) {
    if (a->n_items < 1 || a->n_merges < 0 || a->n_merges > a->n_items || a->n_states < 0 || a->n_states > a->n_items ||
        (a->half != 0 && a->half != 1))
      return MPFA_ERR_INVALID;
    if (a->half && item_tokens(a->h_q / a->h_kv, 1) == 0) return MPFA_ERR_INVALID;
    if (a->n_merges > 65535 || (int64_t)a->n_items * a->h_kv > (int64_t)UINT32_MAX / 512) return MPFA_ERR_UNSUPPORTED;
    if (a->n_states > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < a->n_states * state_bytes(a->h_kv, a->half)))
      return MPFA_ERR_WORKSPACE;
    p.items = a->items;
    p.n_items = a->n_items;
    p.n_merges = a->n_merges;
    p.half = a->half;
    p.states = static_cast<float*>(workspace);
  } else {
    const int tm = item_tokens(a->h_q / a->h_kv, 0);
    const int64_t items = ((int64_t)p.max_seqlen_q + tm - 1) / tm * a->h_kv * a->batch;
    if (items > (int64_t)UINT32_MAX / 512) return MPFA_ERR_UNSUPPORTED;
  }
#ifdef MPFA_DEBUG_CHECKS
  if (const mpfa_status st = check_attn(a, false, reinterpret_cast<hipStream_t>(stream))) return st;
#endif
  return done(mpfa::launch_kv4_prefill(p, reinterpret_cast<hipStream_t>(stream)));
}

mpfa_status mpfa_kv4_decode_plan(int32_t batch, const int32_t* kv_len_host, int32_t h_q, int32_t h_kv, int32_t q_tokens,
                                 int32_t window, int32_t sinks, uint32_t flags, int32_t num_cus, int32_t* partition_tokens,
                                 int32_t* max_partitions, size_t* workspace_bytes) {
  if (batch < 1 || batch > 65535 || !kv_len_host || !kv_heads_ok(h_kv) || h_q < 1 || h_q > MPFA_MAX_HEADS || h_q % h_kv || q_tokens < 1 ||
      q_tokens > 65535 || window < 0 || sinks < 0 || (flags & ~MPFA_KV4_WEIGHTS) || num_cus < 1 || !partition_tokens || !max_partitions ||
      !workspace_bytes)
    return MPFA_ERR_INVALID;
  const int64_t cols = (int64_t)q_tokens * (h_q / h_kv), per = mpfa::kv4_wide_columns(cols) ? 32 : 16;
  const int64_t chunks = (cols + per - 1) / per;
  auto seen = [&](int b) {
    return seen_tiles((int64_t)kv_len_host[b] - q_tokens, (int64_t)kv_len_host[b] - 1, window, sinks);
  };
  int64_t most = 1, bound = 1;
  for (int b = 0; b < batch; ++b) {
    if (kv_len_host[b] < 0) return MPFA_ERR_INVALID;
    most = std::max(most, seen(b));
    bound = std::max(bound, most_tiles(kv_len_host[b], q_tokens, window, sinks));
  }
  if ((double)batch * most * chunks * h_kv > 1e15) return MPFA_ERR_INVALID;   // no workspace is as large
  // A workgroup holds four partitions (waves) of a KV head.  The units of the card take
  // equally many workgroups, rounded up, of `part` tiles and about one tile's time to start
  // and store each; where a row has more than four there is a launch that merges them: the
  // smallest such sum wins.  (32 contexts of 16K to 64K keys, 32:8 heads:
  // 10 tiles 222 us, 12 tiles, with a last round of few, 260; 4 of 32K: 8 tiles 35 us, 5
  // tiles 40, 2 tiles 46; one of 64K, 40:8: 4 tiles 25.5, 3 tiles 32; one of 1000 or eight:
  // 2 tiles, four partitions, 9.2 and 9.9, 1 tile 11.3 and 11.1; 16 of 2000: 2 tiles 13.8, 4
  // tiles, without the merge, 15.0.)
  int64_t part = 1, best = INT64_MAX;
  for (int64_t t = 1; t <= 128; ++t) {
    int64_t groups = 0;
    for (int b = 0; b < batch; ++b) groups += ((seen(b) + t - 1) / t * chunks + 3) / 4 * h_kv;
    const int64_t cost = (groups + num_cus - 1) / num_cus * (t + 1) +
                         (mpfa::kv4_direct(chunks, (bound + t - 1) / t, flags & MPFA_KV4_WEIGHTS) ? 0 : kMergeTiles);
    if (cost < best) {
      best = cost;
      part = t;
    }
    if (t >= most) break;   // one partition each: longer ones change nothing
  }
  const int64_t parts = (bound + part - 1) / part;
  if (!decode_grids_ok(h_q, h_kv, q_tokens, part * MPFA_KV_TILE, parts, flags & MPFA_KV4_WEIGHTS)) return MPFA_ERR_UNSUPPORTED;
  DecodeSpace s;
  if (!decode_space(batch, h_q, q_tokens, (int)part * MPFA_KV_TILE, (int)parts, flags & MPFA_KV4_WEIGHTS, &s)) return MPFA_ERR_INVALID;
  *partition_tokens = (int32_t)(part * MPFA_KV_TILE);
  *max_partitions = (int32_t)parts;
  *workspace_bytes = s.states + s.scores;
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
  if (!decode_grids_ok(a->h_q, a->h_kv, a->q_tokens, a->partition_tokens, a->max_partitions, weights)) return MPFA_ERR_UNSUPPORTED;
  DecodeSpace s;
  if (!decode_space(a->batch, a->h_q, a->q_tokens, a->partition_tokens, a->max_partitions, weights, &s)) return MPFA_ERR_INVALID;
  if (!workspace || workspace_bytes < s.states + s.scores || !aligned16(workspace)) return MPFA_ERR_WORKSPACE;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  p.states = reinterpret_cast<float*>(ws);
  if (weights) p.scores = reinterpret_cast<float*>(ws + s.states);
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
