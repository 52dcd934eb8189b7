// linear_api.cpp -- the C ABI of linear attention and of the norm (include/mpfa.h): host-side
// validation (no HIP call before an argument set is accepted).
#include "mpfa.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "linear_internal.h"
#include "mpfa_internal.h"

#ifdef MPFA_DEBUG_CHECKS
#include <new>
#include <vector>
#endif

namespace {

constexpr int kMostTokens = 1 << 28;              // of one call
constexpr int kMostRows = 1024;                   // of one sequence in a decode call
constexpr int64_t kMaxStride = (int64_t)1 << 25;  // elements between tokens: 64 of them in 32 bits of bytes
constexpr int64_t kMaxRow = (int64_t)1 << 31;     // elements between rows of the norm
static_assert(mpfa::kLinUnits == mpfa::kComputeUnits, "by which prompts are cut");

bool aligned16(const void* x) { return (reinterpret_cast<uintptr_t>(x) & 15) == 0; }

bool stride_ok(int64_t stride, int heads) {
  return stride >= (int64_t)heads * MPFA_HEAD_DIM && stride % 8 == 0 && stride < kMaxStride;
}

bool heads_ok(int h_q, int h_kv) { return h_kv >= 1 && h_q >= 1 && h_q <= MPFA_MAX_HEADS && h_q % h_kv == 0; }

mpfa_status done(hipError_t e) { return e == hipSuccess ? MPFA_OK : MPFA_ERR_HIP; }

// What both calls check; fills what does not depend on the kind.
mpfa_status linear_params(const mpfa_linear_args* a, bool decode, mpfa::LinearParams& p) {
  if (!a) return MPFA_ERR_INVALID;
  if (a->head_dim != MPFA_HEAD_DIM) return a->head_dim > 0 ? MPFA_ERR_UNSUPPORTED : MPFA_ERR_INVALID;
  if (a->batch < 1 || a->batch > 65535 || !heads_ok(a->h_q, a->h_kv) || a->flags || !std::isfinite(a->scale) || a->num_states < 0)
    return MPFA_ERR_INVALID;
  if (decode ? a->q_tokens < 1 || a->q_tokens > kMostRows : a->total_tokens < 0 || a->max_seqlen < 0) return MPFA_ERR_INVALID;
  if (!stride_ok(a->q_stride, a->h_q) || !stride_ok(a->k_stride, a->h_kv) || !stride_ok(a->v_stride, a->h_kv)) return MPFA_ERR_INVALID;
  if (a->decay_stride != 0 && (a->decay_stride < a->h_kv || a->decay_stride >= kMaxStride)) return MPFA_ERR_INVALID;
  // without tokens only states move, and with no slot not even those
  const bool tokens = decode || a->total_tokens > 0;
  if (!a->state_src || !a->state_dst || (a->num_states > 0 && !a->states) || !aligned16(a->states)) return MPFA_ERR_INVALID;
  if (tokens && (!a->q || !a->k || !a->v || !a->log_decay || !a->out)) return MPFA_ERR_INVALID;
  if (!decode && !a->cu_seqlens) return MPFA_ERR_INVALID;
  if (!aligned16(a->q) || !aligned16(a->k) || !aligned16(a->v) || !aligned16(a->out)) return MPFA_ERR_INVALID;
  p = mpfa::LinearParams{};
  p.batch = a->batch;
  p.h_q = a->h_q;
  p.h_kv = a->h_kv;
  p.q_tokens = a->q_tokens;
  p.scale = a->scale;
  p.q_stride = a->q_stride;
  p.k_stride = a->k_stride;
  p.v_stride = a->v_stride;
  p.decay_stride = a->decay_stride;
  p.cu_seqlens = a->cu_seqlens;
  p.q = static_cast<const uint16_t*>(a->q);
  p.k = static_cast<const uint16_t*>(a->k);
  p.v = static_cast<const uint16_t*>(a->v);
  p.log_decay = a->log_decay;
  p.state_src = a->state_src;
  p.state_dst = a->state_dst;
  p.states = a->states;
  p.out = static_cast<uint16_t*>(a->out);
  return MPFA_OK;
}

#ifdef MPFA_DEBUG_CHECKS
template <typename T>
bool to_host(const T* dev, size_t n, std::vector<T>& out) {
  out.resize(n);
  return n == 0 || hipMemcpy(out.data(), dev, n * sizeof(T), hipMemcpyDeviceToHost) == hipSuccess;
}

// Index ranges, slots that two sequences would write or one write and another read, finite q, k and v,
// decays at most 0.
mpfa_status check_linear(const mpfa_linear_args* a, bool decode, hipStream_t s) try {
  if (hipStreamSynchronize(s) != hipSuccess) return MPFA_ERR_HIP;
  std::vector<int32_t> cu, src, dst;
  if (!to_host(a->state_src, (size_t)a->batch, src) || !to_host(a->state_dst, (size_t)a->batch, dst) ||
      (!decode && !to_host(a->cu_seqlens, (size_t)a->batch + 1, cu)))
    return MPFA_ERR_HIP;
  int64_t tokens = (int64_t)a->batch * a->q_tokens;
  if (!decode) {
    if (cu[0] != 0 || cu[a->batch] > a->total_tokens) return MPFA_ERR_DATA;
    for (int b = 0; b < a->batch; ++b)
      if (cu[b + 1] < cu[b] || cu[b + 1] - cu[b] > a->max_seqlen) return MPFA_ERR_DATA;
    tokens = cu[a->batch];
  }
  std::vector<int32_t> writer((size_t)a->num_states, -1);
  for (int b = 0; b < a->batch; ++b) {
    if (src[b] >= a->num_states || dst[b] >= a->num_states || (dst[b] >= 0 && writer[dst[b]] >= 0)) return MPFA_ERR_DATA;
    if (dst[b] >= 0) writer[dst[b]] = b;
  }
  for (int b = 0; b < a->batch; ++b)
    if (src[b] >= 0 && writer[src[b]] >= 0 && writer[src[b]] != b) return MPFA_ERR_DATA;
  if (tokens == 0) return MPFA_OK;
  int* flag = nullptr;
  if (hipMalloc(&flag, sizeof(int)) != hipSuccess) return MPFA_ERR_HIP;
  int h = 0;
  bool ok = hipMemsetAsync(flag, 0, sizeof(int), s) == hipSuccess;
  auto scan = [&](const void* x, int64_t row, int64_t stride) {
    const int64_t parts = stride == row ? 1 : tokens, n = stride == row ? tokens * row : row;
    for (int64_t t = 0; t < parts; ++t)
      ok = ok && mpfa::launch_scan_nonfinite(static_cast<const uint16_t*>(x) + t * stride, n, flag, s) == hipSuccess;
  };
  scan(a->q, (int64_t)a->h_q * MPFA_HEAD_DIM, a->q_stride);
  scan(a->k, (int64_t)a->h_kv * MPFA_HEAD_DIM, a->k_stride);
  scan(a->v, (int64_t)a->h_kv * MPFA_HEAD_DIM, a->v_stride);
  ok = ok && mpfa::launch_scan_decay(a->log_decay, a->decay_stride ? tokens : 1, a->h_kv, a->decay_stride, flag, s) == hipSuccess;
  ok = ok && hipMemcpyAsync(&h, flag, sizeof(int), hipMemcpyDeviceToHost, s) == hipSuccess && hipStreamSynchronize(s) == hipSuccess;
  (void)hipFree(flag);
  if (!ok) return MPFA_ERR_HIP;
  return h ? MPFA_ERR_DATA : MPFA_OK;
} catch (const std::bad_alloc&) {
  return MPFA_ERR_HIP;
}
#endif

}  // namespace

extern "C" {

mpfa_status mpfa_linear_prefill_workspace_size(int32_t batch, int32_t total_tokens, int32_t max_seqlen, int32_t h_q, int32_t h_kv,
                                               size_t* bytes) {
  if (!bytes || batch < 1 || batch > 65535 || total_tokens < 0 || max_seqlen < 0 || !heads_ok(h_q, h_kv)) return MPFA_ERR_INVALID;
  if (total_tokens > kMostTokens) return MPFA_ERR_UNSUPPORTED;
  *bytes = mpfa::linear_most_space(batch, total_tokens, max_seqlen, h_q, h_kv);
  return MPFA_OK;
}

mpfa_status mpfa_linear_prefill(const mpfa_linear_args* a, void* workspace, size_t workspace_bytes, mpfa_stream_t stream) {
  mpfa::LinearParams p;
  if (const mpfa_status st = linear_params(a, false, p)) return st;
  if (a->total_tokens > kMostTokens) return MPFA_ERR_UNSUPPORTED;
  const mpfa::LinearSpace s = mpfa::linear_space(a->batch, a->total_tokens, a->max_seqlen, a->h_q, a->h_kv);
  if (s.items > (int64_t)UINT32_MAX / 512 - 8) return MPFA_ERR_UNSUPPORTED;
  if (s.bytes && (!workspace || workspace_bytes < s.bytes || !aligned16(workspace))) return MPFA_ERR_WORKSPACE;
  p.segment = s.segment;
  p.split = s.split;
  p.parts = s.parts;
  p.heads = s.heads;
  p.items = (int)s.items;
  // what the longest sequence has to join, in one turn if four waves can; with one or two KV heads there are few
  // workgroups and long sequences (32768 tokens of 16:1 heads 102 us by four waves, 99 by sixteen; 4096 of 32:8 49.3
  // by four, 49.9 by eight)
  const int64_t places = std::min(a->max_seqlen, a->total_tokens) / s.segment;
  p.join_waves = (int)std::max<int64_t>(1, std::min<int64_t>((places + mpfa::kLinJoin - 1) / mpfa::kLinJoin, std::max(4, mpfa::kLinJoinWaves / a->h_kv)));
  p.starts = s.bytes ? static_cast<float*>(workspace) : nullptr;
  p.decays = s.bytes ? p.starts + s.starts / sizeof(float) : nullptr;
#ifdef MPFA_DEBUG_CHECKS
  if (const mpfa_status st = check_linear(a, false, reinterpret_cast<hipStream_t>(stream))) return st;
#endif
  return done(mpfa::launch_linear_prefill(p, reinterpret_cast<hipStream_t>(stream)));
}

mpfa_status mpfa_linear_decode(const mpfa_linear_args* a, mpfa_stream_t stream) {
  mpfa::LinearParams p;
  if (const mpfa_status st = linear_params(a, true, p)) return st;
  if ((int64_t)a->batch * a->h_kv * 4 > (int64_t)UINT32_MAX / 256) return MPFA_ERR_UNSUPPORTED;
#ifdef MPFA_DEBUG_CHECKS
  if (const mpfa_status st = check_linear(a, true, reinterpret_cast<hipStream_t>(stream))) return st;
#endif
  return done(mpfa::launch_linear_decode(p, reinterpret_cast<hipStream_t>(stream)));
}

mpfa_status mpfa_rms_norm(const mpfa_rms_norm_args* a, mpfa_stream_t stream) {
  if (!a || a->rows < 0 || a->width < 8 || a->width % 8) return MPFA_ERR_INVALID;
  if (!(a->eps > 0.0f) || !std::isfinite(a->eps)) return MPFA_ERR_INVALID;
  if (a->scales ? a->group != 0 && (a->group < 32 || a->group > 512 || (a->group & (a->group - 1))) : a->group != 0) return MPFA_ERR_INVALID;
  if (a->rows == 0) return MPFA_OK;
  if (a->x_stride < (a->rows > 1 ? a->width : 0) || a->x_stride % 8 || a->x_stride >= kMaxRow) return MPFA_ERR_INVALID;
  if (!a->x || !a->out || (a->residual != nullptr) != (a->residual_out != nullptr)) return MPFA_ERR_INVALID;
  if (!aligned16(a->x) || !aligned16(a->weight) || !aligned16(a->residual) || !aligned16(a->residual_out)) return MPFA_ERR_INVALID;
  if ((reinterpret_cast<uintptr_t>(a->out) & (a->scales ? 7 : 15)) || (reinterpret_cast<uintptr_t>(a->scales) & 3)) return MPFA_ERR_INVALID;
  if (a->width > mpfa::kNormWidth || (int64_t)a->rows * mpfa::norm_threads(a->width) >= (int64_t)UINT32_MAX - 256) return MPFA_ERR_UNSUPPORTED;
  mpfa::NormParams p{};
  p.rows = a->rows;
  p.width = a->width;
  p.group = a->group ? a->group : a->width;
  p.eps = a->eps;
  p.x_stride = a->x_stride;
  p.x = static_cast<const uint16_t*>(a->x);
  p.weight = static_cast<const uint16_t*>(a->weight);
  p.residual = static_cast<const uint16_t*>(a->residual);
  p.residual_out = static_cast<uint16_t*>(a->residual_out);
  p.out = a->out;
  p.scales = a->scales;
  return done(mpfa::launch_rms_norm(p, reinterpret_cast<hipStream_t>(stream)));
}

}  // extern "C"
