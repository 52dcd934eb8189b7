// linear_prefill.hip -- linear attention with a decay over packed prompts for gfx950.
//
// S_t = a_t S_{t-1} + k_t v_t^T, o_t = scale q_t^T S_t, a_t = exp(g_t).  With b_i the sum of g over the
// tokens of a chunk up to i and S the state before it,
//   o_i = scale (exp(b_i) q_i^T S + sum_{j <= i} exp(b_i - b_j) (q_i . k_j) v_j),
//   S'  = exp(b_last) S + sum_j exp(b_last - b_j) k_j v_j^T:
// four products of 64-token chunks on the matrix cores, every exponent <= 0.
//
// A sequence is cut into segments so that there is work for every unit: `sums` adds up each segment's own
// state, `join` makes the state before each segment out of those, `outputs` goes through the segments' chunks.
#include <algorithm>

#include "linear_internal.h"
#include "mpfa_device.h"

namespace mpfa {

namespace {

constexpr int kC = kLinChunk;
constexpr int kRow = kD + 8;          // elements of a token's row in LDS
constexpr double kLog2e = 1.4426950408889634;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

union Frag {   // an operand of eight values
  u32x4 w;
  u32x2 d[2];
  s16x4 s[2];
  bf16x8 b;
};

struct Segment {
  int b, s, count;        // sequence, segment of it, of so many
  int64_t t0;             // first token
  int n;                  // tokens
};

// Segment number id: the last sequence whose first number is at most id, by 64-ary search.
__device__ __forceinline__ bool find_segment(const LinearParams& p, int id, Segment* g) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = p.batch;
  while (n > 1) {
    const int step = (n + 63) >> 6, at = lane * step;
    const bool before = at < n && p.cu_seqlens[lo + min(at, n - 1)] / p.segment + lo + at <= id;
    const int last = __popcll(__builtin_amdgcn_ballot_w64(before)) - 1;
    lo += last * step;
    n = min(step, n - last * step);
  }
  const int begin = p.cu_seqlens[lo], len = p.cu_seqlens[lo + 1] - begin;
  g->b = lo;
  g->s = id - (begin / p.segment + lo);
  g->count = max(1, (len + p.segment - 1) / p.segment);
  g->t0 = (int64_t)begin + (int64_t)g->s * p.segment;
  g->n = min(p.segment, len - g->s * p.segment);
  return g->s < g->count;
}

struct Lds {
  uint16_t k[kC][kRow], v[kC][kRow], q[kC][kRow];
  u32x4 p[3][2][2][64];                        // scores: block, step of 16 keys, high and low parts, lane
  float hi[kC], lo[kC];                        // log2 of the decays from the chunk's start, in two parts
  float from[kC], to[kC];                      // exp2 of them; exp2 from each token to the chunk's end
};

// Four tokens (rows t .. t + 3) of the lane's column c0 + lane % 32, t = t0 + 4 * (lane / 32): each
// group of 16 lanes reads a block of four rows and 16 columns, and gets it transposed.
__device__ __forceinline__ s16x4 column4(const uint16_t (*rows)[kRow], int t0, int c0) {
  typedef __attribute__((address_space(3))) s16x4 lds4;
  const int lane = threadIdx.x & 63, i = lane & 15;
  const uint16_t* at = &rows[t0 + 4 * (lane >> 5) + (i >> 2)][c0 + (lane & 16) + 4 * (i & 3)];
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)at);
}
// The tokens of one 16-token step in the order in which an accumulator holds its rows.
__device__ __forceinline__ Frag columns(const uint16_t (*rows)[kRow], int t0, int c0) {
  Frag f;
  f.s[0] = column4(rows, t0, c0);
  f.s[1] = column4(rows, t0 + 8, c0);
  return f;
}

__device__ __forceinline__ float bits_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bits_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 r = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, r);
}
// Eight FP32 values as the sum of kParts BF16 operands.  Two lose at most 2^-16 of each value, little beside
// the rounding of an output to BF16; three 2^-24, as FP32 itself, for sums that stay in the state.
template <int kParts>
__device__ __forceinline__ void split8(float* x, Frag* part) {
#pragma unroll
  for (int i = 0; i < kParts; ++i)
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const uint32_t h = pack_bf16(x[e], x[e + 1]);
      part[i].w[e >> 1] = h;
      x[e] -= bits_lo(h);
      x[e + 1] -= bits_hi(h);
    }
}

// Rows t .. of a chunk, 16 lanes a row: four rows of each thread; zeros from row n on.
struct Rows {
  u32x4 w[4];
};
__device__ __forceinline__ void load_rows(Rows& r, const uint16_t* x, int64_t stride, int n) {
  const int row = threadIdx.x >> 4, c = threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r.w[i] = (u32x4){0, 0, 0, 0};
    if (row + 16 * i < n) r.w[i] = *reinterpret_cast<const u32x4*>(x + (row + 16 * i) * stride + 8 * c);
  }
}
__device__ __forceinline__ void store_rows(const Rows& r, uint16_t (*to)[kRow]) {
  const int row = threadIdx.x >> 4, c = threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<u32x4*>(&to[row + 16 * i][8 * c]) = r.w[i];
}

// The state's part of a wave: 32 columns (channels of v), accumulator db the rows (channels of k) 32 db ..
struct State {
  f32x16 a[4];
};
__device__ __forceinline__ int state_row(int db, int r) { return 32 * db + 8 * (r >> 2) + 4 * ((threadIdx.x & 63) >> 5) + (r & 3); }

__device__ __forceinline__ void state_zero(State& s) {
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) s.a[db][r] = 0.0f;
}
__device__ __forceinline__ void state_load(State& s, const float* from) {
  const int col = 32 * (threadIdx.x >> 6) + (threadIdx.x & 31);
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) s.a[db][r] = from[state_row(db, r) * kD + col];
}
__device__ __forceinline__ void state_store(const State& s, float* to) {
  const int col = 32 * (threadIdx.x >> 6) + (threadIdx.x & 31);
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) to[state_row(db, r) * kD + col] = s.a[db][r];
}
// In the workspace a state lies as the accumulators do.
__device__ __forceinline__ f32x4* raw_at(float* ws, int db, int r4) {
  return reinterpret_cast<f32x4*>(ws) + (((threadIdx.x >> 6) * 4 + db) * 4 + r4) * 64 + (threadIdx.x & 63);
}
__device__ __forceinline__ void raw_store(const State& s, float* ws) {
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4)
      *raw_at(ws, db, r4) = (f32x4){s.a[db][4 * r4], s.a[db][4 * r4 + 1], s.a[db][4 * r4 + 2], s.a[db][4 * r4 + 3]};
}
__device__ __forceinline__ void raw_load(State& s, float* ws) {
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const f32x4 x = *raw_at(ws, db, r4);
#pragma unroll
      for (int e = 0; e < 4; ++e) s.a[db][4 * r4 + e] = x[e];
    }
}

// log2 of the decay from the chunk's start to each token (lane = token).  Summed in 64 bits: after a token
// that clears the state, sums are large and their differences small.
__device__ __forceinline__ double decay_sums(const LinearParams& p, int64_t t, int n, int hk) {
  const int lane = threadIdx.x & 63;
  double x = 0.0;
  if (lane < n) x = (double)fminf(fmaxf(p.log_decay[(t + lane) * p.decay_stride + hk], kLinLeastDecay), 0.0f) * kLog2e;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

// One workgroup of four waves per (segment, KV head).  kOut: the outputs of its tokens from the state before
// it, and of a sequence's last segment the state after it; else the segment's own state, for the next.
template <bool kOut>
__global__ __launch_bounds__(256) void linear_chunks_kernel(LinearParams p) {
  __shared__ Lds s;
  const int hk = blockIdx.x % p.h_kv, id = blockIdx.x / p.h_kv;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, l32 = lane & 31;
  const int grp = p.h_q / p.h_kv;
  Segment g;
  if (!find_segment(p, id, &g)) return;
  const bool last = g.s == g.count - 1;
  if (!kOut && last) return;
  float* const slot = p.split ? p.starts + ((int64_t)id * p.h_kv + hk) * kLinState : nullptr;

  State st;
  state_zero(st);
  if (g.s == 0 && (!kOut || g.count == 1)) {
    const int src = p.state_src[g.b];
    if (src >= 0) state_load(st, p.states + ((int64_t)src * p.h_kv + hk) * kLinState);
    if (!kOut) raw_store(st, slot);   // the slot that it comes from may be written by `outputs`
  } else if (kOut) {
    raw_load(st, slot);
  }

  double total = 0.0;
  for (int c = 0; c < g.n; c += kC) {
    const int64_t t = g.t0 + c;
    const int n = min(kC, g.n - c);
    Rows rk, rv, rq;
    load_rows(rk, p.k + t * p.k_stride + hk * kD, p.k_stride, n);
    load_rows(rv, p.v + t * p.v_stride + hk * kD, p.v_stride, n);
    const double b = decay_sums(p, t, n, hk), end = __shfl(b, 63);
    total += end;
    __syncthreads();
    store_rows(rk, s.k);
    store_rows(rv, s.v);
    if (wave == 0) {
      const float hi = (float)b;
      s.hi[lane] = hi;
      s.lo[lane] = (float)(b - (double)hi);
      s.from[lane] = __builtin_amdgcn_exp2f(hi);
      s.to[lane] = __builtin_amdgcn_exp2f((float)(end - b));
    }
    const float whole = __builtin_amdgcn_exp2f((float)end);
    __syncthreads();

    Frag vf[4];   // V columns of this wave: steps of 16 tokens
#pragma unroll
    for (int j = 0; j < 4; ++j) vf[j] = columns(s.v, 16 * j, 32 * wave);

    if (kOut) {
      Frag sf[4][2][2];
#pragma unroll
      for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = st.a[db][8 * x + e];
          split8<2>(y, sf[db][x]);
        }
      for (int h = hk * grp; h < hk * grp + grp; ++h) {
        load_rows(rq, p.q + t * p.q_stride + h * kD, p.q_stride, n);
        __syncthreads();
        store_rows(rq, s.q);
        __syncthreads();
        if (wave < 3) {   // scores: keys j0 .. against queries i0 .., transposed
          const int i0 = wave == 0 ? 0 : 32, j0 = wave == 2 ? 32 : 0;
          f32x16 x;
#pragma unroll
          for (int r = 0; r < 16; ++r) x[r] = 0.0f;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            Frag a, q;
            a.w = *reinterpret_cast<const u32x4*>(&s.k[j0 + l32][16 * k + 8 * half]);
            q.w = *reinterpret_cast<const u32x4*>(&s.q[i0 + l32][16 * k + 8 * half]);
            x = mfma32_bf16(a.b, q.b, x);
          }
          const float hi = s.hi[i0 + l32], lo = s.lo[i0 + l32];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int j = j0 + 16 * y + 8 * (e >> 2) + 4 * half + (e & 3);
              const float d = __builtin_amdgcn_exp2f((hi - s.hi[j]) + (lo - s.lo[j]));
              w[e] = j <= i0 + l32 ? x[8 * y + e] * d : 0.0f;
            }
            Frag f[2];
            split8<2>(w, f);
            s.p[wave][y][0][lane] = f[0].w;
            s.p[wave][y][1][lane] = f[1].w;
          }
        }
        __syncthreads();
#pragma unroll
        for (int ib = 0; ib < 2; ++ib) {
          const int i = 32 * ib + l32;
          f32x16 o;
#pragma unroll
          for (int r = 0; r < 16; ++r) o[r] = 0.0f;
#pragma unroll
          for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              Frag q;
              q.d[0] = *reinterpret_cast<const u32x2*>(&s.q[i][32 * db + 16 * x + 4 * half]);
              q.d[1] = *reinterpret_cast<const u32x2*>(&s.q[i][32 * db + 16 * x + 8 + 4 * half]);
              o = mfma32_bf16(sf[db][x][1].b, q.b, o);
              o = mfma32_bf16(sf[db][x][0].b, q.b, o);
            }
          const float from = s.from[i];
#pragma unroll
          for (int r = 0; r < 16; ++r) o[r] *= from;
#pragma unroll
          for (int blk = ib; blk <= 2 * ib; ++blk)   // score blocks of these queries: 0, or 1 and 2
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const Frag v = vf[(blk == 2 ? 2 : 0) + y];
              Frag w;
              w.w = s.p[blk][y][1][lane];
              o = mfma32_bf16(v.b, w.b, o);
              w.w = s.p[blk][y][0][lane];
              o = mfma32_bf16(v.b, w.b, o);
            }
          if (i < n) {
            uint16_t* to = p.out + ((t + i) * p.h_q + h) * kD + 32 * wave + 4 * half;
#pragma unroll
            for (int a = 0; a < 4; ++a)
              *reinterpret_cast<u32x2*>(to + 8 * a) = (u32x2){pack_bf16(o[4 * a] * p.scale, o[4 * a + 1] * p.scale),
                                                             pack_bf16(o[4 * a + 2] * p.scale, o[4 * a + 3] * p.scale)};
          }
        }
      }
    }

#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) st.a[db][r] *= whole;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t w = vf[j].w[e >> 1];
        y[e] = (e & 1 ? bits_hi(w) : bits_lo(w)) * s.to[16 * j + 8 * (e >> 2) + 4 * half + (e & 3)];
      }
      Frag f[3];
      split8<3>(y, f);
#pragma unroll
      for (int db = 0; db < 4; ++db) {
        const Frag k = columns(s.k, 16 * j, 32 * db);
#pragma unroll
        for (int i = 2; i >= 0; --i) st.a[db] = mfma32_bf16(k.b, f[i].b, st.a[db]);
      }
    }
  }

  if (!kOut) {
    raw_store(st, slot + (int64_t)p.h_kv * kLinState);
    if (threadIdx.x == 0) p.decays[(int64_t)id * p.h_kv + hk] = __builtin_amdgcn_exp2f((float)total);
  } else if (last) {
    const int dst = p.state_dst[g.b];
    if (dst >= 0) state_store(st, p.states + ((int64_t)dst * p.h_kv + hk) * kLinState);
  }
}

// The states before the segments of a sequence: `sums` left, in the place of segment s + 1, the state that
// segment s alone leaves (segment 0 with the sequence's first state).  A thread takes four values through
// all segments.
constexpr int kJoinBlocks = kLinState / 4 / 256;
__global__ __launch_bounds__(256) void linear_join_kernel(LinearParams p, int segments) {
  const int part = blockIdx.x % kJoinBlocks, hk = blockIdx.x / kJoinBlocks;
  for (int id = blockIdx.y; id < segments; id += gridDim.y) {
    Segment g;
    if (!find_segment(p, id, &g) || g.s != 1 || g.count < 3) continue;
    f32x4* at = reinterpret_cast<f32x4*>(p.starts + ((int64_t)id * p.h_kv + hk) * kLinState) + part * 256 + threadIdx.x;
    const float* decay = p.decays + (int64_t)id * p.h_kv + hk;
    f32x4 x = *at;
    for (int s = 2; s < g.count; ++s) {
      at += p.h_kv * (kLinState / 4);
      x = x * *decay + *at;
      *at = x;
      decay += p.h_kv;
    }
  }
}

}  // namespace

hipError_t launch_linear_prefill(const LinearParams& p, hipStream_t stream) {
  const int64_t segments = linear_segments(p.batch, p.total_tokens, p.segment);
  const dim3 grid((unsigned)(segments * p.h_kv));
  if (p.split) {
    linear_chunks_kernel<false><<<grid, dim3(256), 0, stream>>>(p);
    linear_join_kernel<<<dim3(kJoinBlocks * p.h_kv, (unsigned)std::min<int64_t>(segments, 2048)), dim3(256), 0, stream>>>(p, (int)segments);
  }
  linear_chunks_kernel<true><<<grid, dim3(256), 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace mpfa
