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

// Rows of 128 channels in LDS lie without padding, their 16-byte pieces exchanged by row so that neither 16
// rows' same piece nor four rows' same 64 bytes (a transposing read) meet in a bank.
typedef uint16_t LdsRows[kC][kD];
__device__ __forceinline__ int piece(int row, int c) { return 8 * (c ^ ((row & 3) << 2 | (row >> 2 & 3))); }

struct Lds {
  LdsRows k, v, q;                             // q: in each 16 channels those of a lane half side by side
  u32x4 p[3][2][2][64];                        // scores: block, step of 16 keys, high and low parts, lane
  struct Decays {
    float hi[kC], lo[kC];                      // log2 of the decays from the chunk's start, in two parts
    float from[kC], to[kC];                    // exp2 of them; exp2 from each token to the chunk's end
  } d[2];                                      // of this chunk and the next
};

// What stands before in the source stays before.  Products and the vector work of the next ones are written in
// turns: a wave's own matrix and vector instructions overlap only so, and with two waves a SIMD there is too
// little else to run beside them.  The compiler by itself puts all products of a step behind all its vector work.
__device__ __forceinline__ void turn() { __builtin_amdgcn_sched_barrier(0); }

// The lane, by a value of each use's own: what is worked out from it (LDS addresses above all) is not kept in
// registers from one use to the next, of which there are not enough.
__device__ __forceinline__ int lane_here() {
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  return lane;
}

// Four tokens (rows t .. t + 3) of the lane's column c0 + lane % 32, t = t0 + 4 * (lane / 32): each
// group of 16 lanes reads a block of four rows and 16 columns, and gets it transposed.
__device__ __forceinline__ s16x4 column4(const LdsRows& rows, int lane, int t0, int c0) {
  typedef __attribute__((address_space(3))) s16x4 lds4;
  const int i = lane & 15, row = t0 + 4 * (lane >> 5) + (i >> 2);
  const uint16_t* at = &rows[row][piece(row, c0 / 8 + (lane >> 4 & 1) * 2 + (i >> 1 & 1)) + 4 * (i & 1)];
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)at);
}
// The tokens of one 16-token step in the order in which an accumulator holds its rows.
__device__ __forceinline__ Frag columns(const LdsRows& rows, int lane, int t0, int c0) {
  Frag f;
  f.s[0] = column4(rows, lane, t0, c0);
  f.s[1] = column4(rows, lane, t0 + 8, c0);
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
// The i-th part of values 2 w and 2 w + 1; x becomes what is left.
__device__ __forceinline__ void split2(float* x, Frag* part, int i, int w) {
  uint32_t h = pack_bf16(x[2 * w], x[2 * w + 1]);
  asm("" : "+v"(h));   // else the compiler makes the low half once more by itself
  part[i].w[w] = h;
  x[2 * w] -= bits_lo(h);
  x[2 * w + 1] -= bits_hi(h);
}
template <int kParts>
__device__ __forceinline__ void split8(float* x, Frag* part) {
#pragma unroll
  for (int i = 0; i < kParts; ++i)
#pragma unroll
    for (int w = 0; w < 4; ++w) split2(x, part, i, w);
}

// Rows of a chunk, 16 lanes a row, four rows of each thread.  Rows from n (at least 1) on are row n - 1 again:
// nothing of them reaches an output or the state, by the scores' mask and a decay of 0.
struct Rows {
  u32x4 w[4];
};
__device__ __forceinline__ void load_rows(Rows& r, const uint16_t* x, int64_t stride, int n) {
  const int row = threadIdx.x >> 4, c = threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.w[i] = *reinterpret_cast<const u32x4*>(x + min(row + 16 * i, n - 1) * stride + 8 * c);
}
__device__ __forceinline__ void store_rows(const Rows& r, LdsRows& to) {
  const int row = threadIdx.x >> 4, c = threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<u32x4*>(&to[row + 16 * i][piece(row + 16 * i, c)]) = r.w[i];
}
// Queries: of 16 channels 0-3, 8-11 | 4-7, 12-15.
__device__ __forceinline__ void store_queries(const Rows& r, LdsRows& to) {
  const int row = threadIdx.x >> 4, c = threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int x = 0; x < 2; ++x)
      *reinterpret_cast<u32x2*>(&to[row + 16 * i][piece(row + 16 * i, (c & ~1) + x) + 4 * (c & 1)]) = (u32x2){r.w[i][2 * x], r.w[i][2 * x + 1]};
}

// The value is in its registers here: loads of it have arrived, and what is made of it is not made before.
__device__ __forceinline__ void keep(f32x16& x) { asm volatile("" : "+v"(x)); }

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

// Log decays of a chunk (lane = token; 0 behind its last).
__device__ __forceinline__ float load_decays(const LinearParams& p, int64_t t, int n, int hk) {
  const int lane = threadIdx.x & 63;
  return lane < n ? p.log_decay[(t + lane) * p.decay_stride + hk] : 0.0f;
}

template <int kControl, int kRows>
__device__ __forceinline__ double moved(double x) {   // lanes without a source get 0
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (uint32_t)u, kControl, kRows, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (uint32_t)(u >> 32), kControl, kRows, 0xF, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// What a chunk of n tokens needs of its decays g; returns log2 of the whole chunk's.  Summed in 64 bits: after a token that
// clears the state sums are large and their differences small.
__device__ __forceinline__ double put_decays(Lds::Decays& d, float g, int n) {
  const int lane = threadIdx.x & 63;
  double x = (double)fminf(fmaxf(g, kLinLeastDecay), 0.0f) * kLog2e;
  x += moved<0x111, 0xF>(x);   // from 1, 2, 4, 8 lanes before in a row of 16
  x += moved<0x112, 0xF>(x);
  x += moved<0x114, 0xF>(x);
  x += moved<0x118, 0xF>(x);
  x += moved<0x142, 0xA>(x);   // the last lane of a row to the next row, rows 1 and 3
  x += moved<0x143, 0xC>(x);   // lane 31 to rows 2 and 3
  const double end = __shfl(x, 63);
  const float hi = (float)x;
  d.hi[lane] = hi;
  d.lo[lane] = (float)(x - (double)hi);
  d.from[lane] = __builtin_amdgcn_exp2f(hi);
  d.to[lane] = lane < n ? __builtin_amdgcn_exp2f((float)(end - x)) : 0.0f;
  return end;
}

// S' = exp(b_last) S + K^T (exp(b_last - b_j) V): K is an operand as it is, V with its decay in three parts.
__device__ __forceinline__ void update(State& st, const Lds& s, const Lds::Decays& d) {
  const int wave = threadIdx.x >> 6, lane = lane_here(), half = lane >> 5;
  const float whole = d.from[kC - 1];
  Frag v[2], k[2][4], f[2][3];
  f32x4 to[2][2];
  float y[8];
  auto read_v = [&](int j) { v[j & 1] = columns(s.v, lane, 16 * j, 32 * wave); };
  auto read_to = [&](int j, int q) { to[j & 1][q] = *reinterpret_cast<const f32x4*>(&d.to[16 * j + 8 * q + 4 * half]); };
  auto read_k = [&](int j, int db) { k[j & 1][db] = columns(s.k, lane, 16 * j, 32 * db); };
  auto split = [&](int j, int i, int w) {   // part i of the w-th pair of step j
    if (i == 0) {
      const uint32_t x = v[j & 1].w[w];
      y[2 * w] = bits_lo(x) * to[j & 1][w >> 1][2 * (w & 1)];
      y[2 * w + 1] = bits_hi(x) * to[j & 1][w >> 1][2 * (w & 1) + 1];
    }
    split2(y, f[j & 1], i, w);
  };
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    read_v(j);
    read_to(j, 0);
    read_to(j, 1);
  }
#pragma unroll
  for (int db = 0; db < 4; ++db) read_k(0, db);
  turn();
#pragma unroll
  for (int i = 0; i < 3; ++i)
#pragma unroll
    for (int w = 0; w < 4; ++w) split(0, i, w);
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) st.a[db][r] *= whole;
  turn();
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int n = 0; n < 12; ++n) {
      const int i = 2 - n / 4, db = n % 4;
      st.a[db] = mfma32_bf16(k[j & 1][db].b, f[j & 1][i].b, st.a[db]);
      if (j < 3) {
        split(j + 1, n / 4, n % 4);
        if (n < 4) read_k(j + 1, n);
      }
      if (j < 2 && n >= 9) {   // the last reads of step j + 1's v and decays are behind
        if (n == 9) read_v(j + 2);
        else read_to(j + 2, n - 10);
      }
      turn();
    }
}

// Scores of one block (keys j0 .., queries i0 ..), transposed, with their decays, as operands.
__device__ __forceinline__ void scores(Lds& s, const Lds::Decays& d, int block) {
  const int lane = lane_here(), half = lane >> 5, l32 = lane & 31;
  const int i0 = block == 0 ? 0 : 32, j0 = block == 2 ? 32 : 0, i = i0 + l32, jr = j0 + l32;
  Frag a[4], q[4];
  f32x4 jh[2], jl[2];
  auto read = [&](int k) {
    a[k & 3].d[0] = *reinterpret_cast<const u32x2*>(&s.k[jr][piece(jr, 2 * k) + 4 * half]);
    a[k & 3].d[1] = *reinterpret_cast<const u32x2*>(&s.k[jr][piece(jr, 2 * k + 1) + 4 * half]);
    q[k & 3].w = *reinterpret_cast<const u32x4*>(&s.q[i][piece(i, 2 * k + half)]);
  };
  auto read_decays = [&](int r4) {
    const int j = j0 + 8 * r4 + 4 * half;
    jh[r4 & 1] = *reinterpret_cast<const f32x4*>(&d.hi[j]);
    jl[r4 & 1] = *reinterpret_cast<const f32x4*>(&d.lo[j]);
  };
  read_decays(0);
#pragma unroll
  for (int k = 0; k < 4; ++k) read(k);
  read_decays(1);
  const float hi = d.hi[i], lo = d.lo[i];
  const int last = block == 1 ? kC : i;   // of the keys that the query sees: in block 1 all
  turn();
  f32x16 x;
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = 0.0f;
  float decay[16];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    x = mfma32_bf16(a[k & 3].b, q[k & 3].b, x);
    if (k < 4) read(k + 4);
#pragma unroll
    for (int r = 2 * k; r < 2 * k + 2; ++r) {
      const float reach = (hi - jh[r >> 2 & 1][r & 3]) + (lo - jl[r >> 2 & 1][r & 3]);
      decay[r] = __builtin_amdgcn_exp2f(j0 + 8 * (r >> 2) + 4 * half + (r & 3) <= last ? reach : -INFINITY);
    }
    if (k == 1 || k == 3) read_decays(k / 2 + 2);
    turn();
  }
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = x[8 * y + e] * decay[8 * y + e];
    Frag f[2];
    split8<2>(w, f);
    s.p[block][y][0][lane] = f[0].w;
    s.p[block][y][1][lane] = f[1].w;
  }
}

// o (transposed: rows are channels of v, 32 queries each) = exp(b_i) S^T q_i.  The state's parts are made for each
// query head anew: there is no room to keep them.
__device__ __forceinline__ void from_state(f32x16 (&o)[2], State& st, const Lds& s, const Lds::Decays& d) {
  const int lane = lane_here(), half = lane >> 5, l32 = lane & 31;
  Frag q[2][2], f[2][2];
  float y[8];
  auto read = [&](int g, int ib) {
    const int i = 32 * ib + l32;
    q[g & 1][ib].w = *reinterpret_cast<const u32x4*>(&s.q[i][piece(i, 2 * g + half)]);
  };
  auto split = [&](int g, int w) {
    y[2 * w] = st.a[g >> 1][8 * (g & 1) + 2 * w];
    y[2 * w + 1] = st.a[g >> 1][8 * (g & 1) + 2 * w + 1];
    split2(y, f[g & 1], 0, w);
    split2(y, f[g & 1], 1, w);
  };
#pragma unroll
  for (int db = 0; db < 4; ++db) keep(st.a[db]);
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int ib = 0; ib < 2; ++ib) read(g, ib);
  float from[2];
#pragma unroll
  for (int ib = 0; ib < 2; ++ib) from[ib] = d.from[32 * ib + l32];
#pragma unroll
  for (int w = 0; w < 4; ++w) split(0, w);
#pragma unroll
  for (int ib = 0; ib < 2; ++ib)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[ib][r] = 0.0f;
  turn();
#pragma unroll
  for (int g = 0; g < 8; ++g)
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int ib = n & 1;
      o[ib] = mfma32_bf16(f[g & 1][1 - n / 2].b, q[g & 1][ib].b, o[ib]);
      if (g < 7) split(g + 1, n);
      if (g < 6 && n >= 2) read(g + 2, ib);
      turn();
    }
#pragma unroll
  for (int ib = 0; ib < 2; ++ib)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[ib][r] *= from[ib];
}

// o += V^T scores.
__device__ __forceinline__ void from_chunk(f32x16 (&o)[2], const Lds& s) {
  const int lane = lane_here(), wave = threadIdx.x >> 6;
  Frag v[2][2], w[2][2][2];
  auto read = [&](int block) {
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      v[block & 1][y] = columns(s.v, lane, (block == 2 ? 32 : 0) + 16 * y, 32 * wave);
#pragma unroll
      for (int i = 0; i < 2; ++i) w[block & 1][y][i].w = s.p[block][y][i][lane];
    }
  };
  read(0);
  read(1);
  turn();
#pragma unroll
  for (int block = 0; block < 3; ++block) {
    f32x16& to = o[block == 0 ? 0 : 1];
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int i = 1; i >= 0; --i) to = mfma32_bf16(v[block & 1][y].b, w[block & 1][y][i].b, to);
    if (block == 0) read(2);
    turn();
  }
}

// The halves of a wave exchange channels, so that each lane stores 16 bytes of its query's row.
__device__ __forceinline__ void store_out(const f32x16& o, uint16_t* row, float scale) {
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int a = 0; a < 4; a += 2) {
    u32x4 w;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const uint32_t first = pack_bf16(o[4 * a + 2 * x] * scale, o[4 * a + 2 * x + 1] * scale);
      const uint32_t second = pack_bf16(o[4 * a + 4 + 2 * x] * scale, o[4 * a + 5 + 2 * x] * scale);
      const auto both = __builtin_amdgcn_permlane32_swap(first, second, false, false);
      w[x] = both[0];
      w[2 + x] = both[1];
    }
    if (row) *reinterpret_cast<u32x4*>(row + 8 * a + 8 * half) = w;
  }
}

// One workgroup of four waves per (segment, KV head) and, for outputs, part of its query heads.  kOut: the
// outputs of its tokens from the state before it, and of a sequence's last segment the state after it; else
// the segment's own state, for the next.  What the next step reads is on its way to registers during this one.
template <bool kOut>
__global__ __launch_bounds__(256, 2) void linear_chunks_kernel(LinearParams p, int items) {
  __shared__ Lds s;
  // parts of an item follow each other on one XCD
  const int parts = kOut ? p.parts : 1, item = blockIdx.x / (8 * parts) * 8 + blockIdx.x % 8, part = blockIdx.x / 8 % parts;
  if (item >= items) return;
  const int hk = item % p.h_kv, id = item / p.h_kv;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31;
  const int grp = p.h_q / p.h_kv, h0 = hk * grp + part * p.heads, h1 = min(h0 + p.heads, hk * grp + grp);
  Segment g;
  if (!find_segment(p, id, &g)) return;
  const bool last = g.s == g.count - 1;
  if (!kOut && last) return;
  float* const slot = p.split ? p.starts + ((int64_t)id * p.h_kv + hk) * kLinState : nullptr;
  const uint16_t* const k0 = p.k + g.t0 * p.k_stride + hk * kD;
  const uint16_t* const v0 = p.v + g.t0 * p.v_stride + hk * kD;
  const uint16_t* const q0 = p.q + g.t0 * p.q_stride;

  Rows rk, rv, rq;
  float decay = 0.0f;   // of the chunk after the next
  double total = 0.0;
  if (g.n > 0) {
    load_rows(rk, k0, p.k_stride, g.n);
    load_rows(rv, v0, p.v_stride, g.n);
    if (kOut) load_rows(rq, q0 + h0 * kD, p.q_stride, g.n);
  }

  State st;
  state_zero(st);
  if (g.s == 0 && (!kOut || g.count == 1)) {
    const int src = p.state_src[g.b];
    if (src >= 0) state_load(st, p.states + ((int64_t)src * p.h_kv + hk) * kLinState);
    if (!kOut) raw_store(st, slot);   // the slot that it comes from may be written by `outputs`
  } else if (kOut) {
    raw_load(st, slot);
  }
#pragma unroll
  for (int db = 0; db < 4; ++db) keep(st.a[db]);   // else the first use in the loop waits, in every chunk, for all loads before it
  if (wave == 3) {
    total = put_decays(s.d[0], load_decays(p, g.t0, g.n, hk), g.n);
    decay = load_decays(p, g.t0 + kC, g.n - kC, hk);
  }
  if (g.n > 0) {
    store_rows(rk, s.k);
    store_rows(rv, s.v);
    if (kOut) store_queries(rq, s.q);
  }

  for (int c = 0, x = 0; c < g.n; c += kC, x ^= 1) {
    const int rest = g.n - c - kC;   // tokens behind this chunk
    const Lds::Decays& d = s.d[x];
    __syncthreads();
    if (rest > 0) {
      load_rows(rk, k0 + (c + kC) * p.k_stride, p.k_stride, rest);
      load_rows(rv, v0 + (c + kC) * p.v_stride, p.v_stride, rest);
    }
    if (wave == 3 && rest > 0) {
      total += put_decays(s.d[x ^ 1], decay, rest);
      decay = load_decays(p, g.t0 + c + 2 * kC, rest - kC, hk);
    }
    if (kOut) {
      for (int h = h0; h < h1; ++h) {
        const bool more = h + 1 < h1;
        if (more || rest > 0) load_rows(rq, q0 + (more ? c : c + kC) * p.q_stride + (more ? h + 1 : h0) * kD, p.q_stride, more ? rest + kC : rest);
        if (h > h0) __syncthreads();
        if (wave < 3) scores(s, d, wave);
        f32x16 o[2];
        from_state(o, st, s, d);
        __syncthreads();
        if (more) store_queries(rq, s.q);
        from_chunk(o, s);
#pragma unroll
        for (int ib = 0; ib < 2; ++ib) {
          const int i = c + 32 * ib + l32;
          store_out(o[ib], i < g.n ? p.out + ((g.t0 + i) * p.h_q + h) * kD + 32 * wave : nullptr, p.scale);
        }
      }
    }
    if (!kOut || rest > 0 || (last && part == 0)) update(st, s, d);
    if (rest > 0) {
      __syncthreads();
      store_rows(rk, s.k);
      store_rows(rv, s.v);
      if (kOut) store_queries(rq, s.q);
    }
  }

  if (!kOut) {
    raw_store(st, slot + (int64_t)p.h_kv * kLinState);
    if (threadIdx.x == 255) p.decays[(int64_t)id * p.h_kv + hk] = __builtin_amdgcn_exp2f((float)total);
  } else if (last && part == 0) {
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
    const int64_t step = (int64_t)p.h_kv * (kLinState / 4);
    f32x4 x = *at;
    for (int s = 2; s < g.count; s += 8) {   // eight loads in flight
      f32x4 y[8];
      float a[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int j = min(i, g.count - 1 - s);
        y[i] = at[(j + 1) * step];
        a[i] = decay[j * p.h_kv];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (s + i >= g.count) break;
        x = x * a[i] + y[i];
        at[(i + 1) * step] = x;
      }
      at += 8 * step;
      decay += 8 * p.h_kv;
    }
  }
}

}  // namespace

hipError_t launch_linear_prefill(const LinearParams& p, hipStream_t stream) {
  const int64_t segments = linear_segments(p.batch, p.total_tokens, p.segment);
  const int items = (int)(segments * p.h_kv), eighths = (items + 7) / 8 * 8;
  if (p.split) {
    linear_chunks_kernel<false><<<dim3(eighths), dim3(256), 0, stream>>>(p, items);
    linear_join_kernel<<<dim3(kJoinBlocks * p.h_kv, (unsigned)std::min<int64_t>(segments, 2048)), dim3(256), 0, stream>>>(p, (int)segments);
  }
  linear_chunks_kernel<true><<<dim3((unsigned)(eighths * (int64_t)p.parts)), dim3(256), 0, stream>>>(p, items);
  return hipGetLastError();
}

}  // namespace mpfa
