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
// Chunks of 64: the products with the state cost a token 2 * 128 * 128 each whatever the chunk, those within it
// 64 * 128, and the decays' vector work grows with it too.
//
// What bounds it for long prompts is what a workgroup's waves can issue, not memory (65536 tokens of 32:8 heads, 1.3 GB
// in 403 us): products and vector instructions fill 70 % of a SIMD's cycles between them in `outputs`, 53 % in `sums`,
// with the two waves that the state's registers leave it, at 2.0 GHz and below, to which this work brings the clock
// (the first calls, at 2.3, take 278 us of `outputs`, later ones 320 to 355).  Where a unit has one workgroup waves wait
// for each other: 52 % and 36 % for 8192 tokens of 32:32 heads, 33 % and 12 % for four prompts of 40:8.
#include <algorithm>
#include <type_traits>

#include "linear_internal.h"
#include "mpfa_device.h"

namespace mpfa {

namespace {

constexpr int kC = kLinChunk;
constexpr int kThreads = 256;         // four waves of 32 columns (channels of v) each
constexpr int kStreamed = 2;          // a buffer access's non-temporal bit
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

__device__ __forceinline__ int count_of(const LinearParams& p, int len) { return linear_count(len, p.segment, p.split); }

// Sums over the lanes up to each: from 1, 2, 4, 8 lanes before in a row of 16, then the last lane of a row to the next
// row (rows 1 and 3), then lane 31 to rows 2 and 3.
template <int kControl, int kRows>
__device__ __forceinline__ int moved(int x) { return __builtin_amdgcn_update_dpp(0, x, kControl, kRows, 0xF, false); }
template <int kControl, int kRows>
__device__ __forceinline__ double moved(double x) {   // lanes without a source get 0
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, (uint64_t)(uint32_t)moved<kControl, kRows>((int)(u >> 32)) << 32 | (uint32_t)moved<kControl, kRows>((int)u));
}
template <typename T>
__device__ __forceinline__ T sums_to(T x) {
  x += moved<0x111, 0xF>(x);
  x += moved<0x112, 0xF>(x);
  x += moved<0x114, 0xF>(x);
  x += moved<0x118, 0xF>(x);
  x += moved<0x142, 0xA>(x);
  x += moved<0x143, 0xC>(x);
  return x;
}

// Segments are numbered over the batch.  Up to 64 sequences: without a gap, so that the workgroups that have work are
// the first ones and lie evenly over the units (eight prompts of 1000 tokens 92 -> 70 us); lane b has the first number
// of sequence b.
__device__ __forceinline__ int first_dense(const LinearParams& p, int* begin, int* count) {
  const int lane = threadIdx.x & 63;
  *begin = *count = 0;
  if (lane < p.batch) {
    *begin = p.cu_seqlens[lane];
    *count = count_of(p, p.cu_seqlens[lane + 1] - *begin);
  }
  return sums_to(*count) - *count;
}
// More: with gaps.
__device__ __forceinline__ int first_spread(const LinearParams& p, int begin, int b) { return linear_first(begin, p.segment, b); }

// Segment number id.
__device__ __forceinline__ bool find_segment(const LinearParams& p, int id, Segment* g) {
  const int lane = threadIdx.x & 63;
  int first;
  if (p.batch == 1) {
    g->b = first = 0;
  } else if (p.batch <= kLinDense) {
    int begin, count;
    const int mine = first_dense(p, &begin, &count);
    const uint64_t at = __builtin_amdgcn_ballot_w64(mine <= id && id < mine + count);
    if (at == 0) return false;
    g->b = __builtin_ctzll(at);
    first = __builtin_amdgcn_readlane(mine, g->b);
  } else {
    g->b = linear_search(p.cu_seqlens, p.batch, p.segment, id, [lane](auto before) {
      return (int)__popcll(__builtin_amdgcn_ballot_w64(before(lane)));
    });
    first = first_spread(p, p.cu_seqlens[g->b], g->b);
  }
  const int begin = p.cu_seqlens[g->b], len = p.cu_seqlens[g->b + 1] - begin;
  g->s = id - first;
  g->count = count_of(p, len);
  g->t0 = (int64_t)begin + (int64_t)g->s * p.segment;
  g->n = min(p.segment, len - g->s * p.segment);
  return g->s >= 0 && g->s < g->count;
}

// Rows of 128 channels in LDS lie without padding, their 16-byte pieces exchanged by row so that neither 16
// rows' same piece nor four rows' same four pieces (a transposing read) meet in a bank.
typedef uint16_t LdsRows[kC][kD];
__device__ __forceinline__ int piece_row(int row) { return (row & 3) << 2 | (row >> 2 & 3); }
// Of queries and outputs, whose half pieces of two rows that follow each other are written and read at once.
__device__ __forceinline__ int query_row(int row) { return row & 15; }

// What a chunk needs of its decays.
struct Decays {
  float hi[kC], lo[kC];                        // log2 of the decays from the chunk's start, in two parts
  float from[kC], to[kC];                      // exp2 of them times the scale; exp2 from each token to the chunk's end
};
struct Keys {                                  // `sums` has these alone
  LdsRows k, v;
  Decays d[2];                                 // of this chunk and the next
};
struct Lds : Keys {
  LdsRows q;                                   // queries, then outputs; see head_slot
  u32x4 p[3][2][2][64];                        // scores: block, step of 16 keys, high and low parts, lane
  f32x4 w[3][4][64];                           // their decays, for a chunk's second and later heads
};

// What stands before in the source stays before.  Products and the vector work of the next ones are written in
// turns: a wave's own matrix and vector instructions overlap only so, and with two waves a SIMD there is too
// little else to run beside them.  The compiler by itself puts all products of a step behind all its vector work.
__device__ __forceinline__ void turn() { __builtin_amdgcn_sched_barrier(0); }

// The thread, by a value of each use's own: what is worked out from it (LDS addresses above all) is not kept in
// registers from one use to the next, of which there are not enough.
__device__ __forceinline__ uint32_t thread_here() {
  uint32_t thread = threadIdx.x;
  asm volatile("" : "+v"(thread));
  return thread;
}
__device__ __forceinline__ int lane_here() { return thread_here() & 63; }

// LDS by byte offsets: rows are 256 bytes, so a piece's exchange is an exclusive or of a lane's offset, which
// serves all rows that lie a constant apart.
template <typename T>
__device__ __forceinline__ T read_lds(const LdsRows& rows, int at) {
  typedef __attribute__((address_space(3))) const char lds_char;
  typedef __attribute__((address_space(3))) const T lds_T;
  return *(lds_T*)((lds_char*)&rows + at);
}

// Offset of the lane's own row of 32 rows, in it the piece 0.
__device__ __forceinline__ int row_at(int lane) { return 256 * (lane & 31) + 16 * piece_row(lane); }
__device__ __forceinline__ int query_at(int lane) { return 256 * (lane & 31) + 16 * query_row(lane); }

// Transposing reads: four tokens t .. t + 3, t = t0 + 4 * (lane / 32), of the lane's column c0 + lane % 32: each
// group of 16 lanes reads a block of four rows and 16 columns.  columns_at: of t0 = c0 = 0.
__device__ __forceinline__ int columns_at(int lane) {
  const int i = lane & 15, row = 4 * (lane >> 5) + (i >> 2);
  return 256 * row + 16 * (((lane >> 4 & 1) * 2 + (i >> 1 & 1)) ^ piece_row(row)) + 8 * (i & 1);
}
__device__ __forceinline__ s16x4 column4(const LdsRows& rows, int at) {
  typedef __attribute__((address_space(3))) s16x4 lds4;
  typedef __attribute__((address_space(3))) char lds_char;
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)((lds_char*)const_cast<LdsRows*>(&rows) + at));
}
// The tokens t0 .. t0 + 15 in the order in which an accumulator holds its rows.
__device__ __forceinline__ Frag columns(const LdsRows& rows, int at, int t0) {
  Frag f;
  f.s[0] = column4(rows, at + 256 * t0);
  f.s[1] = column4(rows, (at ^ 32) + 256 * (t0 + 8));
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

// Rows of a chunk, 16 lanes a row; 0 from row n on.
struct Rows {
  static constexpr int kEach = kC * 16 / kThreads, kStep = kThreads / 16;
  u32x4 w[kEach];
  // stride: bytes between rows, of which 64 stay below 2^32; buffer loads check each row's offset by themselves
  __device__ __forceinline__ void load(const uint16_t* x, uint32_t stride, int n) {
    const uint32_t thread = thread_here();
    uint32_t at = (thread / 16) * stride + 16 * (thread & 15);
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(x), 0, (min(n, kC) - 1) * stride + 256, 0x00027000);
#pragma unroll
    for (int i = 0; i < kEach; ++i, at += kStep * stride) w[i] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 0, 0);
  }
};
// Pieces lie in the same place kStep rows on.
static_assert(Rows::kStep % 16 == 0, "see piece_row");
__device__ __forceinline__ void store_rows(const Rows& r, LdsRows& to) {
  const uint32_t thread = thread_here();
  char* const at = reinterpret_cast<char*>(&to) + 256 * (thread / 16) + 16 * ((thread & 15) ^ piece_row(thread / 16));
#pragma unroll
  for (int i = 0; i < Rows::kEach; ++i) *reinterpret_cast<u32x4*>(at + 256 * Rows::kStep * i) = r.w[i];
}
// Queries of a head and later its outputs: of 16 channels those that a lane half takes side by side, 0-3 and 8-11 |
// 4-7 and 12-15.  A thread's 16 bytes lie in two halves of pieces, for queries and outputs the same, so a thread
// that has read its outputs may put queries in their place.
struct HeadSlot {
  char* at[2];
  __device__ __forceinline__ HeadSlot(LdsRows& rows) {
    const uint32_t thread = thread_here(), c = thread & 15;
#pragma unroll
    for (int x = 0; x < 2; ++x) at[x] = reinterpret_cast<char*>(&rows) + 256 * (thread / 16) + 16 * (((c & ~1u) + x) ^ query_row(thread / 16)) + 8 * (c & 1);
  }
  __device__ __forceinline__ u32x2* operator()(int i, int x) const { return reinterpret_cast<u32x2*>(at[x] + 256 * Rows::kStep * i); }
};
__device__ __forceinline__ void store_queries(const Rows& r, LdsRows& to) {
  const HeadSlot slot(to);
#pragma unroll
  for (int i = 0; i < Rows::kEach; ++i)
#pragma unroll
    for (int x = 0; x < 2; ++x) *slot(i, x) = (u32x2){r.w[i][2 * x], r.w[i][2 * x + 1]};
}

// The value is in its registers here: loads of it have arrived.
__device__ __forceinline__ void keep(f32x16& x) { asm volatile("" : "+v"(x)); }

// A wave's part of the state: its 32 columns (channels of v), blocks of 32 rows (channels of k).
struct State {
  f32x16 a[4];
};
__device__ __forceinline__ int wave_here() { return threadIdx.x >> 6; }
__device__ __forceinline__ int state_at(int m, int r) {   // in [128][128]
  const int lane = threadIdx.x & 63;
  return (32 * m + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)) * kD + 32 * wave_here() + (lane & 31);
}
__device__ __forceinline__ void state_zero(State& s) {
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) s.a[m][r] = 0.0f;
}
__device__ __forceinline__ void state_load(State& s, const float* from) {
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) s.a[m][r] = from[state_at(m, r)];
}
__device__ __forceinline__ void state_store(const State& s, float* to) {
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) to[state_at(m, r)] = s.a[m][r];
}
// In the workspace a state lies as the accumulators do.
__device__ __forceinline__ void raw_store(const State& s, float* ws) {
#pragma unroll
  for (int n = 0; n < 16; ++n) {
    const f32x16& a = s.a[n >> 2];
    const int r = 4 * (n & 3);
    reinterpret_cast<f32x4*>(ws)[n * kThreads + threadIdx.x] = (f32x4){a[r], a[r + 1], a[r + 2], a[r + 3]};
  }
}
__device__ __forceinline__ void raw_load(State& s, const float* ws) {
#pragma unroll
  for (int n = 0; n < 16; ++n) {
    const f32x4 x = reinterpret_cast<const f32x4*>(ws)[n * kThreads + threadIdx.x];
#pragma unroll
    for (int e = 0; e < 4; ++e) s.a[n >> 2][4 * (n & 3) + e] = x[e];
  }
}

// Log decays of a chunk (lane = token; 0 behind its last).
__device__ __forceinline__ float load_decays(const LinearParams& p, int64_t t, int n, int hk) {
  const int lane = lane_here();
  return lane < n ? p.log_decay[(t + lane) * p.decay_stride + hk] : 0.0f;
}

// What a chunk of n tokens needs of its decays g; returns log2 of the whole chunk's.  Summed in 64 bits: after a token that
// clears the state sums are large and their differences small.
__device__ __forceinline__ double put_decays(Decays& d, float g, int n, float scale) {
  const int lane = lane_here();
  const double x = sums_to((double)fminf(fmaxf(g, kLinLeastDecay), 0.0f) * kLog2e);
  const double end = __shfl(x, 63);
  const float hi = (float)x;
  d.hi[lane] = hi;
  d.lo[lane] = (float)(x - (double)hi);
  d.from[lane] = __builtin_amdgcn_exp2f(hi) * scale;
  d.to[lane] = lane < n ? __builtin_amdgcn_exp2f((float)(end - x)) : 0.0f;
  return end;
}

// S' = exp(b_last) S + K^T (exp(b_last - b_j) V): K is an operand as it is, V with its decay in three parts.
struct Update {
  Frag v[4], f[2][3];                          // V of 16 tokens each; the parts of a step and of the next
  f32x4 to[2][2];                              // the decays of a step's and the next one's tokens
  float y[8], whole;

  __device__ __forceinline__ void read(const Keys& s, int vat) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = columns(s.v, vat, 16 * j);
  }
  __device__ __forceinline__ void read_to(const Decays& d, int half, int j, int q) {
    to[j & 1][q] = *reinterpret_cast<const f32x4*>(&d.to[16 * j + 8 * q + 4 * half]);
  }
  // part i of the w-th pair of step j
  __device__ __forceinline__ void split(int j, int i, int w) {
    if (i == 0) {
      const uint32_t x = v[j].w[w];
      y[2 * w] = bits_lo(x) * to[j & 1][w >> 1][2 * (w & 1)];
      y[2 * w + 1] = bits_hi(x) * to[j & 1][w >> 1][2 * (w & 1) + 1];
    }
    split2(y, f[j & 1], i, w);
  }
  // What comes before the products, as twelve turns' worth: a reading of decays, then a step's parts and the
  // state's decay.
  __device__ __forceinline__ void begin(const Decays& d, int half) {
    whole = __builtin_amdgcn_exp2f(d.hi[kC - 1]);
#pragma unroll
    for (int q = 0; q < 2; ++q) read_to(d, half, 0, q);
  }
  __device__ __forceinline__ void prepare(State& st, int n) {
    split(0, n / 4, n % 4);
#pragma unroll
    for (int e = 6 * n; e < 6 * n + 6; ++e)
      if (e < 64) st.a[e >> 4][e & 15] *= whole;
  }
  // The products, a step's parts beside those of the step before.
  __device__ __forceinline__ void add(State& st, const Keys& s, const Decays& d) {
    const int lane = lane_here(), at = columns_at(lane);
    Frag k[4];
    auto read_k = [&](int j, int m) { k[m] = columns(s.k, at ^ 64 * m, 16 * j); };
#pragma unroll
    for (int m = 0; m < 4; ++m) read_k(0, m);
#pragma unroll
    for (int q = 0; q < 2; ++q) read_to(d, lane >> 5, 1, q);
    turn();
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int n = 0; n < 12; ++n) {
        const int i = 2 - n / 4, m = n % 4;
        st.a[m] = mfma32_bf16(k[m].b, f[j & 1][i].b, st.a[m]);
        if (j < 3) {
          split(j + 1, n / 4, n % 4);
          if (n >= 8) read_k(j + 1, m);   // the last product with it
        }
        if (j < 2 && n >= 10) read_to(d, lane >> 5, j + 2, n - 10);   // step j's decays are used up
        turn();
      }
  }
};

// A block of scores: queries i .., keys j .. (32 each).  Three of them hold all keys that queries see.
struct Block {
  int i, j;
};
__device__ __forceinline__ Block block_of(int b) { return {b == 0 ? 0 : 32, b == 2 ? 32 : 0}; }

// Scores of one block, transposed, as operands, with their decays times the scale (0 for keys behind the query).
// kFirst: the chunk's first head makes the decays, and with kMore keeps them for the others.
template <bool kFirst, bool kMore>
__device__ __forceinline__ void scores(Lds& s, const Decays& d, int b, float scale) {
  const int lane = lane_here(), half = lane >> 5;
  const Block at = block_of(__builtin_amdgcn_readfirstlane(b));
  const int ka = (row_at(lane) ^ 16 * half) + 256 * at.j, qa = query_at(lane) + 8 * half + 256 * at.i;
  const int i = at.i + (lane & 31), j0 = at.j + 4 * half;
  Frag a[4], q[4];
  f32x4 jh[2], jl[2], decay[4];
  float hi = 0.0f, lo = 0.0f;
  auto read = [&](int k) {   // 16 channels each
    a[k & 3].w = read_lds<u32x4>(s.k, ka ^ 32 * k);
    q[k & 3].d[0] = read_lds<u32x2>(s.q, qa ^ 32 * k);
    q[k & 3].d[1] = read_lds<u32x2>(s.q, qa ^ (32 * k + 16));
  };
  auto read_decays = [&](int r4) {
    if (kFirst) {
      jh[r4 & 1] = *reinterpret_cast<const f32x4*>(&d.hi[j0 + 8 * r4]);
      jl[r4 & 1] = *reinterpret_cast<const f32x4*>(&d.lo[j0 + 8 * r4]);
    } else {
      decay[r4] = s.w[b][r4][lane];
    }
  };
  if (kFirst) {
    hi = d.hi[i];
    lo = d.lo[i];
  }
  read(0);
  read_decays(0);
#pragma unroll
  for (int k = 1; k < 4; ++k) read(k);
  read_decays(1);
  turn();
  f32x16 x;
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = 0.0f;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    x = mfma32_bf16(a[k & 3].b, q[k & 3].b, x);
    if (k < 4) read(k + 4);
    if (kFirst) {
#pragma unroll
      for (int r = 2 * k; r < 2 * k + 2; ++r) {
        const float reach = (hi - jh[r >> 2 & 1][r & 3]) + (lo - jl[r >> 2 & 1][r & 3]);
        decay[r >> 2][r & 3] = __builtin_amdgcn_exp2f(j0 + 8 * (r >> 2) + (r & 3) <= i ? reach : -INFINITY) * scale;
      }
      if (kMore && (k & 1)) s.w[b][k >> 1][lane] = decay[k >> 1];
    }
    if (k == 1 || k == 3) read_decays(k / 2 + 2);
    turn();
  }
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = x[8 * y + e] * decay[2 * y + (e >> 2)][e & 3];
    Frag f[2];
    split8<2>(w, f);
#pragma unroll
    for (int i = 0; i < 2; ++i) s.p[b][y][i][lane] = f[i].w;
  }
}

// Outputs of the chunk's queries, 32 a block: rows are the wave's channels of v.
struct Outputs {
  f32x16 o[2];
};

// The state as operands: 16 channels of k each, high and low parts.
struct Parts {
  Frag f[8][2];
};

// o = scale exp(b_i) S^T q_i.  kFirst: the chunk's first head makes the state's parts.
template <bool kFirst>
__device__ __forceinline__ void from_state(Outputs& to, const State& st, Parts& parts, const Lds& s, const Decays& d) {
  const int lane = lane_here(), qa = query_at(lane) ^ 16 * (lane >> 5);
  Frag q[2][2];
  float y[8];
  auto read = [&](int g, int i) { q[g & 1][i].w = read_lds<u32x4>(s.q, (qa ^ 32 * g) + 256 * 32 * i); };
  auto split = [&](int g, int w) {
    y[2 * w] = st.a[g >> 1][8 * (g & 1) + 2 * w];
    y[2 * w + 1] = st.a[g >> 1][8 * (g & 1) + 2 * w + 1];
    split2(y, parts.f[g], 0, w);
    split2(y, parts.f[g], 1, w);
  };
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int i = 0; i < 2; ++i) read(g, i);
  float from[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) from[i] = d.from[32 * i + (lane & 31)];
  if (kFirst) {
#pragma unroll
    for (int w = 0; w < 4; ++w) split(0, w);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) to.o[i][r] = 0.0f;
  turn();
#pragma unroll
  for (int g = 0; g < 8; ++g)
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int i = n & 1;
      to.o[i] = mfma32_bf16(parts.f[g][1 - n / 2].b, q[g & 1][i].b, to.o[i]);
      if (kFirst && g < 7) split(g + 1, n);
      if (g < 6 && n >= 2) read(g + 2, i);
      turn();
    }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) to.o[i][r] *= from[i];
}

// o += V^T scores.  kFinal: beside the products the state's update is prepared.
template <bool kFinal>
__device__ __forceinline__ void from_chunk(Outputs& to, Update& u, State& st, const Lds& s, const Decays& d) {
  const int lane = lane_here(), vat = columns_at(lane) ^ 64 * wave_here();
  Frag w[2][2][2];
  auto read = [&](int b, int y) {
#pragma unroll
    for (int i = 0; i < 2; ++i) w[b & 1][y][i].w = s.p[b][y][i][lane];
  };
  if (kFinal) u.begin(d, lane >> 5);
  u.read(s, vat);
#pragma unroll
  for (int y = 0; y < 2; ++y)
#pragma unroll
    for (int b = 0; b < 2; ++b) read(b, y);
  turn();
  // blocks 0 and 1, of one 16 keys and of different queries, in turns, then block 2
#pragma unroll
  for (int n = 0; n < 12; ++n) {
    const int b = n < 8 ? n & 1 : 2, y = n < 8 ? n >> 2 : n >> 1 & 1, i = n < 8 ? 1 - (n >> 1 & 1) : 1 - (n & 1);
    f32x16& o = to.o[b == 0 ? 0 : 1];
    o = mfma32_bf16(u.v[(b == 2 ? 2 : 0) + y].b, w[b & 1][y][i].b, o);
    if (n == 3 || n == 7) read(2, n >> 2);   // block 0's of the same keys are used up
    if (kFinal) u.prepare(st, n);
    turn();
  }
}

// Outputs to the place of the queries, from there whole rows to memory.
__device__ __forceinline__ void put_outputs(const Outputs& out, LdsRows& rows) {
  const int lane = lane_here(), at = query_at(lane) ^ (64 * wave_here() + 16 * (lane >> 5));
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = pack_bf16(out.o[i][8 * x + 2 * e], out.o[i][8 * x + 2 * e + 1]);
      *reinterpret_cast<u32x4*>(reinterpret_cast<char*>(&rows) + (at ^ 32 * x) + 256 * 32 * i) = w;
    }
}
__device__ __forceinline__ void read_outputs(Rows& r, LdsRows& rows) {
  const HeadSlot slot(rows);
#pragma unroll
  for (int i = 0; i < Rows::kEach; ++i) {
    const u32x2 a = *slot(i, 0), b = *slot(i, 1);
    r.w[i] = (u32x4){a[0], a[1], b[0], b[1]};
  }
}
// Of n rows, a multiple of 256 bytes apart; buffer stores, which drop what lies behind the last row without a
// branch: a wait for loads behind stores that are not always made would be one for these too.  Streamed past the
// cache, which K, V and the states of other heads need (four prompts 66 -> 61 us, 8192 tokens of 32:32 heads 131.5
// -> 129.5).
__device__ __forceinline__ void store_outputs(const Rows& r, uint16_t* to, int h_q, int n) {
  const uint32_t thread = thread_here(), stride = 256 * h_q;
  uint32_t at = (thread / 16) * stride + 16 * (thread & 15);
  const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(to, 0, (min(n, kC) - 1) * stride + 256, 0x00027000);
#pragma unroll
  for (int i = 0; i < Rows::kEach; ++i, at += Rows::kStep * stride) __builtin_amdgcn_raw_buffer_store_b128(r.w[i], rsrc, at, 0, kStreamed);
}

// Item number to KV head and segment.  A KV head's rows are 256 bytes of each token: were the heads dealt to the
// XCDs in order, an XCD would read from few of its L2's channels alone, so they rotate from segment to segment.
struct Item {
  int id, hk;
};
__device__ __forceinline__ Item item_of(const LinearParams& p, int item) {
  const int id = item / p.h_kv;
  return {id, (int)((uint32_t)(item + id + id / 8) % p.h_kv)};
}

// One workgroup per (segment, KV head): the segment's own state, for the next.  Three BF16 parts of V with its decay
// make 48 products a wave and chunk, beside 450 vector instructions, most of which make the parts; the loads of two
// chunks are on their way meanwhile.  2.7 us a chunk and unit (81 us for 65536 tokens of eight KV heads, 45 for 8192
// of 32); without its loads 10 % less, with a third of the products 13 %, with a third of the parts 2 %.  A sequence's first state goes to the
// place of its first segment, where several workgroups read it: its slot is written by whichever is done first.
__global__ __launch_bounds__(kThreads, 2) void linear_sums_kernel(LinearParams p) {
  __shared__ Keys s;
  const Item item = item_of(p, blockIdx.x);
  const int id = item.id, hk = item.hk;
  const int wave = wave_here();
  Segment g;
  if (!find_segment(p, id, &g)) return;
  const bool last = g.s == g.count - 1;
  if (last && (g.s > 0 || p.parts == 1)) return;
  float* const slot = p.starts + ((int64_t)id * p.h_kv + hk) * kLinState;
  const uint16_t* const k0 = p.k + g.t0 * p.k_stride + hk * kD;
  const uint16_t* const v0 = p.v + g.t0 * p.v_stride + hk * kD;
  const uint32_t kb = 2 * (uint32_t)p.k_stride, vb = 2 * (uint32_t)p.v_stride;
  struct {
    Rows k, v;
  } r[2];   // of the next chunk and the one after it
  auto load = [&](int x, int c) {   // behind the last chunk any rows will do
    const int at = c < g.n ? c : 0;
    r[x].k.load(k0 + at * p.k_stride, kb, g.n - at);
    r[x].v.load(v0 + at * p.v_stride, vb, g.n - at);
  };
  float now = 0.0f, decay = 0.0f;   // of this chunk and the next
  double total = 0.0;
  if (!last) {
    load(0, 0);
    load(1, kC);
    if (wave == 3) {
      now = load_decays(p, g.t0, g.n, hk);
      decay = load_decays(p, g.t0 + kC, g.n - kC, hk);
    }
  }
  State st;
  state_zero(st);
  if (g.s == 0) {
    const int src = p.state_src[g.b];
    if (src >= 0) state_load(st, p.states + ((int64_t)src * p.h_kv + hk) * kLinState);
    raw_store(st, slot);
    if (last) return;
  }
  if (wave == 3) total = put_decays(s.d[0], now, g.n, 1.0f);
  auto chunk = [&](int x, int c) {
    const int rest = g.n - c - kC;
    store_rows(r[x].k, s.k);
    store_rows(r[x].v, s.v);
    __syncthreads();
    load(x, c + 2 * kC);
    if (wave == 3 && rest > 0) {
      total += put_decays(s.d[x ^ 1], decay, rest, 1.0f);
      decay = load_decays(p, g.t0 + c + 2 * kC, rest - kC, hk);
    }
    Update u;
    const int lane = lane_here();
    u.begin(s.d[x], lane >> 5);
    u.read(s, columns_at(lane) ^ 64 * wave_here());
    turn();
#pragma unroll
    for (int n = 0; n < 12; ++n) u.prepare(st, n);
    turn();
    u.add(st, s, s.d[x]);
    __syncthreads();
  };
  for (int c = 0;; c += 2 * kC) {
    chunk(0, c);
    if (c + kC >= g.n) break;
    chunk(1, c + kC);
    if (c + 2 * kC >= g.n) break;
  }
  raw_store(st, slot + (int64_t)p.h_kv * kLinState);
  if (threadIdx.x == kThreads - 1) p.decays[(int64_t)id * p.h_kv + hk] = __builtin_amdgcn_exp2f((float)total);
}

// One workgroup per (segment, KV head, part of its query heads): the outputs of its tokens from the state before
// it, and of a sequence's last segment the state after it.  What is read next is on its way to registers meanwhile.
// The state's 128 columns lie in four waves' accumulators, so that it takes no LDS and its parts are made once for a
// chunk's heads; scores are made by three waves, one block each, and go to all four through LDS.  (Eight waves of 16
// columns, four a SIMD, read queries, keys and scores twice as often and were no faster: four prompts 73 us by them
// and 71 by these, 65536 tokens 430 and 433, where both were built alike.)
__global__ __launch_bounds__(kThreads, 2) void linear_outputs_kernel(LinearParams p) {
  __shared__ Lds s;
  // parts of an item follow each other on one XCD
  const int number = blockIdx.x / (8 * p.parts) * 8 + blockIdx.x % 8, part = blockIdx.x / 8 % p.parts;
  if (number >= p.items) return;
  const Item item = item_of(p, number);
  const int id = item.id, hk = item.hk;
  const int grp = p.h_q / p.h_kv, h0 = hk * grp + part * p.heads, h1 = min(h0 + p.heads, hk * grp + grp);
  const int wave = wave_here();
  Segment g;
  if (!find_segment(p, id, &g)) return;
  const bool last = g.s == g.count - 1;
  const uint16_t* const k0 = p.k + g.t0 * p.k_stride + hk * kD;
  const uint16_t* const v0 = p.v + g.t0 * p.v_stride + hk * kD;
  const uint16_t* const q0 = p.q + g.t0 * p.q_stride;
  const uint32_t kb = 2 * (uint32_t)p.k_stride, vb = 2 * (uint32_t)p.v_stride, qb = 2 * (uint32_t)p.q_stride;
  Rows rk, rv, rq;
  float now = 0.0f, decay = 0.0f;   // log decays of this chunk and the next
  if (g.n > 0) {
    if (wave == 3) {
      now = load_decays(p, g.t0, g.n, hk);
      decay = load_decays(p, g.t0 + kC, g.n - kC, hk);
    }
    rk.load(k0, kb, g.n);
    rv.load(v0, vb, g.n);
    rq.load(q0 + h0 * kD, qb, g.n);
  }
  State st;
  state_zero(st);
  if (g.count > 1 || p.parts > 1) {
    raw_load(st, p.starts + ((int64_t)id * p.h_kv + hk) * kLinState);
  } else {
    const int src = p.state_src[g.b];
    if (src >= 0) state_load(st, p.states + ((int64_t)src * p.h_kv + hk) * kLinState);
  }
#pragma unroll
  for (int m = 0; m < 4; ++m) keep(st.a[m]);   // else the first use in the loop waits, in every chunk, for all loads before it
  if (g.n > 0) {
    if (wave == 3) put_decays(s.d[0], now, g.n, p.scale);
    store_rows(rk, s.k);
    store_rows(rv, s.v);
    store_queries(rq, s.q);
  }

  for (int c = 0, x = 0; g.n > 0; c += kC, x ^= 1) {
    const int rest = g.n - c - kC, next = rest > 0 ? c + kC : c;   // behind the last chunk any rows will do
    const Decays& d = s.d[x];
    __syncthreads();
    Parts parts;
    if (wave == 3 && rest > 0) {
      put_decays(s.d[x ^ 1], decay, rest, p.scale);
      decay = load_decays(p, g.t0 + c + 2 * kC, rest - kC, hk);
    }
    auto step = [&](auto first, auto final, int h) {
      const int from = decltype(final)::value ? next : c;
      rq.load(q0 + from * p.q_stride + (decltype(final)::value ? h0 : h + 1) * kD, qb, g.n - from);
      // what all waves wait for goes before the other workgroup's work: the scores, then all between the barriers (four
      // prompts 59.4 -> 58.3 us, 65536 tokens 407 -> 400)
      __builtin_amdgcn_s_setprio(2);
      if (wave < 3) scores<decltype(first)::value, !decltype(final)::value>(s, d, wave, p.scale);
      __builtin_amdgcn_s_setprio(0);
      Outputs out;
      from_state<decltype(first)::value>(out, st, parts, s, d);
      if (decltype(final)::value) {   // not before: the state's parts were in these registers
        rk.load(k0 + next * p.k_stride, kb, g.n - next);
      }
      __syncthreads();   // the scores are there, the queries used
      __builtin_amdgcn_s_setprio(1);
      Update u;
      from_chunk<decltype(final)::value>(out, u, st, s, d);
      put_outputs(out, s.q);
      if (decltype(final)::value) {
        turn();
        rv.load(v0 + next * p.v_stride, vb, g.n - next);   // nor this: the scores and outputs were
      }
      if (decltype(final)::value && (rest > 0 || (last && part == 0))) u.add(st, s, d);
      __syncthreads();
      Rows ro;
      read_outputs(ro, s.q);
      store_queries(rq, s.q);
      if (decltype(final)::value) {
        store_rows(rk, s.k);
        store_rows(rv, s.v);
      }
      __builtin_amdgcn_s_setprio(0);
      store_outputs(ro, p.out + ((g.t0 + c) * p.h_q + h) * kD, p.h_q, g.n - c);
      if (!decltype(final)::value) __syncthreads();
    };
    const std::true_type yes;
    const std::false_type no;
    if (h0 + 1 == h1) {
      step(yes, yes, h0);
    } else {
      step(yes, no, h0);
      for (int h = h0 + 1; h < h1 - 1; ++h) step(no, no, h);
      step(no, yes, h1 - 1);
    }
    if (rest <= 0) break;
  }
  if (last && part == 0) {
    const int dst = p.state_dst[g.b];
    if (dst >= 0) state_store(st, p.states + ((int64_t)dst * p.h_kv + hk) * kLinState);
  }
}

// The states before the segments of a sequence: `sums` left, in the place of segment s + 1, the state that
// segment s alone leaves (segment 0 with the sequence's first state).  A workgroup has 256 values of it; each of
// its waves reads up to kLinJoin places at once, and adds to their sums what the segments before them left.  Memory
// and latency bound it: 33 MB read and 33 written in 14 us for 65536 tokens of 32:8 heads, 6 us for four prompts of
// 40:8 cut into 23 segments; eight places a wave, which leave room for half the waves, took 13 for 34 segments of
// theirs, four 8.
__global__ __launch_bounds__(64 * kLinJoinWaves) void linear_join_kernel(LinearParams p) {
  constexpr int kBlocks = kLinState / 256;
  __shared__ f32x4 s_end[kLinJoinWaves][64];
  __shared__ float s_decay[kLinJoinWaves];
  const int part = blockIdx.x % kBlocks, hk = blockIdx.x / kBlocks, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int64_t step = (int64_t)p.h_kv * (kLinState / 4);
  int dense = 0;
  if (p.batch > 1 && p.batch <= kLinDense) {
    int begin, count;
    dense = first_dense(p, &begin, &count);
  }
  for (int b = blockIdx.y; b < p.batch; b += gridDim.y) {
    const int begin = p.cu_seqlens[b], id = 1 + (p.batch <= kLinDense ? __shfl(dense, b) : first_spread(p, begin, b));   // of segment 1
    const int last = (p.cu_seqlens[b + 1] - begin + p.segment - 1) / p.segment - 2;   // places 1 .. last behind its own
    if (last < 1) continue;
    f32x4* const at = reinterpret_cast<f32x4*>(p.starts + ((int64_t)id * p.h_kv + hk) * kLinState) + part * 64 + lane;
    const float* const decay = p.decays + (int64_t)id * p.h_kv + hk;
    f32x4 carry = *at;
    for (int base = 1; base <= last; base += waves * kLinJoin) {
      const int first = base + wave * kLinJoin;
      f32x4 x[kLinJoin];
      float a[kLinJoin];
#pragma unroll
      for (int i = 0; i < kLinJoin; ++i) {
        x[i] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
        a[i] = 1.0f;
        if (first + i <= last) {
          x[i] = at[(first + i) * step];
          a[i] = decay[(int64_t)(first + i - 1) * p.h_kv];
        }
      }
#pragma unroll
      for (int i = 1; i < kLinJoin; ++i) {
        x[i] += x[i - 1] * a[i];
        a[i] *= a[i - 1];
      }
      __syncthreads();
      // behind the last place the decays are 1 and the sums 0: the wave's end is its last place's
      s_end[wave][lane] = x[kLinJoin - 1];
      if (lane == 0) s_decay[wave] = a[kLinJoin - 1];
      __syncthreads();
      f32x4 before = carry;
      for (int w = 0; w < waves; ++w) {
        if (w == wave) before = carry;
        carry = carry * s_decay[w] + s_end[w][lane];
      }
#pragma unroll
      for (int i = 0; i < kLinJoin; ++i)
        if (first + i <= last) at[(first + i) * step] = x[i] + before * a[i];
    }
  }
}

}  // namespace

hipError_t launch_linear_prefill(const LinearParams& p, hipStream_t stream) {
  const int eighths = (p.items + 7) / 8 * 8;
  if (p.split || p.parts > 1) linear_sums_kernel<<<dim3(p.items), dim3(kThreads), 0, stream>>>(p);
  if (p.split) {
    linear_join_kernel<<<dim3(kLinState / 256 * p.h_kv, std::min(p.batch, 64)), dim3(64 * p.join_waves), 0, stream>>>(p);
  }
  linear_outputs_kernel<<<dim3((unsigned)(eighths * (int64_t)p.parts)), dim3(kThreads), 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace mpfa
