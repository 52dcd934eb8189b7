// linear_cut.h -- how a prefill of linear attention is cut into segments, how these are numbered, and the workspace
// that follows from it: what the host decides from the sizes alone, and the rules that host and kernels share.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace mpfa {

constexpr int kLinChunk = 64;                  // tokens of a chunk
constexpr int kLinState = 128 * 128;           // floats of a state
constexpr int kLinDense = 64;                  // sequences whose segments are numbered without gaps
constexpr int64_t kLinUnits = 256;

// Segments of a sequence.
constexpr int linear_count(int len, int segment, int split) { return split ? std::max(1, (len + segment - 1) / segment) : 1; }
// With gaps, sequence b has the numbers from here on, of which ceil(len / segment) lie before the next one's.
constexpr int linear_first(int begin, int segment, int b) { return begin / segment + b; }
// The last of its sequences whose first number is at most id (the first one, if there is none), by 64-ary search; `lanes`
// counts the lanes of 64 for which it is told to.
template <typename Offsets, typename Lanes>
constexpr int linear_search(const Offsets& cu_seqlens, int batch, int segment, int id, const Lanes& lanes) {
  int lo = 0, n = batch;
  while (n > 1) {
    const int step = (n + 63) >> 6;
    const int last = std::max(1, lanes([&](int lane) {
      const int at = lane * step;
      return at < n && linear_first(cu_seqlens[lo + std::min(at, n - 1)], segment, lo + at) <= id;
    })) - 1;
    lo += last * step;
    n = std::min(step, n - last * step);
  }
  return lo;
}
// Numbers of segments that a batch may have.
constexpr int64_t linear_segments(int64_t batch, int64_t total_tokens, int64_t segment) { return total_tokens / segment + batch; }

// How prompts are cut.  Into as many segments (times KV heads: items) as there are units, or, where these get long,
// two a unit: two at once on a unit take less than one after the other, but every segment's states are written and
// read twice, 256 KB, which is what the rows of some hundred tokens are.  us with one and with two items a unit, by
// the chunks of the longer segments:
//   one head per KV head   8: 75, 82 (16384 tokens of 8:8)   16: 125, 124   24: 174, 174   32: 228, 221 (16384 of 32:32)
//   two                    8: 89, 100                         16: 167, 159
//   four                   2: 46, 52 (4096 of 32:8)   4: 71, 76   8: 130, 126   16: 238, 227   32: 474, 424
//   eight                  4: 106, 110 (32768 of 16:2)   8: 201, 196
//   sixteen                4: 178, 192 (65536 of 16:1)   8: 327, 335
// The rule is by the heads in turn; for sixteen it takes two a unit at eight chunks, which are 2 % slower there.
// Then the query heads of a KV head go in parts to workgroups of their own, where that fills the card better; each
// part takes the state through the segment for itself.
struct LinearCut {
  int chunks, parts, heads;   // of a segment; of a KV head's query heads; of a part
  int64_t items;              // at most
};
// What a chunk takes, in heads' times: its keys and the state's update once, every head; and more beside another
// workgroup of the unit.  us measured: 777 tokens of 32:8 heads, 104 items, 27.4 with four heads together, 24.8 with
// two, 25.6 one by one; 8192 (256) 71, 73, 88; 16384 of 16:1 in 128 items 87, 59 by eight, 56 by four, 64 by two; 5000
// of 10:2 (158) 33.9, 33.9 by three, 31.8 by two.
inline double linear_time(int heads, int64_t workgroups) {
  const double busy = (double)(workgroups - kLinUnits) / kLinUnits;
  return (1.33 + heads) * (busy <= 0.0 ? 1.0 : 1.25 + 0.37 * busy);
}
inline LinearCut linear_cut(int batch, int64_t total_tokens, int max_seqlen, int h_q, int h_kv) {
  const int grp = h_q / h_kv;
  const int64_t longest = std::min<int64_t>(max_seqlen, total_tokens);
  // segments of n chunks: at most, and as many as sequences of any lengths are cut into on average
  auto ends = [&](int64_t n) { return batch * std::max<int64_t>(1, (longest + n * kLinChunk - 1) / (n * kLinChunk)); };
  auto some = [&](int64_t n) {
    const int64_t spread = (total_tokens + n * kLinChunk - 1) / (n * kLinChunk) + (batch - 1) / 2;
    return std::max<int64_t>(batch, std::min(spread, ends(n)));
  };
  auto chunks = [&](int64_t items) {
    const int64_t least = std::max<int64_t>(1, (total_tokens * h_kv + items * kLinChunk - 1) / (items * kLinChunk));
    if ((int64_t)batch * h_kv <= items)
      for (int64_t n = least; n <= 2 * least; ++n)
        if (some(n) * h_kv <= items) return n;
    return least;   // sequences fill the card by themselves
  };
  LinearCut c;
  int64_t n = chunks(kLinUnits);
  if (n >= std::max(8, 24 / grp)) n = chunks(2 * kLinUnits);
  const int64_t items = some(n) * h_kv;
  c.chunks = (int)n;
  c.heads = grp;
  c.parts = 1;
  const double copy = longest > n * kLinChunk ? 0.0 : 2.0 / n;   // a launch that only parts need
  double best = linear_time(grp, items);
  for (int64_t parts = 2; parts <= grp && parts * items <= 2 * kLinUnits; ++parts) {
    const int heads = (grp + (int)parts - 1) / (int)parts;
    const double time = linear_time(heads, (grp + heads - 1) / heads * items) + copy;
    if (time < best) {
      best = time;
      c.heads = heads;
      c.parts = (grp + heads - 1) / heads;
    }
  }
  // without gaps in the numbers the longest sequence bounds them too
  const int64_t numbers = linear_segments(batch, total_tokens, n * kLinChunk);
  c.items = (batch <= kLinDense ? std::min(numbers, ends(n)) : numbers) * h_kv;
  return c;
}

// A prefill's cut and the two tables in its workspace: states before segments, then decays.
struct LinearSpace {
  int segment, parts, heads;
  bool split;
  int64_t items;
  size_t starts, bytes;
};
inline LinearSpace linear_space(int batch, int total_tokens, int max_seqlen, int h_q, int h_kv) {
  const LinearCut cut = linear_cut(batch, total_tokens, max_seqlen, h_q, h_kv);
  LinearSpace s;
  s.segment = cut.chunks * kLinChunk;
  s.parts = cut.parts;
  s.heads = cut.heads;
  s.items = cut.items;
  s.split = std::min(max_seqlen, total_tokens) > s.segment;
  const int64_t places = linear_segments(batch, total_tokens, s.segment) * h_kv;
  s.starts = ((size_t)places * kLinState * sizeof(float) + 255) / 256 * 256;
  s.bytes = s.split || s.parts > 1 ? s.starts + (size_t)places * sizeof(float) : 0;
  return s;
}

// A workspace that serves every call of up to these sizes.  Longer prompts may be cut into fewer segments than shorter
// ones, but no prompts into more than a chunk each or, beside one for each sequence, than two items a unit.
inline size_t linear_most_space(int batch, int total_tokens, int max_seqlen, int h_q, int h_kv) {
  if (h_q == h_kv && std::min(max_seqlen, total_tokens) <= kLinChunk) return 0;   // one segment, one workgroup a state
  const int64_t places = std::min<int64_t>((int64_t)(total_tokens / kLinChunk) * h_kv, 2 * kLinUnits) + (int64_t)batch * h_kv;
  return (size_t)places * (kLinState + 1) * sizeof(float);
}

}  // namespace mpfa
