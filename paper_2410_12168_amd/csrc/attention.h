// attention.h -- what the kernels of attention over the paged cache share: lane
// operations, the codes as matrix operands, and which block does which part of a
// ragged batch.
#pragma once

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged.h"

namespace comet {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kNone = -1e30f;  // maximum of no scores
constexpr int kTile = 64;        // tokens a wave takes at a time
constexpr int kWaves = 4;
// q is scaled so that a row's largest value lies in [2^kQueryBits, 2^(kQueryBits + 1)): as
// far up as fp16 goes, since small channels reach its lower end (odd ones a 16th of that)
constexpr int kQueryBits = 14;
// fewest tiles in a range: one for each wave
constexpr int kMinTiles = kWaves;

__device__ inline float low_half(uint32_t w) {
  return __half2float(__ushort_as_half((unsigned short)w));
}

// Rows of 16 lanes: the odd rows of a change places with the even rows of b
// (swap16), or a's upper half with b's lower (swap32).
__device__ inline void swap16(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}
__device__ inline void swap32(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}

// Maximum and sum over the four lanes of a column (l, l ^ 16, l ^ 32, l ^ 48).
template <typename F>
__device__ inline float over_quads(float v, F f) {
  uint32_t a = __float_as_uint(v), b = a;
  swap16(a, b);
  v = f(__uint_as_float(a), __uint_as_float(b));
  a = b = __float_as_uint(v);
  swap32(a, b);
  return f(__uint_as_float(a), __uint_as_float(b));
}
__device__ inline float quad_max(float v) {
  return over_quads(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ inline float quad_sum(float v) {
  return over_quads(v, [](float a, float b) { return a + b; });
}

// Sums over the lanes up to each (the last lane has all 64), without LDS: shifts
// within rows of 16, then the last lanes of rows 0 and 2, then of row 1.
template <int CTRL, int ROWS, typename T>
__device__ inline T shifted(T v) {
  return __builtin_bit_cast(
      T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xF, ROWS == 0xF));
}
template <typename T>
__device__ inline T sum_upto(T v) {
  v += shifted<0x111, 0xF>(v);
  v += shifted<0x112, 0xF>(v);
  v += shifted<0x114, 0xF>(v);
  v += shifted<0x118, 0xF>(v);
  v += shifted<0x142, 0xA>(v);
  v += shifted<0x143, 0xC>(v);
  return v;
}

// Eight codes as fp16, order (0, 4, 1, 5, 2, 6, 3, 7), times 2^-24 and, for the
// odd ones, 2^-20.
__device__ inline f16x8 codes_f16(uint32_t x) {
  const u32x4 r = {x & 0x000F000Fu, x & 0x00F000F0u, (x >> 8) & 0x000F000Fu,
                   (x >> 8) & 0x00F000F0u};
  return __builtin_bit_cast(f16x8, r);
}

// The same of codes less 8, exact as well: for V, whose weights are rounded.  An
// error of a weight counts times the code, so codes around 0 take most of it away.
__device__ inline f16x8 centered_f16(uint32_t x) {
  const u32x4 eight = {0x80088008u, 0x80808080u, 0x80088008u, 0x80808080u};  // -8 of each
  return codes_f16(x) + __builtin_bit_cast(f16x8, eight);
}

// Whether a {scale, offset} pair of fp16 numbers holds an infinity or not-a-number.
__device__ inline bool not_finite(uint32_t p) {
  return (p & 0x7C00u) == 0x7C00u || (p & 0x7C000000u) == 0x7C000000u;
}

// Tokens t .. t + 63 that a row at position `pos` sees of those in `have`, as bits.
__device__ inline unsigned long long seen_tokens(int pos, int t, int window,
                                                 unsigned long long have) {
  const int last = max(-1, min(kTile - 1, pos - t));
  const int first = window > 0 ? max(0, min(kTile, pos - window + 1 - t)) : 0;
  unsigned long long seen = last < kTile - 1 ? have & ((1ull << (last + 1)) - 1) : have;
  return first < kTile ? seen >> first << first : 0;
}

// ---- which part of the work ------------------------------------------------

struct UnitShape {
  int group;      // q heads per kv head
  int rows;       // q rows (of all heads of a group) per block, a power of two
  int window;
  int target;     // token ranges to aim at, per kv head
  int at_once;    // units that are at work at the same time, per kv head
  int low, high;  // of the sequences with more than `low` and at most `high` q rows
};

struct SeqWork {
  int start, n;    // first row, rows
  int len;         // tokens
  uint32_t blocks; // row blocks
  uint32_t first;  // first tile that any row sees
  uint32_t tiles;  // tiles from there on (1 at least)
};

__device__ inline SeqWork seq_work(const PagedBatch& b, int page_shift, const UnitShape& u,
                                   int seq) {
  SeqWork w{0, 0, 0, 0, 0, 0};
  if (seq >= b.B) return w;
  w.start = max(0, min(b.M, b.row_start[seq]));
  w.n = max(0, max(0, min(b.M, b.row_start[seq + 1])) - w.start);
  w.len = max(-b.M, min(1 << 30, b.seq_lens[seq]));
  const int seen = max(0, min(w.len, b.max_pages << page_shift));  // 2^30 at most
  const int low = w.len - w.n - u.window + 1;                       // of the first row's window
  const uint32_t all = (uint32_t)w.n * u.group;
  w.blocks = (int)all > u.low && (int)all <= u.high ? (all + u.rows - 1) >> (31 - __clz(u.rows)) : 0;
  w.first = u.window > 0 ? max(0, low) / kTile : 0;
  w.tiles = max(1, (seen + kTile - 1) / kTile - (int)w.first);
  return w;
}

// One block's work: row block `block` of sequence `seq`, range `range` of
// `ranges`, in which the sequence's tiles are shared out evenly.
struct Unit {
  int seq;
  uint32_t block, range, ranges;
  uint32_t slot;  // of the partial result
  SeqWork w;
};

// Lane `at`'s value (`at` the same in all lanes) where the compiler knows that all
// lanes have it.
template <typename T>
__device__ inline T from_lane(T v, int at) {
  return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), at));
}

__device__ inline uint32_t ranges_of(const SeqWork& w, float per) {
  return (uint32_t)ceilf((float)w.tiles / per);
}

// Unit `index`, counted over sequences, row blocks and ranges (SPLIT: row block
// `index` of those whose sequence has more than one range).  False if there is
// none.  Every wave of a launch works out the same from the lengths of all
// sequences, 64 at a time: first how many tiles a range may have, so that the
// ranges of full length are `target` at most (rounded up by more than the 32-bit
// sum can be off), then where the unit is.  Shorter last ranges can make that more
// units than run at once, and the device waits for a second turn of a few: ranges up
// to half as long again are then tried (64 users of 4096 tokens, 64 heads over 8 of
// 128 channels: 60 us without, 53 with; 32 users of up to 8192: 44 and 41), with up to
// 64 sequences, whose lengths one reading has (65 users of 1024 tokens: 28 us, 64: 21).
// With B sequences a wave reads up to 2 B lengths, and blocks grow with B: their square
// shows from about a thousand on (kv4_attention.hip has the times).  Sums of
// 32 bits: more than a launch can have only in batches that the interface does not
// allow, whose units are then any or none of the batch's.
template <bool SPLIT>
__device__ inline bool find_unit(const PagedBatch& b, int page_shift, const UnitShape& u,
                                 uint32_t index, Unit* out) {
  const int lane = threadIdx.x & 63;
  const SeqWork start = seq_work(b, page_shift, u, lane);
  float total = (float)start.blocks * (float)start.tiles;
  for (int s = 64; s < b.B; s += 64) {
    const SeqWork w = seq_work(b, page_shift, u, s + lane);
    total += (float)w.blocks * (float)w.tiles;
  }
  total = from_lane(sum_upto(total), 63) * 1.001f;
  float per = fmaxf((float)kMinTiles, ceilf(total / (float)u.target));
  uint32_t first_ranges = ranges_of(start, per);
  uint32_t first_upto = sum_upto(start.blocks * first_ranges);
  if (__builtin_expect(from_lane(first_upto, 63) > (uint32_t)u.at_once && b.B <= 64, 0)) {
    const float step = ceilf(per * 0.125f);
    auto fits = [&](float longer, uint32_t* ranges, uint32_t* upto) {
      *ranges = ranges_of(start, longer);
      *upto = sum_upto(start.blocks * *ranges);
      return from_lane(*upto, 63) <= (uint32_t)u.at_once;
    };
    uint32_t ranges, upto;
    if (fits(per + 4 * step, &ranges, &upto)) {  // the longest first: mostly none does
      int i = 1;
      #pragma unroll 1
      while (!fits(per + i * step, &ranges, &upto) && i < 4) ++i;
      first_ranges = ranges;
      first_upto = upto;
    }
  }
  uint32_t before = 0, slots_before = 0;
  for (int s = 0; s < b.B; s += 64) {
    const SeqWork w = s == 0 ? start : seq_work(b, page_shift, u, s + lane);
    const uint32_t ranges = s == 0 ? first_ranges : ranges_of(w, per);
    const uint32_t slots = ranges > 1 ? w.blocks * ranges : 0;
    const uint32_t mine = SPLIT ? (ranges > 1 ? w.blocks : 0) : w.blocks * ranges;
    const uint32_t upto = !SPLIT && s == 0 ? first_upto : before + sum_upto(mine);
    const uint32_t slots_upto = slots_before + sum_upto(slots);
    const unsigned long long hit = __ballot(mine > 0 && upto > index);
    if (hit) {
      const int at = __builtin_amdgcn_readfirstlane(__ffsll((long long)hit) - 1);
      const uint32_t k = index - from_lane(upto - mine, at);
      out->seq = s + at;
      out->ranges = from_lane(ranges, at);
      out->w.start = from_lane(w.start, at);
      out->w.n = from_lane(w.n, at);
      out->w.len = from_lane(w.len, at);
      out->w.blocks = from_lane(w.blocks, at);
      out->w.first = from_lane(w.first, at);
      out->w.tiles = from_lane(w.tiles, at);
      const uint32_t block = SPLIT ? k : k / out->ranges;
      out->range = SPLIT ? 0 : k % out->ranges;
      out->slot = from_lane(slots_upto - slots, at) + block * out->ranges + out->range;
      // the last row blocks see the most tokens: they come first
      out->block = out->w.blocks - 1 - block;
      return block < out->w.blocks;  // (the sums may have run over)
    }
    before = from_lane(upto, 63);
    slots_before = from_lane(slots_upto, 63);
  }
  return false;
}

// Partial results in the workspace: [slot][kv head][rows][D] sums and
// [slot][kv head][rows][2] {maximum (log2), sum of weights}.  A sequence with more
// than one range has more tiles than the longest range may have, which is at
// least all tiles over `target`: there are fewer than 2 * target slots.
struct Partials {
  float* sums;
  float* stats;
  uint32_t slots;
};

// The kernel for sequences of many rows (kv4_attention_many.hip).
constexpr int kManyRows = 128;  // of a block
hipError_t launch_attention_many(const PagedCache& c, const PagedBatch& b, const AttentionArgs& a,
                                 const UnitShape& u, const Partials& part, unsigned blocks,
                                 hipStream_t stream);

}  // namespace comet
