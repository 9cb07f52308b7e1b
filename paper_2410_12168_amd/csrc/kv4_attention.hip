// kv4_attention.hip -- causal attention of new rows over the paged 4-bit cache,
// gfx950.
//
// Row i of sequence b, q head h, at position p = L_b - n_b + i:
//   x_j = scale * q . k_j,  out = sum_j w_j v_j / sum_j w_j,  w_j = exp(x_j)
// over the tokens j <= p that the row sees, with the cached value q s + mn of a
// code.  A group's scale and offset are taken out of the sums,
//   q . k_j = sum_g s_jg (q . codes_j)_g + mn_jg (sum q)_g
//   sum_j w_j v_j = sum_j (w_j s_j) codes_j + sum_j w_j mn_j,
// so that both products run on the codes themselves.  One pass over the tokens
// with the running maximum and sum of the softmax.
//
// Matrix operands (v_mfma_f32_16x16x32_f16; rows: tokens or channels, columns:
// 16 rows of q):
//   - a code c is the fp16 subnormal c * 2^-24, which the matrix cores keep:
//     two masks and a shift make eight of them from a dword, every second one
//     16 times larger (its nibble sits four bits higher), which the other
//     operand takes back.  The order within a dword is (0, 4, 1, 5, 2, 6, 3, 7).
//   - q is scaled by a power of two per row (largest value in [2^14, 2^15)): the factor
//     costs no bits, subnormals cost some from 2^-24 of the largest value down (2^-35 of
//     it at most).  With the largest in [2^10, 2^11) it was from 2^-20 on.
//   - scale * log2(e) is a mantissa, multiplied into K's scales and the sums of q, times
//     a power of two that turns a score into the exponent of its weight (`kappa`).  That
//     product is exact, so that the largest score's exponent is 0 and none is above it,
//     however large the scores: with the whole factor in it, a rounded maximum of 2^24
//     and more left exponents above 0, and weights beyond fp16.
//   - w_j s_j is scaled by a power of two per wave, so that the largest scale of
//     the tokens so far lands in [2^14, 2^15), or a 16th of that for odd tokens, whose
//     codes are 16 times as large: the product loses bits only below 2^-28 (odd tokens:
//     2^-24) of the largest.  It is rounded to fp16 (2^-11 relative).
//   - V's operand needs 8 tokens of a channel in a lane; the cache has channels
//     in a row.  The transposing LDS read (ds_read_b64_tr_b4: 16 rows of 16
//     nibbles) turns 16 tokens x 16 channels at a time.
//   - token 16 j + 4 h + r of a 64-token tile is row 4 h + r of the j-th score
//     product, and V's rows are read in the order that gives quad h of the lanes
//     the tokens whose scores it has: the weights go from one product into the
//     other in place.
//
// V's codes count around 8: sum p c = sum p (c - 8) + 8 sum p, with the same rounded
// weights p in both sums, and the exact weights in the offsets' sum of the codes' 8.
// An error of a weight then counts times |c - 8| instead of c (outputs 3.1e-4 off 64
// bits in the mean without, 2.2e-4 with; rounding the output alone gives 2.1e-4).
//
// Work decomposition: a block of four waves takes one (sequence, kv head, 16 C
// rows of its q heads, range of tokens); the waves take turns at its 64-token
// tiles and add up in LDS at the end.  The token ranges follow from the lengths
// on the device (find_unit): every block of every sequence gets about the same
// number of tiles, about `target` ranges in all, and a second kernel adds up the
// ranges of a sequence that has more than one.
//
// What bounds it (64 q heads over 8 of 128 channels where nothing else is said; times
// of a call, passes back to back, floors at the 4.9 TB/s of a large copy):
//   - 64 users of up to 8192 tokens (284 MB): 73 us, 3.9 TB/s, floor 57: 4.2 TB/s in this
//     kernel (vector operations issue in 58% of its cycles, the matrix core works in 13%),
//     5 us for the sum over ranges.  Users of 8192 tokens each (573 MB): 109 us, 5.2 TB/s;
//     64-channel groups 117, 32-channel ones (673 MB) 161, with more to add up per code
//     and 7 registers spilled.  What holds the ragged batch at 4.2 is not shown; two thirds
//     or twice the token ranges run within 2%.
//   - one user of 131072 tokens, 32 heads (143 MB): 39 us, 3.6 TB/s, floor 29, of which
//     the sum over 96 ranges and the launches are 8.  Fewer or more ranges: 37 us
//     with two thirds, 44 with 4/3.
//   - one user of 100 tokens: 7 us, latency: one tile a wave at most, but the lengths,
//     the table and a tile to fetch one after the other, then the waves' sums.
//   - 16 users with 5 drafted rows each, 12 heads of 64 channels, up to 2000 tokens:
//     16 us (floor 3), 12 of it this kernel and 4 the sum over ranges.
//   - many users: 65 of 8192 tokens 126 us, 128 213, 256 407 (of 1024 tokens, 64: 21, 65:
//     28, 128: 36, 256: 67).  Every wave reads all sequences' lengths to find its unit,
//     which grows with their square: of 200 tokens, 256 31 us (floor 13), 1024 230 (52),
//     4096 2460 (207), 16384 35600 (830), 65536 554000 (3320).
#include <algorithm>
#include <cmath>

#include "attention.h"

namespace comet {

namespace {

// ---- the products --------------------------------------------------------------

// Blocks that a compute unit holds at a time, as the registers allow.  (With 128
// channels in groups of 32 they do not quite: 7 are spilled with C = 1, 5 with C = 2,
// 16 and 24 bytes a lane.)
__host__ __device__ constexpr int resident_few(int D, int G, int C) {
  return (C == 1 ? 3 : 2) + (D == 64 && (C == 1 || G == 64) ? 1 : 0);
}

template <int D, int G, int C>
__global__ __launch_bounds__(64 * kWaves, resident_few(D, G, C)) void kv4_attention_few_kernel(
    PagedCache c, PagedBatch b, AttentionArgs a, UnitShape u, Partials part) {
  constexpr int NG = D / G;         // groups of a head
  constexpr int KS = D / 32;        // steps of the score product
  constexpr int DB = D / 16;        // 16-channel blocks of the output
  constexpr int ROW = D / 2;        // bytes of a row of codes
  constexpr int VL = ROW / 16;      // 16-byte loads of V per lane
  // V's codes, then the parameters in 32 bits: [NG][K's s, mn, V's s, mn][64]
  constexpr int STAGE = kTile * ROW + 4 * NG * kTile * 4;
  constexpr int OPAD = D + 4;       // floats of a row of sums in LDS
  constexpr int SUMS = kWaves * 16 * C * OPAD * 4;
  constexpr int STATS = kWaves * 16 * C * (2 + NG) * 4;
  constexpr int LDS = STAGE * kWaves > SUMS ? STAGE * kWaves : SUMS;
  __shared__ __attribute__((aligned(16))) uint8_t lds[LDS];
  __shared__ __attribute__((aligned(16))) uint8_t lds_stats[STATS];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const int head = blockIdx.x % c.kv_heads;
  Unit unit;
  if (!find_unit<false>(b, c.page_shift, u, blockIdx.x / c.kv_heads, &unit)) return;
  const SeqWork& w = unit.w;
  const int row0 = unit.block * u.rows;             // of n * group
  const int rows = min(u.rows, w.n * u.group - row0);
  // positions of the block's first and last rows
  const int pos0 = w.len - w.n + row0 / u.group;
  const int pos1 = w.len - w.n + (row0 + rows - 1) / u.group;
  const int cap = b.max_pages << c.page_shift;
  // the unit's share of the sequence's tiles, without those its rows do not see
  const uint32_t each = w.tiles / unit.ranges, more = w.tiles % unit.ranges;
  int tile0 = w.first + unit.range * each + min(unit.range, more);
  int tile1 = tile0 + each + (unit.range < more);
  if (pos1 < 0)
    tile1 = 0;
  else
    tile1 = min(tile1, min(pos1, cap - 1) / kTile + 1);
  if (u.window > 0) tile0 = max(tile0, max(0, pos0 - u.window + 1) / kTile);

  // ---- pages: lane 4 i + k has the slab (page and head) of granule k (16 tokens) of
  // this wave's i-th next tile, or -1, so that a tile's slabs are scalars and its loads
  // do not wait behind a load of the table
  const int32_t* table = b.block_table + (long long)unit.seq * b.max_pages;
  const bool one_page = c.page_shift >= 6;  // a tile lies in one
  int slabs = -1;
  auto load_pages = [&](int tile) {
    const int token = (tile + (lane >> 2) * kWaves) * kTile + 16 * (lane & 3);
    const int i = token >> c.page_shift;
    slabs = slab_of(c, head, i < b.max_pages ? table[i] : -1);
  };
  // First rows in the cache of the tile's granules; a hole reads the first page.
  auto granule_rows = [&](int tile, int i, long long (&rows4)[4]) {
    rows4[0] = slab_row(c, __builtin_amdgcn_readlane(slabs, 4 * i), tile * kTile);
    #pragma unroll
    for (int k = 1; k < 4; ++k) rows4[k] = rows4[0] + 16 * k;
    if (!one_page) {
      #pragma unroll
      for (int k = 1; k < 4; ++k)
        rows4[k] = slab_row(c, __builtin_amdgcn_readlane(slabs, 4 * i + k), tile * kTile + 16 * k);
    }
  };

  // ---- loads of a tile: into registers, a tile ahead
  uint32_t kreg[4][KS];
  u32x4 vreg[VL];
  uint32_t preg[2][NG];
  unsigned long long held = 0;  // tokens that are in the cache
  auto load_k = [&](int tile, int ahead) {
    long long rows4[4];
    granule_rows(tile, ahead, rows4);
    #pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint8_t* at = c.k_codes + rows4[j] * ROW + (unsigned)(col * ROW + ROW / 4 * quad);
      if constexpr (KS == 4) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(at);
        kreg[j][0] = v[0], kreg[j][1] = v[1], kreg[j][2] = v[2], kreg[j][3] = v[3];
      } else {
        const u32x2 v = *reinterpret_cast<const u32x2*>(at);
        kreg[j][0] = v[0], kreg[j][1] = v[1];
      }
    }
  };
  auto load_v = [&](int tile, int ahead) {
    long long rows4[4];
    granule_rows(tile, ahead, rows4);
    #pragma unroll
    for (int i = 0; i < VL; ++i) {
      if constexpr (VL == 4) {
        vreg[i] = *reinterpret_cast<const u32x4*>(c.v_codes + rows4[i] * ROW + 16u * lane);
      } else {
        const long long row = lane < 32 ? rows4[2 * i] : rows4[2 * i + 1];
        vreg[i] = *reinterpret_cast<const u32x4*>(c.v_codes + row * ROW + 16u * (lane & 31));
      }
    }
    const long long mine = quad < 2 ? (quad == 0 ? rows4[0] : rows4[1])
                                    : (quad == 2 ? rows4[2] : rows4[3]);
    const long long at = (mine + col) * NG;
    #pragma unroll
    for (int g = 0; g < NG; ++g) {
      preg[0][g] = reinterpret_cast<const uint32_t*>(c.k_params)[at + g];
      preg[1][g] = reinterpret_cast<const uint32_t*>(c.v_params)[at + g];
    }
    held = 0;
    #pragma unroll
    for (int k = 0; k < 4; ++k)
      if (__builtin_amdgcn_readlane(slabs, 4 * ahead + k) >= 0) held |= 0xFFFFull << (16 * k);
    const int left = w.len - tile * kTile;
    if (left < kTile) held &= (1ull << max(left, 0)) - 1;
  };

  const int first = tile0 + wave;
  int ahead = 0;  // where in `slabs` the next tile is
  if (first < tile1) load_pages(first);

  // ---- q: operand [step] of each column block, its sums and factor
  f16x8 q[C][KS];
  float qsum[C][NG], kappa[C], top[C], weight_sum[C], offset[C][NG], rounded[C][NG];
  int pos[C];
  u32x4 raw_q[C][KS];
  #pragma unroll
  for (int cb = 0; cb < C; ++cb) {
    const int r = 16 * cb + col;
    const bool live = r < rows;
    const int i = (row0 + r) / u.group, h = (row0 + r) % u.group;
    pos[cb] = w.len - w.n + i;
    const uint16_t* x = a.Q + (long long)(w.start + i) * a.q_stride + (head * u.group + h) * D;
    #pragma unroll
    for (int s = 0; s < KS; ++s) {
      // a lane's codes of K: D / 4 channels in a row, or 8 of every 32 where the
      // steps have to stay within a group (as load_k's rows are turned)
      const int at = NG == 1 ? D / 4 * quad + 8 * s
                     : KS == 4 ? 32 * s + 8 * quad
                               : 32 * s + 16 * (quad & 1) + 8 * (quad >> 1);
      raw_q[cb][s] = u32x4{0, 0, 0, 0};
      if (live) raw_q[cb][s] = *reinterpret_cast<const u32x4*>(x + at);
    }
  }
  if (first < tile1) {
    load_k(first, 0);
    load_v(first, 0);
  }
  #pragma unroll
  for (int cb = 0; cb < C; ++cb) {
    const u32x4 (&raw)[KS] = raw_q[cb];
    float big = 0.0f;
    #pragma unroll
    for (int s = 0; s < KS; ++s) {
      #pragma unroll
      for (int k = 0; k < 4; ++k)
        big = fmaxf(big, fmaxf(fabsf(low_half(raw[s][k])), fabsf(low_half(raw[s][k] >> 16))));
    }
    big = quad_max(big);
    int e = kQueryBits;
    if (big > 0.0f && big < INFINITY) e = ilogbf(big);
    // an infinity in q: all scores of the row are infinities or not-a-numbers, and its
    // weights not-a-numbers, whatever their sign
    const float f = big < INFINITY ? ldexpf(a.scale < 0.0f ? -1.0f : 1.0f, kQueryBits - e) : NAN;
    // above 0, so that an unseen token's -infinity stays one
    kappa[cb] = fmaxf(ldexpf(1.0f, a.exponent + 24 + e - kQueryBits), 0x1p-120f);
    #pragma unroll
    for (int g = 0; g < NG; ++g) qsum[cb][g] = 0.0f;
    #pragma unroll
    for (int s = 0; s < KS; ++s) {
      float v[8];
      float sum = 0.0f;
      #pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[2 * k] = low_half(raw[s][k]) * f;
        v[2 * k + 1] = low_half(raw[s][k] >> 16) * f;
        sum += v[2 * k] + v[2 * k + 1];
      }
      qsum[cb][32 * s / G % NG] += sum;
      q[cb][s] = f16x8{(_Float16)v[0],            (_Float16)v[4],
                       (_Float16)(v[1] * 0.0625f), (_Float16)(v[5] * 0.0625f),
                       (_Float16)v[2],            (_Float16)v[6],
                       (_Float16)(v[3] * 0.0625f), (_Float16)(v[7] * 0.0625f)};
    }
    #pragma unroll
    for (int g = 0; g < NG; ++g) qsum[cb][g] = quad_sum(qsum[cb][g]) * (0x1p-24f * a.mantissa);
    top[cb] = kNone;
    weight_sum[cb] = 0.0f;
    #pragma unroll
    for (int g = 0; g < NG; ++g) offset[cb][g] = rounded[cb][g] = 0.0f;
  }

  f32x4 o[C][DB];
  #pragma unroll
  for (int cb = 0; cb < C; ++cb)
    #pragma unroll
    for (int d = 0; d < DB; ++d) o[cb][d] = f32x4{0, 0, 0, 0};
  int vexp = -24;  // exponent of the largest scale of V so far
  float weight_unit = ldexpf(1.0f, (lane & 1 ? 10 : 14) - vexp);

  uint8_t* stage = lds + wave * STAGE;
  float* params = reinterpret_cast<float*>(stage + kTile * ROW);

  // Where a 16-byte chunk of V's row lies in LDS: the 16 rows of a transposing read
  // (16 j + 4 quad + r, one chunk) in different banks.
  auto v_place = [](int token, int chunk) {
    if constexpr (VL == 4) return token * ROW + 16 * (chunk ^ token >> 4);
    return (token ^ token >> 5 << 2) * ROW + 16 * (chunk ^ (token >> 4 & 1));
  };

  // ---- one tile
  auto work = [&](int tile, bool whole, unsigned long long have, int ahead) {
    f32x4 x[C][4];
    #pragma unroll
    for (int j = 0; j < 4; ++j) {
      f32x4 dot[C];
      if constexpr (NG > 1 && KS == 4) {  // 16 channels of a quad's 4 loads -> of 4 quads
        swap32(kreg[j][0], kreg[j][2]);
        swap32(kreg[j][1], kreg[j][3]);
        swap16(kreg[j][0], kreg[j][1]);
        swap16(kreg[j][2], kreg[j][3]);
      } else if constexpr (NG > 1) {
        swap32(kreg[j][0], kreg[j][1]);
      }
      #pragma unroll
      for (int g = 0; g < NG; ++g) {
        #pragma unroll
        for (int cb = 0; cb < C; ++cb) dot[cb] = f32x4{0, 0, 0, 0};
        #pragma unroll
        for (int s = g * KS / NG; s < (g + 1) * KS / NG; ++s) {
          const f16x8 k = codes_f16(kreg[j][s]);
          #pragma unroll
          for (int cb = 0; cb < C; ++cb)
            dot[cb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[cb][s], dot[cb], 0, 0, 0);
        }
        if constexpr (NG > 1) __builtin_amdgcn_sched_barrier(0);  // keeps registers few
        const float* at = params + 4 * g * kTile + 16 * j + 4 * quad;
        const f32x4 s = *reinterpret_cast<const f32x4*>(at);
        const f32x4 mn = *reinterpret_cast<const f32x4*>(at + kTile);
        #pragma unroll
        for (int r = 0; r < 4; ++r) {
          #pragma unroll
          for (int cb = 0; cb < C; ++cb) {
            const float more = g ? fmaf(mn[r], qsum[cb][g], x[cb][j][r]) : mn[r] * qsum[cb][g];
            x[cb][j][r] = fmaf(s[r], dot[cb][r], more);
          }
        }
      }
      // done here: put off to their next use, they would keep all parameters and
      // products of the tile in registers
      #pragma unroll
      for (int cb = 0; cb < C; ++cb) asm volatile("" : "+v"(x[cb][j]));
    }
    if (tile + kWaves < tile1) load_k(tile + kWaves, ahead);
    if (!whole) {
      const int t = tile * kTile;
      #pragma unroll
      for (int cb = 0; cb < C; ++cb) {
        unsigned long long seen = seen_tokens(pos[cb], t, u.window, have);
        seen >>= 4 * quad;  // bit 16 j + r
        #pragma unroll
        for (int k = 0; k < 16; ++k) {
          const uint32_t half = (uint32_t)(seen >> (k < 8 ? 0 : 32));
          if (!(half >> (16 * (k / 4 % 2) + k % 4) & 1u)) x[cb][k / 4][k % 4] = -INFINITY;
        }
      }
    }
    // running maximum; what was added up before shrinks with it
    float next[C];
    bool grown = false;
    #pragma unroll
    for (int cb = 0; cb < C; ++cb) {
      float m = x[cb][0][0];
      #pragma unroll
      for (int k = 1; k < 16; ++k) m = fmaxf(m, x[cb][k / 4][k % 4]);
      next[cb] = fmaxf(top[cb], quad_max(m) * kappa[cb]);
      grown |= next[cb] > top[cb];
    }
    if (__any(grown)) {
      #pragma unroll
      for (int cb = 0; cb < C; ++cb) {
        const float f = __builtin_amdgcn_exp2f(top[cb] - next[cb]);
        top[cb] = next[cb];
        weight_sum[cb] *= f;
        #pragma unroll
        for (int g = 0; g < NG; ++g) {
          offset[cb][g] *= f;
          rounded[cb][g] *= f;
        }
        #pragma unroll
        for (int d = 0; d < DB; ++d) o[cb][d] *= f;
      }
    }
    #pragma unroll
    for (int cb = 0; cb < C; ++cb)
      #pragma unroll
      for (int j = 0; j < 4; ++j)
        #pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float p = __builtin_amdgcn_exp2f(fmaf(x[cb][j][r], kappa[cb], -top[cb]));
          x[cb][j][r] = p;
          weight_sum[cb] += p;
        }
    #pragma unroll
    for (int cb = 0; cb < C; ++cb) asm volatile("" : "+v"(weight_sum[cb]));
    // the weighted sum, group by group
    #pragma unroll
    for (int g = 0; g < NG; ++g) {
      if constexpr (NG > 1) __builtin_amdgcn_sched_barrier(0);
      f16x8 p[C][2];
      #pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float* at = params + (4 * g + 2) * kTile + 16 * j + 4 * quad;
        const f32x4 s = *reinterpret_cast<const f32x4*>(at);
        const f32x4 mn = *reinterpret_cast<const f32x4*>(at + kTile);
        #pragma unroll
        for (int r = 0; r < 4; ++r)
          #pragma unroll
          for (int cb = 0; cb < C; ++cb) {
            offset[cb][g] = fmaf(x[cb][j][r], mn[r], offset[cb][g]);
            p[cb][j / 2][2 * r + j % 2] = (_Float16)(x[cb][j][r] * s[r]);
          }
        #pragma unroll
        for (int cb = 0; cb < C; ++cb) asm volatile("" : "+v"(offset[cb][g]));
      }
      // An error of a rounded weight counts times the code.  8 of each weight as rounded
      // are taken off and 8 as they were put back (offsets are those of code 8), which
      // leaves it times the code less 8.
      #pragma unroll
      for (int cb = 0; cb < C; ++cb) {
        #pragma unroll
        for (int k = 0; k < 8; ++k) {
          const f16x8 v = p[cb][k / 4];
          const f16x2 pair = {v[2 * (k % 4)], v[2 * (k % 4) + 1]};
          const _Float16 one = k & 1 ? 16 : 1;  // an odd token's weight is a 16th
          rounded[cb][g] =
              __builtin_amdgcn_fdot2(pair, f16x2{one, one}, rounded[cb][g], false);
        }
        asm volatile("" : "+v"(rounded[cb][g]));
      }
      #pragma unroll
      for (int d = g * DB / NG; d < (g + 1) * DB / NG; ++d) {
        // 16-byte chunk d / 2 of this lane's row, where the store put it
        const uint8_t* at =
            stage + v_place(16 * (col >> 2) + 4 * quad + (col & 3), d / 2) + 8 * (d & 1);
        const i32x2 v = __builtin_amdgcn_ds_read_tr4_b64_v2i32(
            (__attribute__((address_space(3))) i32x2*)at);
        #pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f16x8 vc = codes_f16((uint32_t)v[h]);
          #pragma unroll
          for (int cb = 0; cb < C; ++cb)
            o[cb][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vc, p[cb][h], o[cb][d], 0, 0, 0);
        }
      }
    }
  };

  for (int tile = first; tile < tile1; tile += kWaves) {
    const unsigned long long have = held;
    const bool stored = have >> lane & 1;
    bool bad = false;
    // ---- V and the parameters into LDS; tokens that are not there have none
    uint32_t big = 0;  // scale of V, as bits
    #pragma unroll
    for (int g = 0; g < NG; ++g) {
      preg[0][g] = stored ? preg[0][g] : 0u;
      preg[1][g] = stored ? preg[1][g] : 0u;
      bad |= not_finite(preg[0][g]) || not_finite(preg[1][g]);
    }
    // tokens that are not finite make the rows that see them not-a-number, and no
    // others: they count as zeros in the products
    const unsigned long long poison = __ballot(bad);
    if (poison) {
      #pragma unroll
      for (int cb = 0; cb < C; ++cb)
        if (seen_tokens(pos[cb], tile * kTile, u.window, poison)) weight_sum[cb] = NAN;
    }
    #pragma unroll
    for (int g = 0; g < NG; ++g) {
      preg[0][g] = bad ? 0u : preg[0][g];
      preg[1][g] = bad ? 0u : preg[1][g];
      big = max(big, preg[1][g] & 0xFFFFu);
    }
    // the largest scale sets the unit of the weights
    const float vbig = low_half(big);
    if (__any(vbig >= ldexpf(1.0f, vexp + 1))) {
      float m = vbig;
      #pragma unroll
      for (int s = 1; s < 64; s <<= 1) m = fmaxf(m, __shfl_xor(m, s));
      const int e = ilogbf(m);
      const float f = ldexpf(1.0f, vexp - e);
      vexp = e;
      // an odd token's weight takes back the 16 of its code
      weight_unit = ldexpf(1.0f, (lane & 1 ? 10 : 14) - e);
      #pragma unroll
      for (int cb = 0; cb < C; ++cb) {
        #pragma unroll
        for (int g = 0; g < NG; ++g) rounded[cb][g] *= f;
        #pragma unroll
        for (int d = 0; d < DB; ++d) o[cb][d] *= f;
      }
    }
    #pragma unroll
    for (int g = 0; g < NG; ++g) {
      float* at = params + 4 * g * kTile + lane;
      at[0] = low_half(preg[0][g]) * a.mantissa;
      at[kTile] = low_half(preg[0][g] >> 16);
      at[2 * kTile] = low_half(preg[1][g]) * weight_unit;
      at[3 * kTile] = fmaf(8.0f, low_half(preg[1][g]), low_half(preg[1][g] >> 16));  // of code 8
    }
    #pragma unroll
    for (int i = 0; i < VL; ++i) {
      const int token = i * (64 / VL) + lane / VL;
      *reinterpret_cast<u32x4*>(stage + v_place(token, lane % VL)) = vreg[i];
    }
    if (tile + kWaves < tile1) {
      if (++ahead == 16) {
        load_pages(tile + kWaves);
        ahead = 0;
      }
      load_v(tile + kWaves, ahead);
    }
    // LDS is this wave's own: its accesses stay in order
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const int t = tile * kTile;
    const bool whole = have == ~0ull && t + kTile - 1 <= pos0 &&
                       (u.window == 0 || t > pos1 - u.window);
    work(tile, whole, have, ahead);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }

  // ---- the four waves' results together
  float* stats = reinterpret_cast<float*>(lds_stats);  // [wave][16 C][2 + NG]
  #pragma unroll
  for (int cb = 0; cb < C; ++cb) {
    float* at = stats + (wave * 16 * C + 16 * cb + col) * (2 + NG);
    const float sum = quad_sum(weight_sum[cb]);
    if (quad == 0) {
      at[0] = top[cb];
      at[1] = sum;
    }
    #pragma unroll
    for (int g = 0; g < NG; ++g) {
      const float v = quad_sum(fmaf(rounded[cb][g], ldexpf(-8.0f, vexp - 14), offset[cb][g]));
      if (quad == 0) at[2 + g] = v;
    }
  }
  __syncthreads();
  // factor of this wave's sums; then everything relative to the common maximum
  float factor[C];
  #pragma unroll
  for (int cb = 0; cb < C; ++cb) {
    float m = kNone;
    #pragma unroll
    for (int k = 0; k < kWaves; ++k)
      m = fmaxf(m, stats[(k * 16 * C + 16 * cb + col) * (2 + NG)]);
    factor[cb] = ldexpf(__builtin_amdgcn_exp2f(top[cb] - m), 24 - 14 + vexp);
  }
  // a thread adds up two channels of C rows, 32 channels of all rows at a time
  const int my_row = threadIdx.x >> 4, my_channel = 2 * (threadIdx.x & 15);
  float my_top[C], my_sum[C], my_offset[C][NG];
  #pragma unroll
  for (int cb = 0; cb < C; ++cb) {
    float m = kNone;
    #pragma unroll
    for (int k = 0; k < kWaves; ++k)
      m = fmaxf(m, stats[(k * 16 * C + 16 * cb + my_row) * (2 + NG)]);
    my_top[cb] = m;
    my_sum[cb] = 0.0f;
    #pragma unroll
    for (int g = 0; g < NG; ++g) my_offset[cb][g] = 0.0f;
    #pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      const float* at = stats + (k * 16 * C + 16 * cb + my_row) * (2 + NG);
      const float f = __builtin_amdgcn_exp2f(at[0] - m);
      my_sum[cb] += f * at[1];
      #pragma unroll
      for (int g = 0; g < NG; ++g) my_offset[cb][g] += f * at[2 + g];
    }
  }
  float* sums = reinterpret_cast<float*>(lds);  // [wave][16 C][OPAD]
  #pragma unroll
  for (int cb = 0; cb < C; ++cb)
    #pragma unroll
    for (int d = 0; d < DB; ++d)
      *reinterpret_cast<f32x4*>(sums + (wave * 16 * C + 16 * cb + col) * OPAD + 16 * d +
                                4 * quad) = o[cb][d] * factor[cb];
  __syncthreads();
  #pragma unroll
  for (int cb = 0; cb < C; ++cb) {
    const int r = 16 * cb + my_row;
    if (r >= rows) continue;
    const float f = my_sum[cb] != 0.0f ? 1.0f / my_sum[cb] : 0.0f;
    const int i = (row0 + r) / u.group, h = (row0 + r) % u.group;
    uint16_t* out =
        a.out + (long long)(w.start + i) * a.out_stride + (head * u.group + h) * D + my_channel;
    const long long at = ((long long)unit.slot * c.kv_heads + head) * u.rows + r;
    if (unit.ranges > 1 && unit.slot >= part.slots) continue;  // no batch that comet.h allows
    #pragma unroll
    for (int d = 0; d < D / 32; ++d) {
      const float off = my_offset[cb][32 * d / G];
      f32x2 v = {off, off};
      #pragma unroll
      for (int k = 0; k < kWaves; ++k)
        v += *reinterpret_cast<const f32x2*>(sums + (k * 16 * C + r) * OPAD + 32 * d + my_channel);
      if (unit.ranges > 1)
        *reinterpret_cast<f32x2*>(part.sums + at * D + 32 * d + my_channel) = v;
      else
        *reinterpret_cast<f16x2*>(out + 32 * d) = f16x2{(_Float16)(v[0] * f), (_Float16)(v[1] * f)};
    }
    if (unit.ranges > 1 && my_channel == 0)
      *reinterpret_cast<f32x2*>(part.stats + at * 2) = f32x2{my_top[cb], my_sum[cb]};
  }
}

// Adds up the ranges of the row blocks that have several: a block takes some rows of
// one (grid x: row block and kv head, y: rows).  D / 4 lanes of four channels make a
// group; a group takes a row, or, the more ranges there are, several take turns at
// those of one.
constexpr int kAhead = 8;  // ranges that a group has in flight

__global__ __launch_bounds__(256) void kv4_attention_combine_kernel(PagedCache c, PagedBatch b,
                                                                    AttentionArgs a,
                                                                    UnitShape few,
                                                                    Partials few_part,
                                                                    UnitShape many,
                                                                    Partials many_part,
                                                                    int few_blocks, int few_rows,
                                                                    int many_rows) {
  __shared__ f32x4 sums[256];
  __shared__ f32x2 stats[256];
  const bool is_few = (int)blockIdx.x < few_blocks;
  const UnitShape u = is_few ? few : many;
  const Partials part = is_few ? few_part : many_part;
  const int index = blockIdx.x - (is_few ? 0 : few_blocks);
  const int my_rows = is_few ? few_rows : many_rows;
  if ((int)blockIdx.y * my_rows >= u.rows) return;
  Unit unit;
  if (!find_unit<true>(b, c.page_shift, u, index / c.kv_heads, &unit)) return;
  // no batch that comet.h allows
  if ((unsigned long long)unit.slot + unit.ranges > part.slots) return;
  const int head = index % c.kv_heads;
  const int D = c.head_dim, lanes = D / 4, groups = 256 / lanes;
  int turns = 1;
  while (turns < groups && turns * kAhead < (int)unit.ranges) turns *= 2;
  const int group = threadIdx.x / lanes, channel = 4 * (threadIdx.x % lanes);
  const int turn = group % turns, at_once = groups / turns;
  const int row0 = unit.block * u.rows + blockIdx.y * my_rows;
  // not those of the next row block, nor behind the sequence's last
  const int rows = min(min(my_rows, u.rows - (int)blockIdx.y * my_rows),
                       unit.w.n * u.group - row0);
  for (int r0 = 0; r0 < rows; r0 += at_once) {
    const int r = r0 + group / turns, row = row0 + r;
    const bool live = r < rows;
    float top = kNone, sum = 0.0f;
    f32x4 v = {0, 0, 0, 0};
    if (live) {
      // the ranges' results lie `step` rows apart
      const long long first =
          ((long long)unit.slot * c.kv_heads + head) * u.rows + blockIdx.y * my_rows + r;
      const long long step = (long long)c.kv_heads * u.rows;
      for (int k = turn; k < (int)unit.ranges; k += kAhead * turns) {
        f32x2 st[kAhead];
        f32x4 x[kAhead];
        #pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          st[i] = f32x2{kNone, 0.0f};
          x[i] = f32x4{0, 0, 0, 0};
          if (k + i * turns < (int)unit.ranges) {
            const long long at = first + (k + i * turns) * step;
            st[i] = *reinterpret_cast<const f32x2*>(part.stats + at * 2);
            x[i] = *reinterpret_cast<const f32x4*>(part.sums + at * D + channel);
          }
        }
        float next = top;
        #pragma unroll
        for (int i = 0; i < kAhead; ++i) next = fmaxf(next, st[i][0]);
        const float f = __builtin_amdgcn_exp2f(top - next);
        top = next;
        sum *= f;
        v *= f;
        #pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const float g = __builtin_amdgcn_exp2f(st[i][0] - top);
          sum += g * st[i][1];
          v += g * x[i];
        }
      }
    }
    if (turns > 1) {
      __syncthreads();
      sums[threadIdx.x] = v;
      stats[threadIdx.x] = f32x2{top, sum};
      __syncthreads();
      float all = kNone;
      for (int k = 0; k < turns; ++k)
        all = fmaxf(all, stats[threadIdx.x + (k - turn) * lanes][0]);
      sum = 0.0f;
      v = f32x4{0, 0, 0, 0};
      for (int k = 0; k < turns; ++k) {
        const f32x2 st = stats[threadIdx.x + (k - turn) * lanes];
        const float f = __builtin_amdgcn_exp2f(st[0] - all);
        sum += f * st[1];
        v += f * sums[threadIdx.x + (k - turn) * lanes];
      }
    }
    if (!live || turn) continue;
    const float f = sum != 0.0f ? 1.0f / sum : 0.0f;
    const f16x2 lo = {(_Float16)(v[0] * f), (_Float16)(v[1] * f)};
    const f16x2 hi = {(_Float16)(v[2] * f), (_Float16)(v[3] * f)};
    const long long m = unit.w.start + row / u.group;
    *reinterpret_cast<u32x2*>(a.out + m * a.out_stride +
                              (head * u.group + row % u.group) * D + channel) =
        u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
  }
}

// ---- host ------------------------------------------------------------------------

// Sequences of up to kFewRows q rows (rows times heads of a group) run on the kernel
// above, the others on the kernel for many rows, whose 128 rows to a block are then
// used by half at least.  Here and there, us:
//   64 rows of 64 users, 2048 tokens   69   92      96 rows of them   99   96
//   64 rows of 16 users, 4096 tokens   43   58      96 rows of them   58   63
//   (32-channel groups, 96 rows of 64 users 162 and 148)
// In narrow launches, whose blocks of 16 rows are fewer than two fifths of the compute
// units, all do: the split along the tokens fills the device, and shorter blocks are
// done sooner.  One user, 8 kv heads:
//   128 rows, 1024 tokens  11.5  19.5     16384 tokens  29.2  31.7
//   192 rows               12.8  19.5                   35.3  40.2
//   (32-channel groups     15.3  24.5                   52.3  53.0)
//   240 rows: no more      13.3  19.6                   44.0  42.6
constexpr int kFewRows = 64;
constexpr int kAny = 0x7FFFFFFF;

// What one of the two kernels does of a batch.
struct Part {
  UnitShape u;
  long long blocks;  // of the grid: units that a batch of these sizes may have, times kv heads
  long long slots;   // partial results
  long long row_blocks;
  int most_rows;     // of one
};

// Blocks of a compute unit: `aim` to aim at, `resident` at a time.  (64-channel blocks
// are one more at a time, but shorter, so that their fixed part counts: aiming at one
// more ran 16 users of 2048 tokens in 17.4 us instead of 15.8.)
Part part_of(const PagedCache& c, const PagedBatch& b, int heads, int window, int cus, int rows,
             int aim, int resident, int low, int high) {
  Part p;
  p.u.group = heads / c.kv_heads;
  p.u.rows = rows;
  p.u.window = window > 1 << 30 ? 0 : window;  // no position is further
  p.u.target = std::max(1, cus * aim / c.kv_heads);
  p.u.at_once = std::max(1, cus * resident / c.kv_heads);
  p.u.low = low;
  p.u.high = high;
  p.most_rows = (int)std::min<long long>(rows, (long long)b.max_rows * p.u.group);
  // every sequence's last row block may be ragged; none has more than `high` rows
  const long long sequences = std::min(b.B, b.M);
  const long long q_rows = (long long)b.M * p.u.group;
  const long long each = (std::min<long long>(high, q_rows) + rows - 1) / rows;
  const long long row_blocks = std::min(q_rows / rows + sequences, sequences * each);
  p.row_blocks = row_blocks;
  const long long tiles = (((long long)b.max_pages << c.page_shift) + kTile - 1) / kTile;
  const long long ranges = (tiles + kMinTiles - 1) / kMinTiles;
  p.slots = ranges > 1 ? std::min<long long>(2 * p.u.target, row_blocks * ranges) : 0;
  p.blocks = std::min(row_blocks + p.u.target, row_blocks * ranges) * c.kv_heads;
  return p;
}

struct Shape {
  Part few, many;
  bool any_few, any_many;
  int columns;  // C of the kernel for few rows
};

Shape shape_of(const PagedCache& c, const PagedBatch& b, int heads, int window, int cus) {
  const long long most = (long long)b.max_rows * (heads / c.kv_heads), blocks16 = (most + 15) / 16;
  const bool narrow = 5 * std::min(b.B, b.M) * blocks16 * c.kv_heads < 2 * cus;
  Shape s;
  s.any_many = !narrow && most > kFewRows;
  // Sequences of few rows among others get a launch of their own, except where most
  // sequences must have about as many rows as the longest: the launch costs 4 us where
  // no sequence is for it (8 prompts of 512 rows: 348 and 344 us without), the kernel for
  // many rows takes 8 us and more for a sequence of one row (4 prompts of 512 rows and
  // 4 single ones: 191 us, 228 without)
  s.any_few = !s.any_many || 4ll * b.M < 3ll * b.B * b.max_rows;
  // 32 rows to a block, which read the tokens once for all of them, where that leaves no
  // block half empty and there are blocks enough (us for 16 and 32 rows to a block: 64
  // users of 2048 tokens and 64 rows 78 and 69, 48 rows 61 and 69; one user of 16384 and
  // 32 rows 17.6 and 19.5), and not next to sequences of many rows, where few rows are
  // mostly one token's (64 users of 8192, 32-channel groups, 8 rows: 167 and 210)
  s.columns = s.any_many || narrow || blocks16 % 2 ? 1 : 2;
  s.few = part_of(c, b, heads, window, cus, 16 * s.columns,
                  resident_few(128, 128, s.columns), resident_few(c.head_dim, c.G, s.columns), 0,
                  s.any_many ? kFewRows : kAny);
  s.many = part_of(c, b, heads, window, cus, kManyRows, 2, 2,
                   s.any_few ? kFewRows : 0, kAny);
  return s;
}

size_t partial_floats(const PagedCache& c, const Part& p) {
  return (size_t)p.slots * c.kv_heads * p.u.rows * (c.head_dim + 2);
}

Partials partials_at(float* at, const PagedCache& c, const Part& p) {
  return {at, at + p.slots * c.kv_heads * p.u.rows * c.head_dim, (uint32_t)p.slots};
}

// The sum over ranges: blocks for the row blocks that may have several (half the slots
// at most, and no more than there are), times kv heads, and how many of a row block's
// rows each takes, so that there are about 1024 in all: each looks its unit up, which
// costs more than some rows one after the other (64 users of 8192 tokens 4.9 us, with
// 2048 blocks 6.3, with 4096 10.6; a chunk of 512 rows 12.4 us, with 512 blocks 13.2).
struct Split {
  unsigned blocks = 0, parts = 0;
  int rows = 1;
};

Split split_of(const PagedCache& c, const Part& p) {
  Split s;
  s.blocks = (unsigned)(std::min(p.slots / 2, p.row_blocks) * c.kv_heads);
  if (!s.blocks) return s;
  s.parts = std::max(1u, std::min((unsigned)p.most_rows, 1024u / s.blocks));
  s.rows = (p.most_rows + s.parts - 1) / s.parts;
  const int at_once = 1024 / c.head_dim;  // rows that a block takes, with few ranges
  if (s.rows > at_once) {
    s.rows = s.rows / at_once * at_once;
    s.parts = (p.most_rows + s.rows - 1) / s.rows;
  }
  return s;
}

template <int D, int G>
void launch_few(const PagedCache& c, const PagedBatch& b, const AttentionArgs& a, const Shape& s,
                const Partials& part, hipStream_t stream) {
  const dim3 grid((unsigned)s.few.blocks), block(64 * kWaves);
  if (s.columns == 1)
    hipLaunchKernelGGL((kv4_attention_few_kernel<D, G, 1>), grid, block, 0, stream, c, b, a,
                       s.few.u, part);
  else
    hipLaunchKernelGGL((kv4_attention_few_kernel<D, G, 2>), grid, block, 0, stream, c, b, a,
                       s.few.u, part);
}

}  // namespace

const char* attention_refusal(const PagedCache& c, const PagedBatch& b, int heads, int cus) {
  // a launch's threads are counted in 32 bits
  const Shape s = shape_of(c, b, heads, 0, cus);
  const bool many = (long long)b.M * heads > 1 << 30 ||
                    std::max(s.few.blocks, s.many.blocks) >= (1ll << 32) / (64 * kWaves);
  return many ? "too many rows, heads and sequences for a launch" : nullptr;
}

size_t attention_workspace(const PagedCache& c, const PagedBatch& b, int heads, int cus) {
  const Shape s = shape_of(c, b, heads, 0, cus);
  return sizeof(float) * ((s.any_few ? partial_floats(c, s.few) : 0) +
                          (s.any_many ? partial_floats(c, s.many) : 0));
}

hipError_t launch_kv4_attention(const PagedCache& c, const PagedBatch& b, const AttentionArgs& args,
                                hipStream_t stream) {
  AttentionArgs a = args;
  a.mantissa = std::frexp(std::fabs(a.scale) * kLog2e, &a.exponent);
  const Shape s = shape_of(c, b, a.heads, a.window, a.cus);
  float* ws = static_cast<float*>(a.workspace);
  const Partials few = partials_at(ws, c, s.few);
  const Partials many = partials_at(ws + (s.any_few ? partial_floats(c, s.few) : 0), c, s.many);
  hipError_t e = hipSuccess;
  if (s.any_many) {
    e = launch_attention_many(c, b, a, s.many.u, many, (unsigned)s.many.blocks, stream);
    if (e != hipSuccess) return e;
  }
  if (s.any_few) {
    if (c.head_dim == 128 && c.G == 128)
      launch_few<128, 128>(c, b, a, s, few, stream);
    else if (c.head_dim == 128 && c.G == 64)
      launch_few<128, 64>(c, b, a, s, few, stream);
    else if (c.head_dim == 128)
      launch_few<128, 32>(c, b, a, s, few, stream);
    else if (c.G == 64)
      launch_few<64, 64>(c, b, a, s, few, stream);
    else
      launch_few<64, 32>(c, b, a, s, few, stream);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const Split fs = s.any_few ? split_of(c, s.few) : Split(),
              ms = s.any_many ? split_of(c, s.many) : Split();
  if (fs.blocks + ms.blocks == 0) return e;
  hipLaunchKernelGGL(kv4_attention_combine_kernel,
                     dim3(fs.blocks + ms.blocks, std::max(fs.parts, ms.parts)), dim3(256), 0, stream,
                     c, b, a, s.few.u, few, s.many.u, many, (int)fs.blocks, fs.rows, ms.rows);
  return hipGetLastError();
}

}  // namespace comet
