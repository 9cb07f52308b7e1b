// kv4_attention_many.hip -- causal attention over the paged 4-bit cache for
// sequences of many new rows (chunks of prompts), gfx950.
//
// The mathematics is kv4_attention.hip's.  With many rows the same tokens serve
// all of them, so a block of four waves shares a tile of 64 tokens: each code
// becomes an fp16 number in LDS once, and each wave multiplies 32 rows of q with
// the tile (v_mfma_f32_32x32x16_f16; rows: tokens or channels, columns: rows of
// q).  A second tile is staged while one is used.
//
//   - a code c is the fp16 subnormal c * 2^-24, 16 times that for odd channels;
//     q takes the 16 back for K, the output for V.  Eight channels of a dword lie
//     in the order (0, 4, 1, 5, 2, 6, 3, 7) in both tiles.
//   - token 32 t + 8 a + 4 h + r of a tile is row 8 a + 4 h + r of the t-th score
//     product, element 4 a + r of half h of the lanes; V's operand for tokens
//     32 t + 16 u .. + 15 holds 16 u + 8 e + 4 h + r in half h, so again the weights
//     go from one product into the other in place.  V's rows hold channels, its
//     operand tokens: the transposing read (ds_read_b64_tr_b16: 4 rows of 16 fp16)
//     turns them.
//   - 16-byte chunks of a row in LDS change places with the row's number, so that
//     the reads and writes of 16 lanes meet all banks.
//   - the weights are fp16 pairs, and everything that they multiply is (scales and
//     offsets of V) or counts (their sum): two to an operation, with 32-bit sums.  The
//     sums all go by the same rounded weights.  A weight is scaled by 2^6, a scale of V
//     by a power of two that puts the largest so far into [2^8, 2^9): their product stays
//     below 2^15, a weight keeps its 11 bits down to 2^-20 of the largest and is not lost
//     before 2^-30, a scale down to 2^-22 of the largest.  The product of the two is
//     rounded once more.  (The 2^6 go into the exponent of a weight, next to the row's
//     largest score, which has to leave room for them: not so from 2^22 on, where
//     scores are a quarter apart and more and a weight starts at 1.)  (With weights in 32 bits until that product: a chunk of 512
//     rows 366 us, now 357.)
//   - V's codes count around 8 (c - 8 is as exact), 8 w s is added apart: that takes
//     most of the products' rounding away.
//
// 128 rows to a block: with 256 (eight waves) a chunk of 512 rows ran 2.5% faster, but
// ragged prompts of 2048 rows 6% slower: larger blocks work on more masked tokens, and
// there are fewer to fill the device.  Two blocks on a compute unit (71 KB of LDS and
// 256 registers each): one's staging and softmax run beside the other's products.  The
// last row blocks of a sequence see most tokens and come first, so that short ones
// fill the end.
//
// Held by vector operations and products that hardly overlap: per wave and tile of 32
// rows x 64 tokens 34 products, about 345 other vector operations and 32 exponentials
// share a SIMD's issue with the second block's wave.  Vector operations issue in 61% of
// the cycles, the matrix core works in 37%, neither of them full (in a probe, 4 products
// took 62 ns, 32 multiply-adds 78, both together 94: side by side they could issue in
// about 80%).  A chunk of 512 rows over 16384 tokens, 64 heads of 128 channels (270 GFLOP):
// 349 to 361 us, 750 to 776 TFLOP/s; a large fp16 library product reaches 1307.  Prompts
// of up to 2048 rows, four of them, 32 heads, 64-channel groups: 122 us.  Not kept, as 1
// to 5% slower: the weights' sum by a product with a row of ones, scaling and conversion
// of the weights in one operation, the score products of both halves interleaved, the
// first half's scores next to the second's products (registers), s_setprio around the
// score products, blocks in order of their length over all sequences.
#include "attention.h"

namespace comet {

namespace {

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWeightBits = 6, kScaleBits = 8;

// Maximum and sum over the two lanes of a column (l, l ^ 32).
__device__ inline float pair_max(float v) {
  uint32_t a = __float_as_uint(v), b = a;
  swap32(a, b);
  return fmaxf(__uint_as_float(a), __uint_as_float(b));
}
__device__ inline float pair_sum(float v) {
  uint32_t a = __float_as_uint(v), b = a;
  swap32(a, b);
  return __uint_as_float(a) + __uint_as_float(b);
}

template <int D, int G>
__global__ __launch_bounds__(64 * kWaves, 2) void kv4_attention_many_kernel(
    PagedCache c, PagedBatch b, AttentionArgs a, UnitShape u, Partials part) {
  constexpr int NG = D / G;
  constexpr int KS = D / 16;  // steps of the score product
  constexpr int DT = D / 32;  // 32-channel tiles of the output
  constexpr int ROW = D / 2;  // bytes of a row of codes
  constexpr int KD = D / 32;  // dwords of codes that a thread turns into fp16
  constexpr int F = 2 * D;    // bytes of a row of fp16
  // [NG]: K's s [64], V's {s, mn} as fp16, 4 s and 4 mn in turn
  constexpr int PARAMS = 2 * NG * kTile;
  // of each of the two buffers: K, V, K's offsets (rows of 16 fp16), parameters
  constexpr int V_AT = kTile * F, M_AT = 2 * kTile * F, P_AT = M_AT + kTile * 32;
  constexpr int BUF = P_AT + 4 * PARAMS;
  static_assert(BUF % 256 == 0, "chunks of a row change places within 256 bytes");
  __shared__ __attribute__((aligned(256))) uint8_t lds[2 * BUF];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int head = blockIdx.x % c.kv_heads;
  Unit unit;
  if (!find_unit<false>(b, c.page_shift, u, blockIdx.x / c.kv_heads, &unit)) return;
  const SeqWork& w = unit.w;
  const int row0 = unit.block * u.rows;  // of n * group
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

  // ---- this wave's rows
  const int wave_row = 32 * wave;
  const int wave_rows = min(32, rows - wave_row);  // 0 or less: none
  const int wave_pos0 = w.len - w.n + (row0 + wave_row) / u.group;
  const int wave_pos1 = w.len - w.n + (row0 + wave_row + max(wave_rows, 1) - 1) / u.group;
  const bool live = col < wave_rows;
  const int seq_row = (row0 + wave_row + col) / u.group;
  const int q_head = head * u.group + (row0 + wave_row + col) % u.group;
  const int pos = w.len - w.n + seq_row;
  // ---- pages: lane 4 i + k has the slab (page and head) of granule k (16 tokens) of
  // the i-th next tile, or -1
  const int32_t* table = b.block_table + (long long)unit.seq * b.max_pages;
  const bool one_page = c.page_shift >= 6;  // a tile lies in one
  int slabs = -1;
  auto load_pages = [&](int tile) {
    const int i = (tile * kTile + 16 * lane) >> c.page_shift;
    slabs = slab_of(c, head, i < b.max_pages ? table[i] : -1);
  };
  // ---- loads of a tile: a thread takes a quarter of the codes of one token of its
  // wave's granule, and the parameters of token `lane`
  const int token = 16 * wave + (lane & 15), quarter = lane >> 4;
  uint32_t kreg[KD], vreg[KD], preg[2][NG];
  unsigned long long held = 0;  // tokens that are in the cache
  auto load = [&](int tile, int ahead) {
    const int t = tile * kTile;
    int slab[4];
    slab[0] = __builtin_amdgcn_readlane(slabs, 4 * ahead);
    long long row = slab_row(c, slab[0], t), mine = row + (lane & 48);
    row += 16 * wave;
    held = slab[0] >= 0 ? ~0ull : 0;
    if (!one_page) {
      #pragma unroll
      for (int k = 1; k < 4; ++k) slab[k] = __builtin_amdgcn_readlane(slabs, 4 * ahead + k);
      row = slab_row(c, wave < 2 ? (wave ? slab[1] : slab[0]) : (wave == 2 ? slab[2] : slab[3]),
                     t + 16 * wave);
      mine = slab_row(c, quarter < 2 ? (quarter ? slab[1] : slab[0])
                                     : (quarter == 2 ? slab[2] : slab[3]), t + 16 * quarter);
      held = 0;
      #pragma unroll
      for (int k = 0; k < 4; ++k)
        if (slab[k] >= 0) held |= 0xFFFFull << (16 * k);
    }
    const int left = w.len - t;
    if (left < kTile) held &= (1ull << max(left, 0)) - 1;
    const unsigned at = (lane & 15) * ROW + ROW / 4 * quarter;
    if constexpr (KD == 4) {
      const u32x4 k = *reinterpret_cast<const u32x4*>(c.k_codes + row * ROW + at);
      const u32x4 v = *reinterpret_cast<const u32x4*>(c.v_codes + row * ROW + at);
      #pragma unroll
      for (int i = 0; i < 4; ++i) kreg[i] = k[i], vreg[i] = v[i];
    } else {
      const u32x2 k = *reinterpret_cast<const u32x2*>(c.k_codes + row * ROW + at);
      const u32x2 v = *reinterpret_cast<const u32x2*>(c.v_codes + row * ROW + at);
      #pragma unroll
      for (int i = 0; i < 2; ++i) kreg[i] = k[i], vreg[i] = v[i];
    }
    const long long p = (mine + (lane & 15)) * NG;
    #pragma unroll
    for (int g = 0; g < NG; ++g) {
      preg[0][g] = reinterpret_cast<const uint32_t*>(c.k_params)[p + g];
      preg[1][g] = reinterpret_cast<const uint32_t*>(c.v_params)[p + g];
    }
  };

  if (tile0 < tile1) load_pages(tile0);

  f16x8 q[KS];
  float qsum[NG], offset[NG], eights[NG];
  u32x4 raw[KS];
  #pragma unroll
  for (int s = 0; s < KS; ++s) {
    raw[s] = u32x4{0, 0, 0, 0};
    if (live)
      raw[s] = *reinterpret_cast<const u32x4*>(a.Q + (long long)(w.start + seq_row) * a.q_stride +
                                               q_head * D + 16 * s + 8 * half);
  }
  if (tile0 < tile1) load(tile0, 0);  // in flight while q is converted
  float big = 0.0f;
  #pragma unroll
  for (int s = 0; s < KS; ++s)
    #pragma unroll
    for (int k = 0; k < 4; ++k)
      big = fmaxf(big, fmaxf(fabsf(low_half(raw[s][k])), fabsf(low_half(raw[s][k] >> 16))));
  big = pair_max(big);
  int e = kQueryBits;
  if (big > 0.0f && big < INFINITY) e = ilogbf(big);
  // an infinity in q makes the row not-a-number (see kv4_attention.hip)
  const float qf = big < INFINITY ? ldexpf(a.scale < 0.0f ? -1.0f : 1.0f, kQueryBits - e) : NAN;
  // above 0, so that an unseen token's -infinity stays one
  const float kappa = fmaxf(ldexpf(1.0f, a.exponent + 8 + e - kQueryBits), 0x1p-120f);
  #pragma unroll
  for (int g = 0; g < NG; ++g) qsum[g] = offset[g] = eights[g] = 0.0f;
  #pragma unroll
  for (int s = 0; s < KS; ++s) {
    float v[8];
    float sum = 0.0f;
    #pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = low_half(raw[s][k]) * qf;
      v[2 * k + 1] = low_half(raw[s][k] >> 16) * qf;
      sum += v[2 * k] + v[2 * k + 1];
    }
    qsum[16 * s / G] += sum;
    q[s] = f16x8{(_Float16)v[0],            (_Float16)v[4],
                 (_Float16)(v[1] * 0.0625f), (_Float16)(v[5] * 0.0625f),
                 (_Float16)v[2],            (_Float16)v[6],
                 (_Float16)(v[3] * 0.0625f), (_Float16)(v[7] * 0.0625f)};
  }
  // The offsets' part of a score, sum_g mn_g (sum q)_g, is a step of the score product
  // of its own: three fp16 numbers that add up to (sum q)_g * 2^-8, each against mn_g
  // (off by 2^-33 of the sum or, where that is small, by fp16's smallest steps: 2^-30 of
  // the row's largest value at most).
  f16x8 qsums;
  {
    f16x8 low = {0, 0, 0, 0, 0, 0, 0, 0}, high = low;  // of the halves of the lanes
    #pragma unroll
    for (int g = 0; g < NG; ++g) {
      float rest = pair_sum(qsum[g]) * (0x1p-8f * a.mantissa);
      #pragma unroll
      for (int i = 3 * g; i < 3 * g + 3; ++i) {
        const _Float16 part = (_Float16)rest;
        rest -= (float)part;
        if (i < 8)
          low[i % 8] = part;
        else
          high[i % 8] = part;
      }
    }
    const u32x4 lo = __builtin_bit_cast(u32x4, low), hi = __builtin_bit_cast(u32x4, high);
    u32x4 mine;
    #pragma unroll
    for (int i = 0; i < 4; ++i) mine[i] = half ? hi[i] : lo[i];
    qsums = __builtin_bit_cast(f16x8, mine);
  }
  float top = kNone, weight_sum = 0.0f;
  f32x16 o[DT];
  #pragma unroll
  for (int d = 0; d < DT; ++d)
    #pragma unroll
    for (int k = 0; k < 16; ++k) o[d][k] = 0.0f;
  int vexp = -24;  // the exponent below that `o` goes by

  // The exponent of a row's largest weight.
  auto lift = [](float top) { return fabsf(top) < 0x1p22f ? (float)kWeightBits : 0.0f; };

  // Where a 16-byte chunk (8 channels) of a token lies in LDS.
  auto k_place = [](int t, int chunk) {
    return t * F + 16 * (chunk ^ (D == 128 ? t & 15 : t >> 1 & 7));
  };
  auto v_place = [](int t, int chunk) {
    const int turn = D == 128 ? 4 * (t & 3) + (t >> 2 & 3) : 4 * (t >> 1 & 1) + (t >> 2 & 3);
    return t * F + 16 * (chunk ^ turn);
  };

  // ---- the loaded tile into LDS.  The scale of the weights follows the largest scale
  // of V so far, 2^exponent or more below 2^(exponent + 1): `limit` is that as fp16 bits.
  const int k_to = k_place(token, KD * quarter), v_to = V_AT + v_place(token, KD * quarter);
  int exponent = -24;
  uint32_t limit = 2;
  float scale_unit = ldexpf(1.0f, kScaleBits - exponent);
  unsigned long long poison_next = 0;
  // codes: 2 KD pieces, K's and V's in turn
  auto stage_codes = [&](int buf, int piece) {
    const int to = piece & 1 ? v_to : k_to, i = piece / 2;
    *reinterpret_cast<f16x8*>(lds + (buf + to ^ 16 * i)) =
        piece & 1 ? centered_f16(vreg[i]) : codes_f16(kreg[i]);
  };
  auto stage_params = [&](int buf) {
    const bool stored = held >> lane & 1;
    uint32_t bits = 0, wild = 0;
    #pragma unroll
    for (int g = 0; g < NG; ++g) {
      preg[0][g] = stored ? preg[0][g] : 0u;
      preg[1][g] = stored ? preg[1][g] : 0u;
      bits = max(bits, preg[1][g] & 0xFFFFu);
      // an exponent of all ones carries into the sign
      wild |= (preg[0][g] & 0x7C007C00u) + 0x04000400u;
      wild |= (preg[1][g] & 0x7C007C00u) + 0x04000400u;
    }
    // tokens that are not finite make the rows that see them not-a-number, and no
    // others: they count as zeros in the products
    const bool bad = wild & 0x80008000u;
    poison_next = __ballot(bad);
    if (poison_next) {
      bits = bad ? 0u : bits;
      #pragma unroll
      for (int g = 0; g < NG; ++g) {
        preg[0][g] = bad ? 0u : preg[0][g];
        preg[1][g] = bad ? 0u : preg[1][g];
      }
    }
    if (__any(bits >= limit)) {
      uint32_t m = bits;
      #pragma unroll
      for (int s = 1; s < 64; s <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, s));
      exponent = __builtin_amdgcn_readfirstlane(ilogbf(low_half(m)));
      limit = exponent >= -15 ? (uint32_t)(exponent + 16) << 10 : 1u << (exponent + 25);
      scale_unit = ldexpf(1.0f, kScaleBits - exponent);
    }
    // the waves take turns at the parameters, which all of them have
    float* at = reinterpret_cast<float*>(lds + buf + P_AT) + lane;
    _Float16* v_at = reinterpret_cast<_Float16*>(lds + buf + P_AT) + 8 * (lane >> 2) + (lane & 3);
    #pragma unroll
    for (int g = 0; g < NG; ++g) {
      if (wave == 0) at[2 * g * kTile] = low_half(preg[0][g]) * (65536.0f * a.mantissa);
      if (wave == 1)
        v_at[2 * (2 * g + 1) * kTile] = (_Float16)(low_half(preg[1][g]) * scale_unit);
      if (wave == 2)
        v_at[2 * (2 * g + 1) * kTile + 4] =
            __builtin_bit_cast(_Float16, (unsigned short)(preg[1][g] >> 16));
    }
    if (wave == 3) {
      uint32_t* m = reinterpret_cast<uint32_t*>(lds + buf + M_AT + 32 * lane);
      uint32_t mn[NG];
      #pragma unroll
      for (int g = 0; g < NG; ++g) mn[g] = preg[0][g] >> 16;
      #pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int g0 = 2 * i / 3, g1 = (2 * i + 1) / 3;
        m[i] = (g0 < NG ? mn[g0 % NG] : 0) | (g1 < NG ? mn[g1 % NG] << 16 : 0);
      }
    }
  };

  // ---- 32 rows of q times a tile
  const int lane16 = lane & 15;
  // this lane's chunk 0 of K's row `col`, and of V's row for the transposing reads;
  // other chunks differ by exclusive or
  const int k_at = k_place(col, half);
  const int v_at = V_AT + v_place(4 * half + (lane16 >> 2),
                                  2 * (lane >> 4 & 1) + (lane16 >> 1 & 1)) + 8 * (lane16 & 1);
  constexpr int AHEAD = NG == 1 ? 8 : 4;  // operands of K that are read ahead
  f16x8 k[AHEAD], mn;
  auto k_operand = [&](int buf, int n) {  // of the n-th step, over both halves of the tile
    return *reinterpret_cast<const f16x8*>(lds + (buf + k_at ^ 32 * (n % KS)) + n / KS * 32 * F);
  };
  auto mn_operand = [&](int buf, int t) {
    return *reinterpret_cast<const f16x8*>(lds + buf + M_AT + 32 * (32 * t + col) + 16 * half);
  };
  auto work = [&](int buf, int tile, unsigned long long have, unsigned long long poison) {
    const int t0 = tile * kTile;
    const float* params = reinterpret_cast<const float*>(lds + buf + P_AT);
    if (poison && seen_tokens(pos, t0, u.window, poison)) weight_sum = NAN;
    // The order below is the intended one: next to each product stand the reads of a
    // later one and other arithmetic, which run while the matrix core works (the
    // next tile's codes, the first half's scores).
    f32x16 x[2];
    f32x16 zero;
    #pragma unroll
    for (int i = 0; i < 16; ++i) zero[i] = 0.0f;
    #pragma unroll
    for (int t = 0; t < 2; ++t) {
      __builtin_amdgcn_sched_barrier(0);
      x[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(mn, qsums, zero, 0, 0, 0);
      if (t == 0) mn = mn_operand(buf, 1);
      #pragma unroll
      for (int g = 0; g < NG; ++g) {
        f32x16 d = zero;
        #pragma unroll
        for (int s = g * KS / NG; s < (g + 1) * KS / NG; ++s) {
          const int n = t * KS + s;
          d = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[n % AHEAD], q[s], d, 0, 0, 0);
          if (n + AHEAD < 2 * KS) k[n % AHEAD] = k_operand(buf, n + AHEAD);
          if (n % 2 == 0) {
            #pragma unroll
            for (int i = n / 2 * 2 * KD / KS; i < (n / 2 + 1) * 2 * KD / KS; ++i)
              stage_codes(BUF - buf, i);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        #pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 scale = *reinterpret_cast<const f32x4*>(params + 2 * g * kTile + 32 * t +
                                                              8 * i + 4 * half);
          #pragma unroll
          for (int r = 0; r < 4; ++r)
            x[t][4 * i + r] = fmaf(scale[r], d[4 * i + r], x[t][4 * i + r]);
        }
        // done here (see kv4_attention.hip); with one group the scheduler may put the
        // first half's off until the second's products run
        if (NG > 1 || t == 1) asm volatile("" : "+v"(x[t]));
      }
    }
    if (NG == 1) asm volatile("" : "+v"(x[0]));
    // V's operand for 16 tokens of a 32-channel tile
    auto v_operand = [&](int st, int d) {
      i16x4 v[2];
      #pragma unroll
      for (int i = 0; i < 2; ++i) {
        v[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) i16x4*)(lds + (buf + v_at ^ 64 * d + 32 * i) +
                                                       (16 * st + 8 * i) * F));
      }
      return __builtin_bit_cast(f16x8,
                                __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    f16x8 v[DT];
    #pragma unroll
    for (int d = 0; d < DT; ++d) v[d] = v_operand(0, d);
    u32x4 pairs[2];  // V's {s, mn} of the next operand
    auto load_pairs = [&](int st, int g) {
      #pragma unroll
      for (int i = 0; i < 2; ++i)
        pairs[i] = *reinterpret_cast<const u32x4*>(params + (2 * g + 1) * kTile + 16 * st +
                                                   8 * i + 4 * half);
    };
    load_pairs(0, 0);
    __builtin_amdgcn_sched_barrier(0);
    const bool whole = have == ~0ull && t0 + kTile - 1 <= wave_pos0 &&
                       (u.window == 0 || t0 > wave_pos1 - u.window);
    if (!whole) {
      const unsigned long long seen = seen_tokens(pos, t0, u.window, have) >> (4 * half);
      #pragma unroll
      for (int t = 0; t < 2; ++t)
        #pragma unroll
        for (int k = 0; k < 16; ++k)
          if (!((uint32_t)(seen >> 32 * t) >> (8 * (k / 4) + k % 4) & 1u)) x[t][k] = -INFINITY;
    }
    // running maximum; what was added up before shrinks with it
    float m = x[0][0];
    #pragma unroll
    for (int k = 1; k < 32; ++k) m = fmaxf(m, x[k / 16][k % 16]);
    const float next = fmaxf(top, pair_max(m) * kappa);
    if (__any(next > top)) {
      const float f = __builtin_amdgcn_exp2f(top - next + (lift(next) - lift(top)));
      top = next;
      weight_sum *= f;
      #pragma unroll
      for (int g = 0; g < NG; ++g) {
        offset[g] *= f;
        eights[g] *= f;
      }
      #pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= f;
    }
    // the weighted sum, 16 tokens at a time; the weights of the next 16 are worked out
    // next to the products of these
    // one value of `top` from here on: known to be lift's of the branch above on some
    // paths, it costs 38 spilled registers
    asm volatile("" : "+v"(top));
    const float shift = lift(top) - top;
    const f16x2 ones = {1, 1};
    f16x2 wt[2][4];  // of 16 tokens and the next: pairs of the 8 that this half has
    auto weights = [&](int st, int i) {  // of tokens 8 i + 4 half .. + 3 of the 16
      #pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int k = 8 * (st & 1) + 4 * i + 2 * r;
        const f16x2 w =
            f16x2{(_Float16)__builtin_amdgcn_exp2f(fmaf(x[st / 2][k], kappa, shift)),
                  (_Float16)__builtin_amdgcn_exp2f(fmaf(x[st / 2][k + 1], kappa, shift))};
        wt[st & 1][2 * i + r] = w;
        weight_sum = __builtin_amdgcn_fdot2(w, ones, weight_sum, false);
      }
      asm volatile("" : "+v"(weight_sum));  // here and not after the products
    };
    auto operand = [&](int st, int g) {
      u32x4 p;
      #pragma unroll
      for (int i = 0; i < 2; ++i) {
        const u32x4 v = pairs[i];
        #pragma unroll
        for (int r = 0; r < 2; ++r) {
          const uint32_t sr = v[r], mr = v[2 + r];
          const f16x2 s = __builtin_bit_cast(f16x2, sr), m = __builtin_bit_cast(f16x2, mr);
          const f16x2 w = wt[st & 1][2 * i + r], ws = w * s;
          offset[g] = __builtin_amdgcn_fdot2(w, m, offset[g], false);
          eights[g] = __builtin_amdgcn_fdot2(w, s, eights[g], false);
          p[2 * i + r] = __builtin_bit_cast(uint32_t, ws);
        }
      }
      asm volatile("" : "+v"(offset[g]), "+v"(eights[g]));
      return __builtin_bit_cast(f16x8, p);
    };
    __builtin_amdgcn_s_setprio(1);  // the part with most products first
    weights(0, 0);
    weights(0, 1);
    f16x8 p = operand(0, 0);
    #pragma unroll
    for (int st = 0; st < 4; ++st) {
      #pragma unroll
      for (int g = 0; g < NG; ++g) {
        f16x8 p_next = p;
        #pragma unroll
        for (int d = g * DT / NG; d < (g + 1) * DT / NG; ++d) {
          __builtin_amdgcn_sched_barrier(0);
          if (d == g * DT / NG) {
            if (g + 1 < NG)
              load_pairs(st, g + 1);
            else if (st < 3)
              load_pairs(st + 1, 0);
          }
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[d], p, o[d], 0, 0, 0);
          if (st < 3) {
            v[d] = v_operand(st + 1, d);
            if (d % (DT / 2) == 0) weights(st + 1, d / (DT / 2));
          }
        }
        // the next operand: the next group's, or the first of the next 16 tokens
        if (g + 1 < NG)
          p_next = operand(st, g + 1);
        else if (st < 3)
          p_next = operand(st + 1, 0);
        p = p_next;
      }
    }
    __builtin_amdgcn_s_setprio(0);
  };

  if (tile0 < tile1) {
    stage_params(0);
    #pragma unroll
    for (int i = 0; i < 2 * KD; ++i) stage_codes(0, i);
    int exponent_now = exponent;  // of the tile in work
    unsigned long long have = held, poison = poison_next;
    if (tile0 + 1 < tile1) load(tile0 + 1, 1);
    int ahead = 1;  // where in `pages` the loaded tile is
    for (int tile = tile0; tile < tile1; ++tile) {
      int buf = (tile - tile0) & 1 ? BUF : 0;
      // worked out anew for each tile: the addresses of both buffers would take the
      // registers of q
      asm volatile("" : "+s"(buf));
      __syncthreads();  // the tile is in LDS, and the other buffer is free
      mn = mn_operand(buf, 0);
      #pragma unroll
      for (int n = 0; n < AHEAD; ++n) k[n] = k_operand(buf, n);
      // the next tile is staged on the way (after the last one, once more to no end)
      if (tile + 1 < tile1) stage_params(BUF - buf);
      const unsigned long long have_next = held;
      // a wave whose rows see nothing of the tile works on it like the others: a second
      // path for it would cost the first one its registers
      if (exponent_now != vexp) {
        const float f = ldexpf(1.0f, vexp - exponent_now);
        vexp = exponent_now;
        #pragma unroll
        for (int g = 0; g < NG; ++g) eights[g] *= f;
        #pragma unroll
        for (int d = 0; d < DT; ++d) o[d] *= f;
      }
      work(buf, tile, have, poison);
      if (tile + 2 < tile1) {
        if (++ahead == 16) {
          load_pages(tile + 2);
          ahead = 0;
        }
        load(tile + 2, ahead);
      }
      exponent_now = exponent;
      have = have_next;
      poison = poison_next;
    }
  }

  // ---- out: element 4 i + r of half h is channel (0, 4, 1, 5)[r] + 2 h of chunk
  // 4 d + i; two chunks change halves, so that a lane has the 8 channels of one
  const float even = lift(top) != 0.0f ? 1.0f : ldexpf(1.0f, kWeightBits);  // alike in all ranges
  const float sum = pair_sum(weight_sum) * even;
  const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
  const float factor = ldexpf(even, 24 - kScaleBits + vexp);
  #pragma unroll
  for (int g = 0; g < NG; ++g)
    offset[g] = even * pair_sum(fmaf(eights[g], ldexpf(8.0f, vexp - kScaleBits), offset[g]));
  const bool partial = unit.ranges > 1;
  if (partial && unit.slot >= part.slots) return;  // no batch that comet.h allows
  const long long at =
      ((long long)unit.slot * c.kv_heads + head) * u.rows + wave_row + col;
  if (partial && live && half == 0)
    *reinterpret_cast<f32x2*>(part.stats + at * 2) = f32x2{top, sum};
  uint16_t* out = a.out + (long long)(w.start + seq_row) * a.out_stride + q_head * D;
  #pragma unroll
  for (int d = 0; d < DT; ++d)
    #pragma unroll
    for (int i = 0; i < 4; i += 2) {
      float lo[4], hi[4];
      #pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float f = r < 2 ? factor : factor * 0.0625f;
        uint32_t va = __float_as_uint(fmaf(o[d][4 * i + r], f, offset[32 * d / G]));
        uint32_t vb = __float_as_uint(fmaf(o[d][4 * i + 4 + r], f, offset[32 * d / G]));
        swap32(va, vb);
        lo[r] = __uint_as_float(va);
        hi[r] = __uint_as_float(vb);
      }
      if (live) {
        const int channel = 8 * (4 * d + i + half);
        const f32x4 y0 = {lo[0], lo[2], hi[0], hi[2]}, y1 = {lo[1], lo[3], hi[1], hi[3]};
        if (partial) {
          *reinterpret_cast<f32x4*>(part.sums + at * D + channel) = y0;
          *reinterpret_cast<f32x4*>(part.sums + at * D + channel + 4) = y1;
        } else {
          f16x8 y;
          #pragma unroll
          for (int k = 0; k < 4; ++k) {
            y[k] = (_Float16)(y0[k] * inv);
            y[4 + k] = (_Float16)(y1[k] * inv);
          }
          *reinterpret_cast<f16x8*>(out + channel) = y;
        }
      }
    }
}

template <int D, int G>
void launch(const PagedCache& c, const PagedBatch& b, const AttentionArgs& a, const UnitShape& u,
            const Partials& part, unsigned blocks, hipStream_t stream) {
  hipLaunchKernelGGL((kv4_attention_many_kernel<D, G>), dim3(blocks), dim3(64 * kWaves), 0, stream,
                     c, b, a, u, part);
}

}  // namespace

hipError_t launch_attention_many(const PagedCache& c, const PagedBatch& b, const AttentionArgs& a,
                                 const UnitShape& u, const Partials& part, unsigned blocks,
                                 hipStream_t stream) {
  if (c.head_dim == 128 && c.G == 128)
    launch<128, 128>(c, b, a, u, part, blocks, stream);
  else if (c.head_dim == 128 && c.G == 64)
    launch<128, 64>(c, b, a, u, part, blocks, stream);
  else if (c.head_dim == 128)
    launch<128, 32>(c, b, a, u, part, blocks, stream);
  else if (c.G == 64)
    launch<64, 64>(c, b, a, u, part, blocks, stream);
  else
    launch<64, 32>(c, b, a, u, part, blocks, stream);
  return hipGetLastError();
}

}  // namespace comet
