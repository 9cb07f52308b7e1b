// rope.hip -- rotary positions of the q and k heads for gfx950.
//
// The pair (a, b) of channels i of every head of row m turns by the angle
// theta_i = positions[m] * freqs[i]:
//   a' = a c - b s,  b' = b c + a s,  c = mscale cos theta, s = mscale sin theta.
// A far position times the fastest frequency is an angle of 1e5 and more, which
// 32 bits hold to 0.01 only: the product and its reduction to half a turn are
// taken in 64 bits, sine and cosine of what is left in 32.
//
// Work decomposition: a lane owns 8 pairs (two 16-byte loads and stores) of one
// frequency range and walks over the heads with them, so that an angle is
// worked out once per row and 8 heads, not once per element.
//
// Bound by HBM on long inputs, 2 bytes in and 2 out per channel: 4001 rows of 72 heads,
// half of each rotated, from a wider buffer into a new one (147 MB): 33 us, 4.46 TB/s, of
// the 4.9 TB/s that a large copy reaches (non-temporal stores: 42 us).  By latency on
// short ones: one row of 40 heads 2.8 us on the device, 5.5 with the call.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "../../include/comet.h"
#include "serving.h"

namespace comet {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
// Heads whose loads a lane has in flight: in place, no load may pass a store, so the
// loads of several heads come first.
constexpr int kAhead = 3;
constexpr double kInvTwoPi = 0.15915494309189533577;

__device__ inline void turn(int position, double freq, float mscale, float* c, float* s) {
  const double t = (double)position * freq * kInvTwoPi;  // turns
  const float r = (float)(t - rint(t));
  sincospif(2.0f * r, s, c);
  *c *= mscale;
  *s *= mscale;
}

__device__ inline float half_bits(uint32_t u) {
  return __half2float(__ushort_as_half((unsigned short)u));
}
__device__ inline uint32_t bits_half(float f) { return __half_as_ushort(__float2half_rn(f)); }

// The pair with values a, b turned by (c, s), as two fp16 numbers.
__device__ inline void rotate(float a, float b, float c, float s, uint32_t* ra, uint32_t* rb) {
  *ra = bits_half(a * c - b * s);
  *rb = bits_half(b * c + a * s);
}

// 16-byte aligned rows, rot_dim a multiple of 16.  A group of `lanes` =
// chunks * head_lanes lanes shares a row: chunk = 8 pairs (for the copied tail:
// 16 channels), head_lanes heads at a time.  blockIdx.y: range of heads.
template <bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a, int chunks, int head_lanes,
                                                        int heads_per_block, int rows_per_block) {
  const int lanes = chunks * head_lanes;
  const int r = threadIdx.x / lanes, t = threadIdx.x % lanes;
  const long long m = (long long)blockIdx.x * rows_per_block + r;
  if (r >= rows_per_block || m >= a.M) return;
  const int chunk = t % chunks;
  const int h0 = blockIdx.y * heads_per_block + t / chunks;
  const int h1 = min(a.heads, ((int)blockIdx.y + 1) * heads_per_block);
  const int half = a.rot_dim / 2;
  const bool tail = chunk >= half / 8;
  // channels of the two vectors
  int ca = 16 * chunk, cb = ca + 8;
  if (!INTERLEAVED && !tail) {
    ca = 8 * chunk;
    cb = ca + half;
  }
  const bool second = cb < a.head_dim;  // the tail may end with one vector
  float c[8], s[8];
  if (!tail) {
    const int position = a.positions[m];
    #pragma unroll
    for (int i = 0; i < 8; ++i)
      turn(position, a.freqs[8 * chunk + i], a.mscale, &c[i], &s[i]);
  }
  const uint16_t* x = a.X + m * a.x_stride;
  uint16_t* o = a.out + m * a.out_stride;
  for (int h = h0; h < h1; h += kAhead * head_lanes) {
    u32x4 va[kAhead], vb[kAhead];
    #pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int hj = h + j * head_lanes;
      if (hj >= h1) break;
      const uint16_t* at = x + hj * a.head_dim;
      va[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at + ca));
      if (second) vb[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at + cb));
    }
    #pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int hj = h + j * head_lanes;
      if (hj >= h1) break;
      u32x4 ra = va[j], rb = vb[j];
      if (!tail) {
        #pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t lo, hi;
          if (INTERLEAVED) {  // dword = one pair
            rotate(half_bits(va[j][i]), half_bits(va[j][i] >> 16), c[i], s[i], &lo, &hi);
            ra[i] = lo | hi << 16;
            rotate(half_bits(vb[j][i]), half_bits(vb[j][i] >> 16), c[4 + i], s[4 + i], &lo, &hi);
            rb[i] = lo | hi << 16;
          } else {
            rotate(half_bits(va[j][i]), half_bits(vb[j][i]), c[2 * i], s[2 * i], &lo, &hi);
            ra[i] = lo;
            rb[i] = hi;
            rotate(half_bits(va[j][i] >> 16), half_bits(vb[j][i] >> 16), c[2 * i + 1],
                   s[2 * i + 1], &lo, &hi);
            ra[i] |= lo << 16;
            rb[i] |= hi << 16;
          }
        }
      }
      *reinterpret_cast<u32x4*>(o + hj * a.head_dim + ca) = ra;
      if (second) *reinterpret_cast<u32x4*>(o + hj * a.head_dim + cb) = rb;
    }
  }
}

// Any even rot_dim and any alignment of fp16: one block per row, one lane per
// pair (or copied channel) of a head.  (On rows that the kernel above takes as well,
// 40 heads in place: 512 rows 8.2 us, 4.8 there; 4096 rows 20.5 and 18.1.)
__global__ __launch_bounds__(kThreads) void rope_any_kernel(RopeArgs a) {
  const long long m = blockIdx.x;
  const int half = a.rot_dim / 2, tail = a.head_dim - a.rot_dim;
  const int per_head = half + tail;
  const int position = a.positions[m];
  const uint16_t* x = a.X + m * a.x_stride;
  uint16_t* o = a.out + m * a.out_stride;
  const bool in_place = a.X == a.out;
  for (int t = threadIdx.x; t < per_head; t += kThreads) {
    if (t >= half) {
      if (in_place) continue;
      const int ch = a.rot_dim + t - half;
      for (int h = blockIdx.y; h < a.heads; h += gridDim.y)
        o[h * a.head_dim + ch] = x[h * a.head_dim + ch];
      continue;
    }
    const int ca = a.interleaved ? 2 * t : t, cb = a.interleaved ? ca + 1 : t + half;
    float c, s;
    turn(position, a.freqs[t], a.mscale, &c, &s);
    for (int h = blockIdx.y; h < a.heads; h += gridDim.y) {
      uint32_t ra, rb;
      rotate(half_bits(x[h * a.head_dim + ca]), half_bits(x[h * a.head_dim + cb]), c, s, &ra, &rb);
      o[h * a.head_dim + ca] = (uint16_t)ra;
      o[h * a.head_dim + cb] = (uint16_t)rb;
    }
  }
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, hipStream_t stream) {
  const uintptr_t where = reinterpret_cast<uintptr_t>(a.X) | reinterpret_cast<uintptr_t>(a.out);
  const bool wide = where % 16 == 0 && a.x_stride % 8 == 0 && a.out_stride % 8 == 0 &&
                    a.head_dim % 8 == 0 && a.rot_dim % 16 == 0;
  if (!wide) {
    const int split = a.M < 2 * a.cus ? std::min(a.heads, 8) : 1;
    hipLaunchKernelGGL(rope_any_kernel, dim3(a.M, split), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
  }
  const bool copy = a.X != a.out;
  const int chunks = a.rot_dim / 16 + (copy ? (a.head_dim - a.rot_dim + 15) / 16 : 0);
  // 8 heads at a time, and as many in all as leave 8 blocks to a compute unit (an
  // angle is worked out once per block)
  const int head_lanes = std::max(1, std::min(std::min(8, a.heads), kThreads / chunks));
  const int rows = std::max(1, kThreads / (chunks * head_lanes));
  const int blocks = (a.M + rows - 1) / rows, turns = (a.heads + head_lanes - 1) / head_lanes;
  int per = std::max(1, std::min(turns, (int)((long long)turns * blocks / (8 * a.cus))));
  if (per > kAhead) per = per / kAhead * kAhead;
  const int heads_per_block = per * head_lanes;
  const dim3 grid((a.M + rows - 1) / rows, (a.heads + heads_per_block - 1) / heads_per_block);
  if (a.interleaved)
    hipLaunchKernelGGL(rope_kernel<true>, grid, dim3(kThreads), 0, stream, a, chunks, head_lanes,
                       heads_per_block, rows);
  else
    hipLaunchKernelGGL(rope_kernel<false>, grid, dim3(kThreads), 0, stream, a, chunks, head_lanes,
                       heads_per_block, rows);
  return hipGetLastError();
}

const char* rope_frequencies(double* freqs, int rot_dim, double base, int scaling, double factor,
                             double low, double high, double original_len, float* mscale) {
  const double two_pi = 6.28318530717958647693;
  if (rot_dim < 2 || rot_dim % 2 || rot_dim > 1024) return "rot_dim must be even, 2 .. 1024";
  if (!(std::isfinite(base) && base > 1.0)) return "base must be finite and above 1";
  if (scaling < COMET_ROPE_NONE || scaling > COMET_ROPE_RAMP) return "unknown scaling";
  const bool blend = scaling == COMET_ROPE_BANDS || scaling == COMET_ROPE_RAMP;
  if (scaling != COMET_ROPE_NONE && !(std::isfinite(factor) && factor >= 1.0))
    return "factor must be finite and at least 1";
  if (scaling == COMET_ROPE_BASE && rot_dim < 4) return "a new base needs rot_dim of at least 4";
  if (blend && !(std::isfinite(low) && std::isfinite(high) && 0.0 < low && low < high))
    return "low and high must be finite with 0 < low < high";
  if (blend && !(std::isfinite(original_len) && original_len >= 1.0))
    return "original_len must be finite and at least 1";
  const int half = rot_dim / 2;
  if (scaling == COMET_ROPE_BASE) base *= std::pow(factor, (double)rot_dim / (rot_dim - 2));
  double first = 0.0, last = 0.0;
  if (scaling == COMET_ROPE_RAMP) {
    auto pair = [&](double turns) {
      return rot_dim * std::log(original_len / (two_pi * turns)) / (2.0 * std::log(base));
    };
    first = std::max(0.0, std::floor(pair(high)));
    last = std::min((double)rot_dim - 1.0, std::ceil(pair(low)));
    if (last - first < 0.001) last = first + 0.001;
  }
  for (int i = 0; i < half; ++i) {
    const double f = std::pow(base, -2.0 * i / rot_dim);
    double t = 1.0;  // share of f that keeps its speed
    if (scaling == COMET_ROPE_LINEAR) t = 0.0;
    if (scaling == COMET_ROPE_BANDS) t = (original_len * f / two_pi - low) / (high - low);
    if (scaling == COMET_ROPE_RAMP) t = 1.0 - (i - first) / (last - first);
    t = std::min(1.0, std::max(0.0, t));
    freqs[i] = t == 1.0 ? f : f * ((1.0 - t) / factor + t);
  }
  if (mscale) *mscale = scaling == COMET_ROPE_RAMP ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
  return nullptr;
}

}  // namespace comet
