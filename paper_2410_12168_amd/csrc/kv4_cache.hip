// kv4_cache.hip -- rows of K and V into the paged 4-bit cache and back, gfx950.
//
// The groups, numbers and encodings are kv4.hip's: per group of G channels of a
// row s = fp16(fp32(max - min) / 15), q = clamp(rint((x - min) / s), 0, 15),
// value = fp16(fp32(q * s) + min).
//
// Work decomposition: a lane owns 8 consecutive channels of one head's row (16
// bytes of fp16, 4 bytes of codes); a block covers the rows that fill its
// lanes and walks over the heads of K and of V.  Neighbouring rows of a
// sequence are neighbours in its page, so for one head a block reads and writes
// runs of rows * head_dim / 2 bytes of codes.  Few rows: the heads are spread
// over blocks as well.
//
// 2 bytes per channel on one side, 0.5 and 4 / G on the other.  Eight ragged prompts of
// up to 4096 rows, 8 heads of 128 channels, 32-channel groups:
//   - append (76 MB): 25 us, 3.0 TB/s of a large copy's 4.9.  Bound by the issue of
//     vector operations, in 95% of the cycles: the run-time sizes' divisions, reductions
//     by lane permutes of run-time length, and two divisions a lane.
//   - gather of contexts of up to 4596 (108 MB): 20.5 us, 5.3 TB/s: HBM, mostly writes.
// The rows of fp16 pass the caches by both ways (both calls 46 us, with gather's plain
// stores 52); the codes do not, since attention reads them next (with append's
// non-temporal stores 49).  16 users' single rows: 9 to 10 us for the two calls, which
// is the calls.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "paged.h"

namespace comet {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
// Heads whose loads a lane has in flight: stores may not be passed by loads, since
// nothing says that they go elsewhere, so the loads of several heads come first.
constexpr int kAhead = 4;

__device__ inline float low_half(uint32_t w) {
  return __half2float(__ushort_as_half((unsigned short)w));
}

// Codes (channel i in bits 4i .. 4i + 3) and {s, min} of a group that the
// `lanes` lanes around this one hold, 8 channels each.
__device__ inline void quantize_group(u32x4 v, int lanes, uint32_t* codes, uint32_t* param) {
  float x[8];
  #pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = low_half(v[i]);
    x[2 * i + 1] = low_half(v[i] >> 16);
  }
  float mn = x[0], mx = x[0];
  #pragma unroll
  for (int i = 1; i < 8; ++i) {
    mn = fminf(mn, x[i]);
    mx = fmaxf(mx, x[i]);
  }
  for (int o = 1; o < lanes; o <<= 1) {
    mn = fminf(mn, __shfl_xor(mn, o));
    mx = fmaxf(mx, __shfl_xor(mx, o));
  }
  // zero extremes as +0: fminf / fmaxf may keep either zero of a +0 / -0 tie
  if (mn == 0.0f) mn = 0.0f;
  if (mx == 0.0f) mx = 0.0f;
  const __half h = __float2half_rn((mx - mn) / 15.0f);
  const float s = __half2float(h);
  const float r = s != 0.0f ? 1.0f / s : 0.0f;  // s == 0 gives q = 0
  uint32_t packed = 0;
  #pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = x[i] - mn;
    const float q0 = a * r;
    // the correctly rounded a / s (Markstein's correction; exact for a binary16 s)
    const float q = fmaf(fmaf(-q0, s, a), r, q0);
    packed |= (uint32_t)fminf(rintf(q), 15.0f) << (4 * i);
  }
  *codes = packed;
  *param = (uint32_t)__half_as_ushort(h) | (uint32_t)__half_as_ushort(__float2half_rn(mn)) << 16;
}

// A block's rows: lane t works on row t / (head_dim / 8), chunk t % (head_dim / 8).
struct Place {
  bool in_row;    // a row of some sequence
  int page;       // -1: a hole
  long long pos;
};

__device__ inline Place place_of(const PagedCache& c, const PagedBatch& b, long long m) {
  Place p{false, -1, 0};
  int seq;
  if (m < b.M && find_row(b, (int)m, &seq, &p.pos)) {
    p.in_row = true;
    p.page = token_page(b, seq, p.pos, c.page_shift, c.num_pages);
  }
  return p;
}

__global__ __launch_bounds__(kThreads) void kv4_append_kernel(PagedCache c, PagedBatch b,
                                                              RowBuffers r, int per_block) {
  const int lanes = c.head_dim / 8;  // of a row
  const int chunk = threadIdx.x % lanes;
  const long long m = (long long)blockIdx.x * (kThreads / lanes) + threadIdx.x / lanes;
  const Place p = place_of(c, b, m);
  if (p.page < 0) return;  // all lanes of a row alike
  const int group = c.G / 8;
  const int last = min(2 * c.kv_heads, ((int)blockIdx.y + 1) * per_block);
  for (int i0 = blockIdx.y * per_block; i0 < last; i0 += kAhead) {
    u32x4 x[kAhead];
    #pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int i = min(i0 + j, last - 1);
      const bool v = i >= c.kv_heads;
      const uint16_t* at = (v ? r.v_in + m * r.v_stride : r.k_in + m * r.k_stride) +
                           (v ? i - c.kv_heads : i) * c.head_dim + 8 * chunk;
      x[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at));
    }
    #pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int i = i0 + j;
      if (i >= last) break;
      const bool v = i >= c.kv_heads;
      uint32_t codes, param;
      quantize_group(x[j], group, &codes, &param);
      const long long row = cache_row(c, p.page, v ? i - c.kv_heads : i, p.pos);
      uint32_t* to = reinterpret_cast<uint32_t*>(v ? c.v_codes : c.k_codes);
      to[row * lanes + chunk] = codes;
      if (chunk % group == 0) {
        uint32_t* params = reinterpret_cast<uint32_t*>(v ? c.v_params : c.k_params);
        params[(row * c.head_dim + 8 * chunk) / c.G] = param;
      }
    }
  }
}

__global__ __launch_bounds__(kThreads) void kv4_gather_kernel(PagedCache c, PagedBatch b,
                                                              RowBuffers r, int first, int heads,
                                                              int per_block) {
  const int lanes = c.head_dim / 8;
  const int chunk = threadIdx.x % lanes;
  const long long m = (long long)blockIdx.x * (kThreads / lanes) + threadIdx.x / lanes;
  const Place p = place_of(c, b, m);
  if (!p.in_row) return;
  const int last = min(heads, ((int)blockIdx.y + 1) * per_block);
  for (int j0 = blockIdx.y * per_block; j0 < last; j0 += kAhead) {
    uint32_t q[kAhead], param[kAhead];
    #pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      q[j] = param[j] = 0;
      if (p.page >= 0) {
        const int i = first + min(j0 + j, last - 1);
        const bool v = i >= c.kv_heads;
        const long long row = cache_row(c, p.page, v ? i - c.kv_heads : i, p.pos);
        q[j] = reinterpret_cast<const uint32_t*>(v ? c.v_codes : c.k_codes)[row * lanes + chunk];
        param[j] = reinterpret_cast<const uint32_t*>(
            v ? c.v_params : c.k_params)[(row * c.head_dim + 8 * chunk) / c.G];
      }
    }
    #pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (j0 + j >= last) break;
      const int i = first + j0 + j;
      const bool v = i >= c.kv_heads;
      const float s = low_half(param[j]), mn = low_half(param[j] >> 16);
      u32x4 o;
      #pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float p0 = (float)((q[j] >> (8 * k)) & 15u) * s;
        const float p1 = (float)((q[j] >> (8 * k + 4)) & 15u) * s;
        o[k] = (uint32_t)__half_as_ushort(__float2half_rn(p0 + mn)) |
               (uint32_t)__half_as_ushort(__float2half_rn(p1 + mn)) << 16;
      }
      uint16_t* x = (v ? r.v_out + m * r.v_stride : r.k_out + m * r.k_stride) +
                    (v ? i - c.kv_heads : i) * c.head_dim + 8 * chunk;
      __builtin_nontemporal_store(o, reinterpret_cast<u32x4*>(x));
    }
  }
}

// Heads (of K and V together) per block: as many as leave 8 blocks to a compute unit,
// whole runs of kAhead where they can be.
int heads_per_block(int heads, int row_blocks, int cus) {
  const int per = std::max(1, std::min(heads, (int)((long long)heads * row_blocks / (8 * cus))));
  return per > kAhead ? per / kAhead * kAhead : per;
}

}  // namespace

hipError_t launch_kv4_append(const PagedCache& c, const PagedBatch& b, const RowBuffers& r,
                             int cus, hipStream_t stream) {
  const int rows = kThreads / (c.head_dim / 8);
  const int blocks = (b.M + rows - 1) / rows, heads = 2 * c.kv_heads;
  const int per = heads_per_block(heads, blocks, cus);
  hipLaunchKernelGGL(kv4_append_kernel, dim3(blocks, (heads + per - 1) / per), dim3(kThreads), 0,
                     stream, c, b, r, per);
  return hipGetLastError();
}

hipError_t launch_kv4_gather(const PagedCache& c, const PagedBatch& b, const RowBuffers& r,
                             int cus, hipStream_t stream) {
  const int rows = kThreads / (c.head_dim / 8);
  const int blocks = (b.M + rows - 1) / rows;
  const int first = r.k_out ? 0 : c.kv_heads;
  const int heads = c.kv_heads * ((r.k_out != nullptr) + (r.v_out != nullptr));
  const int per = heads_per_block(heads, blocks, cus);
  hipLaunchKernelGGL(kv4_gather_kernel, dim3(blocks, (heads + per - 1) / per), dim3(kThreads), 0,
                     stream, c, b, r, first, heads, per);
  return hipGetLastError();
}

}  // namespace comet
