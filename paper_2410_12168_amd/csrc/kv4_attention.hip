// kv4_attention.hip -- causal attention of new rows over the paged 4-bit cache,
// gfx950.
//
// Row i of sequence b, q head h, at position p = L_b - n_b + i:
//   x_j = scale * q . k_j,  out = sum_j exp(x_j) v_j / sum_j exp(x_j)
// over the tokens j <= p that the row sees, with the cached value q s + mn of a
// code.  A group's scale and offset are taken out of the sums:
//   q . k_j = sum_g s_jg (q . codes_j)_g + mn_jg (sum q)_g
//   sum_j w_j v_j = sum_j (w_j s_j) codes_j + sum_j w_j mn_j
// One pass over the tokens with the running maximum and sum of the softmax.
//
// Work decomposition: one wave per row and head, 64 tokens at a time: a lane per
// token for the scores, a lane per channel pair for the weighted sum.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged.h"

namespace comet {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;

__device__ inline float low_half(uint32_t w) {
  return __half2float(__ushort_as_half((unsigned short)w));
}

__device__ inline float wave_max(float v) {
  #pragma unroll
  for (int o = 1; o < 64; o <<= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}

__device__ inline float wave_sum(float v) {
  #pragma unroll
  for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
  return v;
}

__global__ __launch_bounds__(64) void kv4_attention_row_kernel(PagedCache c, PagedBatch b,
                                                               AttentionArgs a) {
  __shared__ float q[128];
  __shared__ float weight[64];
  __shared__ int pages[64];
  const int lane = threadIdx.x, h = blockIdx.y;
  const int m = blockIdx.x;
  int seq;
  long long p;
  if (!find_row(b, m, &seq, &p)) return;
  const int D = c.head_dim, G = c.G, head = h / (a.heads / c.kv_heads);
  const uint16_t* x = a.Q + (long long)m * a.q_stride + h * D;
  for (int i = lane; i < D; i += 64) q[i] = low_half(x[i]);
  __syncthreads();
  const long long end = min(p + 1, (long long)b.max_pages << c.page_shift);
  const long long begin = a.window > 0 ? max(0ll, p - a.window + 1) : 0;
  float top = -INFINITY, sum = 0.0f, o0 = 0.0f, o1 = 0.0f;
  for (long long j0 = begin; j0 < end; j0 += 64) {
    const long long j = j0 + lane;
    const int page = j < end ? token_page(b, seq, j, c.page_shift, c.num_pages) : -1;
    float score = -INFINITY;
    if (page >= 0) {
      const long long row = cache_row(c, page, head, j);
      const uint32_t* codes = reinterpret_cast<const uint32_t*>(c.k_codes) + row * (D / 8);
      const uint32_t* params = reinterpret_cast<const uint32_t*>(c.k_params) + row * (D / G);
      score = 0.0f;
      for (int g = 0; g < D / G; ++g) {
        float dot = 0.0f, qs = 0.0f;
        for (int w = 0; w < G / 8; ++w) {
          const uint32_t v = codes[g * (G / 8) + w];
          #pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float e = q[g * G + 8 * w + i];
            dot = fmaf((float)((v >> (4 * i)) & 15u), e, dot);
            qs += e;
          }
        }
        score += low_half(params[g]) * dot + low_half(params[g] >> 16) * qs;
      }
      score *= a.scale * kLog2e;
    }
    const float next = fmaxf(top, wave_max(score));
    const float shrink = next == top ? 1.0f : exp2f(top - next);
    const float w = page >= 0 ? exp2f(score - next) : 0.0f;
    __syncthreads();
    weight[lane] = w;
    pages[lane] = page;
    __syncthreads();
    sum = sum * shrink + wave_sum(w);
    top = next;
    o0 *= shrink;
    o1 *= shrink;
    const int n = (int)min(64ll, end - j0);
    if (lane < D / 2) {
      for (int t = 0; t < n; ++t) {
        if (pages[t] < 0) continue;
        const long long row = cache_row(c, pages[t], head, j0 + t);
        const uint32_t v = c.v_codes[row * (D / 2) + lane];
        const uint32_t param =
            reinterpret_cast<const uint32_t*>(c.v_params)[row * (D / G) + 2 * lane / G];
        const float s = low_half(param), mn = low_half(param >> 16);
        o0 = fmaf(weight[t], fmaf((float)(v & 15u), s, mn), o0);
        o1 = fmaf(weight[t], fmaf((float)(v >> 4), s, mn), o1);
      }
    }
  }
  if (lane < D / 2) {
    const float r = sum != 0.0f ? 1.0f / sum : 0.0f;
    const uint32_t lo = __half_as_ushort(__float2half_rn(o0 * r));
    const uint32_t hi = __half_as_ushort(__float2half_rn(o1 * r));
    reinterpret_cast<uint32_t*>(a.out + (long long)m * a.out_stride + h * D)[lane] = lo | hi << 16;
  }
}

}  // namespace

size_t attention_workspace(const PagedCache&, const PagedBatch&, int, int) { return 0; }

hipError_t launch_kv4_attention(const PagedCache& c, const PagedBatch& b, const AttentionArgs& a,
                                hipStream_t stream) {
  hipLaunchKernelGGL(kv4_attention_row_kernel, dim3(b.M, a.heads), dim3(64), 0, stream, c, b, a);
  return hipGetLastError();
}

}  // namespace comet
