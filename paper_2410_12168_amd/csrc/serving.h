// serving.h -- internal launchers of the operators between a layer's qkv and o
// products: rotary positions, the paged 4-bit K/V cache and attention over it
// (not part of the public C ABI; see include/comet.h for that).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace comet {

struct RopeArgs {
  const uint16_t* X;
  const int32_t* positions;
  const double* freqs;
  uint16_t* out;
  int M, heads, head_dim, rot_dim;
  int x_stride, out_stride;
  bool interleaved;
  float mscale;
  int cus;
};
hipError_t launch_rope(const RopeArgs& a, hipStream_t stream);
// Host: frequencies and *mscale; nullptr on success, else a message.
const char* rope_frequencies(double* freqs, int rot_dim, double base, int scaling, double factor,
                             double low, double high, double original_len, float* mscale);

// A paged cache and a ragged batch as the kernels read them (comet.h has the
// layouts).
struct PagedCache {
  uint8_t* k_codes;
  uint16_t* k_params;
  uint8_t* v_codes;
  uint16_t* v_params;
  int num_pages;
  int page_shift;  // log2 of the tokens of a page
  int kv_heads;
  int head_dim;
  int G;
};
struct PagedBatch {
  const int32_t* row_start;
  const int32_t* seq_lens;
  const int32_t* block_table;
  int B, M, max_pages, max_rows;
};

// Rows [M] of K and V into the cache, and back.
struct RowBuffers {
  const uint16_t* k_in;
  const uint16_t* v_in;
  uint16_t* k_out;
  uint16_t* v_out;
  int k_stride, v_stride;
};
hipError_t launch_kv4_append(const PagedCache& c, const PagedBatch& b, const RowBuffers& r,
                             int cus, hipStream_t stream);
hipError_t launch_kv4_gather(const PagedCache& c, const PagedBatch& b, const RowBuffers& r,
                             int cus, hipStream_t stream);

struct AttentionArgs {
  const uint16_t* Q;
  uint16_t* out;
  int heads;
  int q_stride, out_stride;
  float scale;
  int window;
  void* workspace;
  int cus;
  // |scale| * log2(e) as mantissa * 2^exponent, for the kernels (the launcher's own)
  float mantissa = 0.0f;
  int exponent = 0;
};
// nullptr, or why these sizes cannot run.
const char* attention_refusal(const PagedCache& c, const PagedBatch& b, int heads, int cus);
size_t attention_workspace(const PagedCache& c, const PagedBatch& b, int heads, int cus);
hipError_t launch_kv4_attention(const PagedCache& c, const PagedBatch& b, const AttentionArgs& a,
                                hipStream_t stream);

}  // namespace comet
