// Internal interface of the 8-bit paged cache (qcache_*.hip) and the layout of its
// pages: codes [L][2][P][H][B][d], one OCP e4m3 number a byte, and scales [L][2][P][H].
#pragma once

#include "internal.h"

namespace cm {

struct QCacheDesc {
  int32_t L, H, d, b_shift;  // B = 1 << b_shift
  int64_t pages;
  uint8_t* codes;
  float* scales;
  __host__ __device__ int64_t slice_codes() const { return ((pages * H) << b_shift) * d; }  // of one (layer, K/V)
  __host__ __device__ int64_t slice_scales() const { return pages * H; }
};

// Rows of K or V of a step (cm_qrows), strides in bytes.
struct QRows {
  const uint8_t* data;
  int64_t layer, token, head;
};

// What the attention kernels read and write (strides in elements).
struct QAttention {
  const uint8_t* kc;  // the layer's codes and scales
  const uint8_t* vc;
  const float* ks;
  const float* vs;
  int64_t pages;
  int32_t H, G, b_shift, n;
  const void* q;
  int64_t q_row, q_head;
  void* out;
  int64_t out_row, out_head;
  float* lse;
  const int32_t* rows;
  const int32_t* lens;
  const int32_t* table;
  int64_t width;
  int64_t n_rows;
  int32_t max_rows, window;
  float scale_log2;   // |softmax scale| * log2(e)
  int32_t negate;     // the softmax scale is negative
  // For requests of few query rows and of many: the spans (few) or items (many) that their
  // contexts are cut into for each KV head, places of partial results for each KV head,
  // where they are, [H][few_max] and [H][many_places], and the counters of those for few,
  // [H][few_max][2]; the most items of many rows for each KV head.
  int32_t few_items, few_max, many_items, many_max, many_places;
  float* few_part;
  float* many_part;
  void* many_found;   // the items of many rows that have a place, [many_places]
  int32_t* few_count;
  int32_t few_unit;   // tokens by which few rows' contexts are cut
};

hipError_t launch_qcache_tables(int64_t pages, int32_t b_shift, int32_t n, const int32_t* held,
                                const int32_t* fresh, const int32_t* free_pages, int64_t n_free,
                                int32_t* table, int64_t width, int64_t n_tokens, int64_t* slots,
                                int32_t* rows, int32_t* lens, int64_t* info, hipStream_t stream);
hipError_t launch_qcache_write(const QCacheDesc& c, int32_t first_layer, int32_t n_layers,
                               int32_t dtype, const QRows& k, const QRows& v, int64_t n_tokens,
                               const int64_t* slots, hipStream_t stream);

// Work items of an attention call: the split that fills the GPU and the bound that
// sizes its grid and its workspace, from what the host knows.
// counters at the start of the workspace; 4 H or 2048 are used
constexpr int64_t kCounters = CM_QCACHE_COUNTER_BYTES / (int64_t)sizeof(int32_t);
struct QAttentionPlan {
  int32_t few_unit, few_items, few_max, many_items, many_max;
  int32_t many_places;  // 0: no request of many rows is cut
  size_t few_at, found_at, many_at, bytes;  // partial results in the workspace, its size
};
QAttentionPlan plan_qcache_attention(int32_t H, int32_t d, int32_t G, int32_t n, int64_t n_rows,
                                     int32_t max_rows, int64_t longest, int32_t dtype);
hipError_t launch_qcache_attention(const QAttention& a, int32_t d, int32_t dtype,
                                   hipStream_t stream);

}  // namespace cm
