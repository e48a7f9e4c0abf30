// Internal interface of the operators for drafted decoding (norm_rotate.hip, qcache_tree.hip, verify.hip, qcache_keep.hip).
#pragma once

#include "qcache.h"

namespace cm {

// Heads of queries or of keys (cm_head_rows), strides in bytes; heads 0: none.
struct HeadRows {
  const uint8_t* in;
  uint8_t* out;
  int64_t in_token, in_head, out_token, out_head;
  const void* weight;    // nullptr: not normalised
  int32_t weight_dtype;  // cm_dtype
  int32_t heads;
};

struct RotateArgs {
  HeadRows q, k;
  const int32_t* positions;
  int64_t n_tokens;
  double log2_base;
  double between[8];     // of the launch: a lane's pairs, relative to its first one
  float eps;
};

hipError_t launch_norm_rotate(RotateArgs a, int32_t d, int32_t dtype, int32_t style,
                              hipStream_t stream);

// Pages src[i] to dst[i], i < n, of layers [first_layer, first_layer + n_layers).
hipError_t launch_qcache_copy(const QCacheDesc& c, int32_t first_layer, int32_t n_layers, int64_t n,
                              const int32_t* src, const int32_t* dst, hipStream_t stream);

// cm_qcache_keep.
struct KeepArgs {
  QCacheDesc c;
  int32_t n;
  int64_t n_rows;
  const int32_t* table;
  int64_t width;
  const int32_t* lens;
  const int32_t* rows;
  const int32_t* path;
  const int32_t* counts;
  int32_t* lens_out;
  int32_t* freed;
  int64_t n_freed;
  int64_t* info;
};
hipError_t launch_qcache_keep(const KeepArgs& a, hipStream_t stream);

// Masks and positions of the nodes (cm_qcache_tree).
hipError_t launch_qcache_tree(int32_t n, int64_t n_rows, const int32_t* parents, const int32_t* rows,
                              const int32_t* lens, int64_t window, int32_t words, uint64_t* masks,
                              int32_t* positions, int32_t* info, hipStream_t stream);

// Tree attention: what it reads and writes beside the fields of QAttention that are not of requests of
// many rows; few_items, few_max, few_unit, few_part and many_found are those of its plan.
struct TreeAttention {
  QAttention a;
  const uint64_t* masks;
  int64_t words;
  const int32_t* positions;
  int32_t least;           // units of a span at least
};
// How its work is cut, from what the host knows.
struct TreePlan {
  int32_t tiles;           // row tiles of 16 that a wave takes
  int32_t unit, items, places, least;
  size_t cuts_at, part_at, bytes;  // which tiles are cut and partial results in the workspace, its size
};
TreePlan plan_qcache_tree(int32_t H, int32_t d, int32_t G, int32_t n, int64_t n_rows, int32_t max_rows,
                          int64_t longest, int32_t dtype);
hipError_t launch_qcache_tree_attention(const TreeAttention& a, int32_t d, int32_t dtype, int32_t tiles,
                                        hipStream_t stream);

// cm_verify_drafts; strides of probabilities in elements.
struct VerifyArgs {
  int32_t n;
  int64_t n_rows, V;
  const void* p;
  const void* q;           // nullptr: the drafts were not sampled
  int64_t p_row, q_row;
  const int64_t* drafts;
  const int32_t* parents;
  const int32_t* rows;
  const float* accept;
  const float* sample;
  int32_t* path;
  int32_t* counts;
  int64_t* tokens;
  void* talk;              // verify_workspace() bytes, or nullptr: one workgroup a request
  int32_t groups;          // of the launch: workgroups of a request
  uint64_t helper_wait, sums_wait;  // and verify_waits
};
// How long the workgroups of a request wait for one another, in ticks of 10 ns for each 8192 elements (or
// part of them) of a part of the row: a helper for a pass, the first one for the helpers' sums. Neither is
// needed: a helper that has waited this long ends, and the first one makes the sums itself. With 0 nobody
// looks; tests set them, between launches.
extern uint64_t verify_waits[2];
size_t verify_workspace(int32_t n, int64_t V);
hipError_t launch_verify_drafts(VerifyArgs a, int32_t dtype, hipStream_t stream);

}  // namespace cm
