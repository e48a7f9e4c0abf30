// Drafted trees over the 8-bit paged cache: masks and positions from the nodes' parents
// (cm_qcache_tree), and the launches of the attention (qcache_tree.h), bf16 queries here.
#include "qcache_tree.h"

namespace cm {

namespace {

constexpr int kThreads = 256;

// One workgroup a request: the parents in the LDS, a thread for each (node, word of its mask), which
// follows the node's ancestors up.
__global__ __launch_bounds__(kThreads) void qcache_tree_tables_kernel(
    int64_t n_rows, const int32_t* __restrict__ parents, const int32_t* __restrict__ rows,
    const int32_t* __restrict__ lens, int64_t window, int32_t words, uint64_t* __restrict__ masks,
    int32_t* __restrict__ positions, int32_t* __restrict__ info) {
  __shared__ int16_t up[CM_DRAFT_MAX_NODES];
  const int r = blockIdx.x, tid = threadIdx.x;
  const int64_t first = rows[r], next = rows[r + 1];
  if (first < 0 || next < first || next > n_rows) {
    if (tid == 0) info[r] = CM_EINVAL;
    return;
  }
  const int64_t count = next - first, held = lens[r] - count;
  // a chain without masks may have any number of nodes
  const bool fits = (!parents && !masks) || (count <= CM_DRAFT_MAX_NODES && (!masks || count <= 64 * (int64_t)words));
  bool bad = !fits || held < 0;
  if (!fits) {
    for (int64_t i = tid; i < count; i += kThreads) positions[first + i] = (int32_t)held;
    for (int64_t i = tid; masks && i < count * words; i += kThreads) masks[first * words + i] = 0;
  } else if (!parents) {
    for (int64_t i = tid; i < count; i += kThreads) positions[first + i] = (int32_t)(held + i);
    for (int64_t x = tid; masks && x < count * words; x += kThreads) {
      const int64_t i = x / words, lo = 64 * (x - i * words);
      const int64_t from = window && i - window + 1 > lo ? i - window + 1 - lo : 0, to = i + 1 - lo;
      // bits from .. to - 1 of the word
      const uint64_t below = to >= 64 ? ~0ull : to > 0 ? (1ull << to) - 1 : 0;
      masks[first * words + x] = from >= 64 ? 0 : below & (~0ull << from);
    }
  } else {
    const int c = (int)count;
    for (int i = tid; i < c; i += kThreads) {
      const int p = parents[first + i];
      const bool ok = p >= -1 && p < i;
      bad |= !ok;
      up[i] = (int16_t)(ok ? p : -1);
    }
    __syncthreads();
    for (int x = tid; masks && x < c * words; x += kThreads) {
      const int i = x / words, lo = 64 * (x - i * words);
      uint64_t bits = 0;
      int64_t steps = 0;
      for (int j = i; j >= lo && (!window || steps < window); j = up[j], ++steps)
        if (j < lo + 64) bits |= 1ull << (j - lo);
      masks[first * words + x] = bits;
    }
    for (int i = tid; i < c; i += kThreads) {
      int depth = 0;
      for (int j = up[i]; j >= 0; j = up[j]) ++depth;
      positions[first + i] = (int32_t)(held + depth);
    }
  }
  const int any = __syncthreads_or(bad);
  if (tid == 0) info[r] = any ? CM_EINVAL : CM_OK;
}

}  // namespace

hipError_t launch_qcache_tree(int32_t n, int64_t n_rows, const int32_t* parents, const int32_t* rows,
                              const int32_t* lens, int64_t window, int32_t words, uint64_t* masks,
                              int32_t* positions, int32_t* info, hipStream_t stream) {
  ScopedTiming tm(K_QCACHE_TREE, stream);
  hipLaunchKernelGGL(qcache_tree_tables_kernel, dim3((uint32_t)n), dim3(kThreads), 0, stream, n_rows, parents,
                     rows, lens, window, words, masks, positions, info);
  return hipGetLastError();
}

TreePlan plan_qcache_tree(int32_t H, int32_t d, int32_t G, int32_t n, int64_t n_rows, int32_t max_rows,
                          int64_t longest, int32_t dtype) {
  TreePlan p;
  const int32_t terms = dtype == CM_BF16 ? 1 : 3, most = tree_tiles_most(terms, d);
  const int64_t rows = (int64_t)(max_rows < n_rows ? max_rows : n_rows) * G;
  p.tiles = rows <= 16 ? 1 : rows <= 32 || most == 2 ? 2 : 4;
  p.tiles = p.tiles < most ? p.tiles : most;
  // workgroups that run together
  const int64_t groups = (int64_t)kTreeGroups * device_cu_count();
  p.items = (int32_t)(groups / H > 0 ? groups / H : 1);
  p.places = 2 * p.items;                        // a span's first and last range
  // all contexts together, a request's once for each of its tiles, are less than 2e9 units
  const double tiles = (double)n_rows * G / (16 * p.tiles) + n;
  p.unit = kTreeWaves * kStep;
  while (tiles * (double)(longest / p.unit + 1) > 1.9e9) p.unit *= 2;
  p.least = 2;
  p.cuts_at = sizeof(int32_t) * kCounters;       // (counters are the causal attention's)
  p.part_at = p.cuts_at + align_up(sizeof(TreeCut) * (size_t)p.places, kWsAlign);
  p.bytes = p.part_at + sizeof(float) * (size_t)(16 * p.tiles) * (size_t)(d + 2) * (size_t)H * (size_t)p.places;
  return p;
}

hipError_t launch_tree_bf16(const TreeAttention& a, int32_t d, int32_t tiles, hipStream_t stream) {
  return launch_tree<1>(a, d, tiles, stream);
}

hipError_t launch_qcache_tree_attention(const TreeAttention& a, int32_t d, int32_t dtype, int32_t tiles,
                                        hipStream_t stream) {
  ScopedTiming tm(K_QCACHE_TREE_ATTENTION, stream);
  return dtype == CM_BF16 ? launch_tree_bf16(a, d, tiles, stream)
                          : launch_tree_fp32(a, d, tiles, stream);
}

}  // namespace cm
