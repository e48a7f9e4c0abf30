// Launches of the attention over the 8-bit paged cache (cm_qcache_attention): one kernel, for
// decoding steps the one that takes few query rows of a request alone, else the one that
// takes both kinds of requests (qcache_prompt.hip).
#include <type_traits>

#include "qcache_few.h"

namespace cm {

namespace {

constexpr int kFewWaves = 4;

template <int TERMS, int D>
__global__ __launch_bounds__(64 * kFewWaves, 2) void qcache_few_rows_kernel(QAttention a) {
  __shared__ FewShared<TERMS, D, kFewWaves> lds;
  few_rows_span<TERMS, D, kFewWaves>(a, blockIdx.x, lds);
}

}  // namespace

QAttentionPlan plan_qcache_attention(int32_t H, int32_t d, int32_t G, int32_t n, int64_t n_rows,
                                     int32_t max_rows, int64_t longest, int32_t dtype) {
  QAttentionPlan p;
  // workgroups that run together for few rows: two on a compute unit
  const int64_t groups = 2 * device_cu_count();
  const int32_t terms = dtype == CM_BF16 ? 1 : 3;
  const int64_t rows = n_rows * G;
  const bool many = !few_rows((int64_t)max_rows * G);
  const auto per_head = [&](int64_t all) { return (int32_t)(all / H > 0 ? all / H : 1); };
  // all contexts together are less than 2^31 units
  p.few_unit = kUnit;
  while (n * (longest / p.few_unit + 1) > 0x7FFFFFFF) p.few_unit *= 2;
  p.few_items = per_head(groups);
  p.many_items = per_head(device_cu_count() * many_groups(d, terms));
  p.few_max = 2 * p.few_items;                       // a span's first and last segment
  // 4/3 of the items that run together, and every tile's ranges round up once
  p.many_max = many ? (int32_t)((rows + kManyRows - 1) / kManyRows + n + p.many_items * 4 / 3 + 1) : 0;
  // Partial results of the items of cut tiles alone. Such a tile sees more units than a range has, so
  // its ranges are less than twice the quotient, and the quotients' sum is at most 4/3
  // many_items (find_item). Where there are more heads than items that run together, no tile is
  // cut.
  const int32_t most = p.many_items > 1 ? p.many_items * 8 / 3 + 1 : 0;
  p.many_places = p.many_max < most ? p.many_max : most;
  const size_t row = sizeof(float) * (size_t)(d + 4) * (size_t)H;
  p.few_at = sizeof(int32_t) * kCounters;
  p.found_at = p.few_at + align_up(row * kFewRows * (size_t)p.few_max, kWsAlign);
  p.many_at = p.found_at + align_up(sizeof(Item) * (size_t)p.many_places, kWsAlign);
  p.bytes = p.many_at + row * kManyRows * (size_t)p.many_places;
  return p;
}

hipError_t launch_qcache_attention(const QAttention& a, int32_t d, int32_t dtype,
                                   hipStream_t stream) {
  const auto go = [&](auto terms, auto dd) -> hipError_t {
    constexpr int TERMS = decltype(terms)::value, D = decltype(dd)::value;
    const uint32_t few = (uint32_t)head_groups(a.H, a.few_items);
    ScopedTiming tm(K_QCACHE_ATTENTION, stream);
    if (a.many_max)
      return launch_qcache_any_rows<TERMS, D>(a, (uint32_t)head_groups(a.H, a.many_max), few, stream);
    hipLaunchKernelGGL((qcache_few_rows_kernel<TERMS, D>), dim3(few), dim3(64 * kFewWaves), 0, stream,
                       a);
    return hipGetLastError();
  };
  const auto by_d = [&](auto terms) {
    switch (d) {
      case 64: return go(terms, std::integral_constant<int, 64>{});
      case 128: return go(terms, std::integral_constant<int, 128>{});
      default: return go(terms, std::integral_constant<int, 256>{});
    }
  };
  return dtype == CM_BF16 ? by_d(std::integral_constant<int, 1>{})
                          : by_d(std::integral_constant<int, 3>{});
}

}  // namespace cm
