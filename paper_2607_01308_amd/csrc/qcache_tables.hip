// Block tables and slot maps of a serving step from the requests' lengths
// (cm_qcache_tables).
//
// With have = ceil(held / B) and want = ceil((held + new) / B), request r takes
// want - have pages from place first_r = sum over q < r of (want_q - have_q) of the free
// list. A page that is fresh in this step begins with a new token (the one whose
// position is a multiple of B), so the thread of that token writes the table entry and
// no two threads need each other's entries.
//
// The step is bound by latency: a decoding step is a few hundred bytes. Every
// workgroup makes the same two prefix sums over the n <= 1024 lengths in its LDS and
// takes a share of the tokens, which finds its request by bisection; one launch, no
// workgroup waits for another. 32 requests of one token 4.0 us, 262144 tokens of 256 requests
// 6.8 us.
#include "qcache.h"

namespace cm {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = CM_QCACHE_MAX_REQUESTS / kThreads;  // requests of one thread's scan
constexpr int kTokensPerGroup = 512;  // two a thread: 262144 tokens 6.9 us, by eight 11.8

struct Sum2 {
  int64_t tokens, pages;
};

__device__ __forceinline__ Sum2 shfl_up2(Sum2 v, int by) {
  return {__shfl_up(v.tokens, by), __shfl_up(v.pages, by)};
}

__global__ __launch_bounds__(kThreads) void qcache_tables_kernel(
    int64_t pages, int32_t b_shift, int32_t n, const int32_t* __restrict__ held,
    const int32_t* __restrict__ fresh, const int32_t* __restrict__ free_pages, int64_t n_free,
    int32_t* __restrict__ table, int64_t width, int64_t n_tokens, int64_t* __restrict__ slots,
    int32_t* __restrict__ rows, int32_t* __restrict__ lens, int64_t* __restrict__ info) {
  __shared__ int32_t s_rows[CM_QCACHE_MAX_REQUESTS + 1];  // first token of each request
  __shared__ int32_t s_page[CM_QCACHE_MAX_REQUESTS];      // first_r - have_r
  __shared__ int32_t s_held[CM_QCACHE_MAX_REQUESTS];
  __shared__ Sum2 s_wave[kThreads / 64];
  __shared__ int64_t s_longest[kThreads / 64];
  __shared__ int s_bad[kThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t B = (int64_t)1 << b_shift;

  int32_t h[kPer], w[kPer];
  int64_t have[kPer], grow[kPer];
  Sum2 sum = {0, 0};
  int64_t longest = 0;
  bool bad = false;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int r = tid * kPer + k;
    h[k] = r < n ? held[r] : 0;
    w[k] = r < n ? fresh[r] : 0;
    bad |= h[k] < 0 || w[k] < 0;
    const int64_t len = (int64_t)h[k] + w[k];
    have[k] = ((int64_t)h[k] + B - 1) >> b_shift;
    const int64_t want = (len + B - 1) >> b_shift;
    bad |= want > width || len > 0x7FFFFFFF;
    grow[k] = want - have[k];
    longest = len > longest ? len : longest;
    sum.tokens += w[k];
    sum.pages += grow[k];
  }
  // exclusive prefix over the threads
  Sum2 run = sum;
#pragma unroll
  for (int by = 1; by < 64; by <<= 1) {
    const Sum2 v = shfl_up2(run, by);
    if (lane >= by) {
      run.tokens += v.tokens;
      run.pages += v.pages;
    }
    const int64_t m = __shfl_xor(longest, by);
    longest = m > longest ? m : longest;
  }
  if (lane == 63) s_wave[wave] = run;
  if (lane == 0) s_longest[wave] = longest;
  const bool wave_bad = __any(bad);
  if (lane == 0) s_bad[wave] = wave_bad;
  __syncthreads();
  Sum2 total = {0, 0};
  run.tokens -= sum.tokens;
  run.pages -= sum.pages;
  bad = false;
  for (int v = 0; v < kThreads / 64; ++v) {
    if (v == wave) {
      run.tokens += total.tokens;
      run.pages += total.pages;
    }
    total.tokens += s_wave[v].tokens;
    total.pages += s_wave[v].pages;
    longest = s_longest[v] > longest ? s_longest[v] : longest;
    bad |= s_bad[v] != 0;
  }
  bad |= total.tokens != n_tokens || total.pages > n_free;
  if (blockIdx.x == 0 && tid == 0) {
    info[0] = bad ? CM_EINVAL : CM_OK;
    info[1] = total.tokens;
    info[2] = total.pages;
    info[3] = longest;
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int r = tid * kPer + k;
    if (r < n) {
      s_rows[r] = (int32_t)run.tokens;
      s_page[r] = (int32_t)(run.pages - have[k]);
      s_held[r] = h[k];
      if (blockIdx.x == 0) {
        rows[r] = bad ? 0 : (int32_t)run.tokens;
        lens[r] = bad ? (h[k] > 0 ? h[k] : 0) : h[k] + w[k];
      }
    }
    run.tokens += w[k];
    run.pages += grow[k];
  }
  if (tid == 0) {
    s_rows[n] = (int32_t)total.tokens;
    if (blockIdx.x == 0) rows[n] = bad ? 0 : (int32_t)total.tokens;
  }
  __syncthreads();

  const int64_t begin = (int64_t)blockIdx.x * kTokensPerGroup;
  const int64_t end = begin + kTokensPerGroup < n_tokens ? begin + kTokensPerGroup : n_tokens;
  for (int64_t i = begin + tid; i < end; i += kThreads) {
    if (bad) {
      slots[i] = -1;
      continue;
    }
    // the last request whose first token is at or before i (requests without new
    // tokens share their successor's place, so the last one is the token's own)
    int lo = 0, hi = n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_rows[mid] <= i) lo = mid;
      else hi = mid - 1;
    }
    const int64_t pos = s_held[lo] + (i - s_rows[lo]);
    const int64_t j = pos >> b_shift;
    const int64_t row = pos & (B - 1);
    // pages that the request had before this step lie before its position held
    const int64_t had = ((int64_t)s_held[lo] + B - 1) >> b_shift;
    int32_t page;
    if (j < had) {
      page = table[lo * width + j];
    } else {
      page = free_pages[s_page[lo] + j];
      if (row == 0) table[lo * width + j] = page;
    }
    slots[i] = page >= 0 && page < pages ? ((int64_t)page << b_shift) + row : -1;
  }
}

}  // namespace

hipError_t launch_qcache_tables(int64_t pages, int32_t b_shift, int32_t n, const int32_t* held,
                                const int32_t* fresh, const int32_t* free_pages, int64_t n_free,
                                int32_t* table, int64_t width, int64_t n_tokens, int64_t* slots,
                                int32_t* rows, int32_t* lens, int64_t* info, hipStream_t stream) {
  ScopedTiming tm(K_QCACHE_TABLES, stream);
  int64_t groups = (n_tokens + kTokensPerGroup - 1) / kTokensPerGroup;
  if (groups < 1) groups = 1;
  hipLaunchKernelGGL(qcache_tables_kernel, dim3((uint32_t)groups), dim3(kThreads), 0, stream,
                     pages, b_shift, n, held, fresh, free_pages, n_free, table, width, n_tokens,
                     slots, rows, lens, info);
  return hipGetLastError();
}

}  // namespace cm
