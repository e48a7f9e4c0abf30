// Accepted tokens of drafted nodes, moved to the front of their places in the 8-bit paged cache
// (cm_qcache_keep), and whole pages copied (cm_qcache_copy).
//
// A request's path is ascending, so place held + i takes what lies at held + path[i], i <= path[i]:
// rows moved in that order never overwrite one that has still to be moved. The unit of work is
// what a request keeps of one head of one layer's K or V; a wave takes it page by page, rows of 16
// bytes a lane, many rows at a time, all loaded before any is stored. A page that takes rows gets the
// greatest scale of the pages they come from and, where rows lie before them, its own; codes are
// multiplied by old / new scale, at most 1, and rounded again. With scales that are powers of two a
// code changes only where its value falls below 2^-6 of the new scale.
#include <algorithm>

#include "draft.h"
#include "qcache_ops.h"

namespace cm {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
// Slices of a head that a wave of cm_qcache_keep takes together: the chain of loads (rows, path, table, scales,
// codes) is the same for all.
constexpr int kUnits = 2;

// A request's rows of the step as keep sees them.
struct Kept {
  int64_t row0;        // its first row
  int64_t held;        // tokens of its context; below 0: not all nodes have a place
  int32_t count, kept; // nodes, nodes accepted
  bool good;           // rows, length and count are as they have to be
};
__device__ __forceinline__ Kept kept_of(const KeepArgs& a, int r) {
  const int64_t first = a.rows[r], next = a.rows[r + 1];
  Kept k;
  k.good = first >= 0 && next >= first && next <= a.n_rows;
  k.row0 = first;
  k.count = k.good ? (int32_t)(next - first) : 0;
  const int32_t want = a.counts[r];
  k.kept = want < 0 ? 0 : want > k.count ? k.count : want;
  k.held = (int64_t)a.lens[r] - k.count;
  k.good = k.good && k.kept == want && k.held >= 0 && a.lens[r] <= (a.width << a.c.b_shift);
  return k;
}

__device__ __forceinline__ float wave_max(float m) {
#pragma unroll
  for (int by = 1; by < 64; by <<= 1) m = fmaxf(m, __shfl_xor(m, by));
  return m;
}

// Codes times a ratio of at most 1.
__device__ __forceinline__ u32x4 rescaled(u32x4 c, float ratio) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[w], false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[w], true);
    c[w] = codes_of(lo[0] * ratio, lo[1] * ratio, hi[0] * ratio, hi[1] * ratio);
  }
  return c;
}
// (scales of 0 give 0: there is nothing that could be kept)
__device__ __forceinline__ float ratio_of(float old, float now) {
  return old == now ? 1.f : old / now;
}

// The lengths, the free pages and the status: one workgroup.
__device__ __forceinline__ void keep_lengths(const KeepArgs& a) {
  __shared__ int64_t s_sum[kWaves];
  __shared__ int s_bad;
  constexpr int kPer = CM_QCACHE_MAX_REQUESTS / kThreads;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) s_bad = 0;
  __syncthreads();
  int64_t from[kPer], some[kPer], sum = 0;
  bool bad = false;
  const int per = (a.n + kThreads - 1) / kThreads;  // requests of a thread
#pragma unroll
  for (int x = 0; x < kPer; ++x) {
    const int r = tid * per + x;
    from[x] = some[x] = 0;
    if (x >= per || r >= a.n) continue;
    const Kept k = kept_of(a, r);
    bad |= !k.good;
    // (eight loads at a time: one after another the longest path bounds a small step)
    const int kept = k.good ? k.kept : 0;
    int last = -1;
    for (int i = 0; i < kept; i += 8) {
      int p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = a.path[k.row0 + (i + e < kept ? i + e : kept - 1)];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (i + e < kept) {
          bad |= p[e] <= last || p[e] >= k.count;
          last = p[e];
        }
    }
    const int64_t t = a.lens[r] > 0 ? a.lens[r] : 0;
    const int64_t left = k.held + k.kept > 0 ? k.held + k.kept : 0;
    a.lens_out[r] = (int32_t)left;
    const int64_t B = (int64_t)1 << a.c.b_shift;
    from[x] = (left + B - 1) >> a.c.b_shift;
    int64_t end = (t + B - 1) >> a.c.b_shift;
    end = end < a.width ? end : a.width;
    some[x] = end > from[x] ? end - from[x] : 0;
    sum += some[x];
  }
  int64_t upto = sum;
#pragma unroll
  for (int by = 1; by < 64; by <<= 1) {
    const int64_t v = __shfl_up(upto, by);
    if (lane >= by) upto += v;
  }
  if (lane == 63) s_sum[wave] = upto;
  if (bad) s_bad = 1;
  __syncthreads();
  int64_t at = upto - sum, total = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) at += s_sum[w];
    total += s_sum[w];
  }
#pragma unroll
  for (int x = 0; x < kPer; ++x) {
    const int32_t* row = a.table + (int64_t)(tid * per + x) * a.width;
    for (int64_t j = 0; j < some[x]; ++j)
      if (at + j < a.n_freed) a.freed[at + j] = row[from[x] + j];
    at += some[x];
  }
  if (tid == 0) {
    a.info[0] = s_bad || total > a.n_freed ? CM_EINVAL : CM_OK;
    a.info[1] = total;
  }
}

// Workgroup (0, 0) does the lengths; of the others each takes some heads of a request's slices.
template <int D>
__global__ __launch_bounds__(kThreads) void qcache_keep_kernel(KeepArgs a, int32_t units) {
  constexpr int kLanes = D / 16;                 // lanes of a row
  constexpr int kRows = 64 / kLanes;             // rows of a wave's load
  if (blockIdx.x == 0) {
    if (blockIdx.y == 0) keep_lengths(a);
    return;
  }
  const int lane = threadIdx.x & 63;
  const int unit0 = (((int)blockIdx.x - 1) * kWaves + (threadIdx.x >> 6)) * kUnits;  // (layer, K/V, head)
  if (unit0 >= units) return;
  float* scales[kUnits];
  uint8_t* codes[kUnits];
  bool live[kUnits];
#pragma unroll
  for (int y = 0; y < kUnits; ++y) {
    live[y] = unit0 + y < units;
    const int unit = live[y] ? unit0 + y : unit0, slice = unit / a.c.H, h = unit - slice * a.c.H;
    scales[y] = a.c.scales + slice * a.c.slice_scales() + h;
    codes[y] = a.c.codes + slice * a.c.slice_codes() + (((int64_t)h << a.c.b_shift) * D);
  }
  const int64_t page_codes = ((int64_t)a.c.H << a.c.b_shift) * D;
  const int B = 1 << a.c.b_shift;
  for (int r = blockIdx.y; r < a.n; r += gridDim.y) {
    const Kept k = kept_of(a, r);
    if (!k.good || k.kept == 0) continue;
    const int32_t* path = a.path + k.row0;
    const int32_t* table = a.table + (int64_t)r * a.width;
    // a path that is not ascending within the nodes moves nothing
    bool bad = false;
    for (int i = lane; i < k.kept; i += 64) {
      const int p = path[i];
      bad |= p >= k.count || p <= (i ? path[i - 1] : -1);
    }
    if (__any(bad)) continue;
    const int64_t end = k.held + k.kept;
    for (int64_t t = k.held; t < end;) {
      // rows t .. stop - 1 of one page, the i0-th kept one first
      const int64_t stop = (t | (B - 1)) + 1 < end ? (t | (B - 1)) + 1 : end;
      const int i0 = (int)(t - k.held), some = (int)(stop - t), begin = (int)(t & (B - 1));
      const int32_t page = table[t >> a.c.b_shift];
      const bool there = page >= 0 && page < a.c.pages;
      float own[kUnits], was[kUnits][2], top[kUnits];
#pragma unroll
      for (int y = 0; y < kUnits; ++y) {
        own[y] = there ? scales[y][(int64_t)page * a.c.H] : 0.f;
        top[y] = begin > 0 ? own[y] : 0.f;
      }
      // where the rows come from: rows lane and lane + 64 of them
      int32_t from[2], at[2];
      bool same = true;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int i = lane + 64 * x;
        from[x] = -1;
        at[x] = 0;
#pragma unroll
        for (int y = 0; y < kUnits; ++y) was[y][x] = 0.f;
        if (i < some) {
          const int64_t s = k.held + path[i0 + i];
          const int32_t p = table[s >> a.c.b_shift];
          at[x] = (int)(s & (B - 1));
          same = same && s == t + i;
          const bool is = p >= 0 && p < a.c.pages;
          if (is) from[x] = p;
          // (a row that cannot come leaves the page's own scale among them)
#pragma unroll
          for (int y = 0; y < kUnits; ++y)
            was[y][x] = !is || p == page ? own[y] : scales[y][(int64_t)p * a.c.H];
        }
#pragma unroll
        for (int y = 0; y < kUnits; ++y) top[y] = fmaxf(top[y], was[y][x]);
      }
      same = __all(same);
      bool moves[kUnits], any = false;
#pragma unroll
      for (int y = 0; y < kUnits; ++y) {
        top[y] = wave_max(top[y]);
        moves[y] = live[y] && there && !(same && top[y] == own[y]);
        any |= moves[y];
      }
      if (any) {
        const int64_t to = page * page_codes;
#pragma unroll
        for (int y = 0; y < kUnits; ++y)
          if (moves[y] && begin > 0 && top[y] != own[y]) {
            const float ratio = ratio_of(own[y], top[y]);
            for (int u = lane; u < begin * kLanes; u += 64) {
              u32x4* p = reinterpret_cast<u32x4*>(codes[y] + to) + u;
              *p = rescaled(*p, ratio);
            }
          }
        for (int i = 0; i < some; i += kRows) {
          const int mine = i + lane / kLanes, look = mine & 63;
          const int32_t f0 = __shfl(from[0], look), f1 = __shfl(from[1], look);
          const int32_t a0 = __shfl(at[0], look), a1 = __shfl(at[1], look);
          const int32_t f = mine < 64 ? f0 : f1;
          const int32_t row = mine < 64 ? a0 : a1;
          float w[kUnits];
#pragma unroll
          for (int y = 0; y < kUnits; ++y) {
            const float w0 = __shfl(was[y][0], look), w1 = __shfl(was[y][1], look);
            w[y] = mine < 64 ? w0 : w1;
          }
          if (mine < some && f >= 0) {
            u32x4 c[kUnits];
#pragma unroll
            for (int y = 0; y < kUnits; ++y)
              c[y] = *global_ptr<u32x4>(codes[y] + f * page_codes + row * D + lane % kLanes * 16);
#pragma unroll
            for (int y = 0; y < kUnits; ++y)
              if (moves[y])
                *reinterpret_cast<u32x4*>(codes[y] + to + (begin + mine) * D + lane % kLanes * 16) =
                    w[y] == top[y] ? c[y] : rescaled(c[y], ratio_of(w[y], top[y]));
          }
        }
#pragma unroll
        for (int y = 0; y < kUnits; ++y)
          if (moves[y] && lane == 0) scales[y][(int64_t)page * a.c.H] = top[y];
      }
      t = stop;
    }
  }
}

// A page of one layer's K or V is one run of bytes: kPiece of them a workgroup.
constexpr int kPiece = kThreads * 64;
__global__ __launch_bounds__(kThreads) void qcache_copy_kernel(QCacheDesc c, const int32_t* src,
                                                               const int32_t* dst, int32_t bytes,
                                                               int32_t pieces, int64_t from) {
  const int64_t x = from + blockIdx.x;
  const int64_t i = x / pieces;
  const int piece = (int)(x - i * pieces);
  const int64_t s = src[i], t = dst[i];
  if (s < 0 || s >= c.pages || t < 0 || t >= c.pages) return;
  const int64_t slice = blockIdx.y;
  const uint8_t* in = c.codes + slice * c.slice_codes() + s * bytes;
  uint8_t* out = c.codes + slice * c.slice_codes() + t * bytes;
  u32x4 v[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int at = piece * kPiece + (k * kThreads + (int)threadIdx.x) * 16;
    if (at < bytes) v[k] = *global_ptr<u32x4>(in + at);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int at = piece * kPiece + (k * kThreads + (int)threadIdx.x) * 16;
    if (at < bytes) *reinterpret_cast<u32x4*>(out + at) = v[k];
  }
  if (piece == 0) {
    float* sc = c.scales + slice * c.slice_scales();
    for (int h = threadIdx.x; h < c.H; h += kThreads) sc[t * c.H + h] = sc[s * c.H + h];
  }
}

}  // namespace

hipError_t launch_qcache_keep(const KeepArgs& a, hipStream_t stream) {
  const int32_t units = 2 * a.c.L * a.c.H;       // (at most 65535)
  const dim3 grid((uint32_t)(1 + (units + kWaves * kUnits - 1) / (kWaves * kUnits)), (uint32_t)a.n);
  ScopedTiming tm(K_QCACHE_KEEP, stream);
  switch (a.c.d) {
    case 64: hipLaunchKernelGGL(qcache_keep_kernel<64>, grid, dim3(kThreads), 0, stream, a, units); break;
    case 128: hipLaunchKernelGGL(qcache_keep_kernel<128>, grid, dim3(kThreads), 0, stream, a, units); break;
    default: hipLaunchKernelGGL(qcache_keep_kernel<256>, grid, dim3(kThreads), 0, stream, a, units); break;
  }
  return hipGetLastError();
}

hipError_t launch_qcache_copy(const QCacheDesc& c, int32_t first_layer, int32_t n_layers, int64_t n,
                              const int32_t* src, const int32_t* dst, hipStream_t stream) {
  if (n == 0 || n_layers == 0) return hipSuccess;
  QCacheDesc from = c;
  from.codes += 2 * (int64_t)first_layer * c.slice_codes();
  from.scales += 2 * (int64_t)first_layer * c.slice_scales();
  const int64_t bytes = ((int64_t)c.H << c.b_shift) * c.d;  // (a page: at most 2^31 - 1, checked)
  const int32_t pieces = (int32_t)((bytes + kPiece - 1) / kPiece);
  const int64_t blocks = n * pieces;
  ScopedTiming tm(K_QCACHE_COPY, stream);
  // a launch holds at most 2^24 - 1 workgroups of 256 threads a row of the grid
  for (int64_t done = 0; done < blocks; done += (1 << 24) - 1) {
    const int64_t some = std::min<int64_t>(blocks - done, (1 << 24) - 1);
    hipLaunchKernelGGL(qcache_copy_kernel, dim3((uint32_t)some, (uint32_t)(2 * n_layers)), dim3(kThreads), 0,
                       stream, from, src, dst, (int32_t)bytes, pieces, done);
  }
  return hipGetLastError();
}

}  // namespace cm
