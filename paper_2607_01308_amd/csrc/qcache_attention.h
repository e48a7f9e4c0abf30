// Device code that the attention kernels of the 8-bit paged cache share: which part of
// the step a workgroup takes, and how results and partial results are written.
#pragma once

#include "qcache_ops.h"

namespace cm {

constexpr float kNone = -__builtin_inff();
constexpr int kFewRows = 16;    // query rows of a tile of the kernel for few rows
constexpr int kManyRows = 128;  // and of the kernel for many

// A request's query rows (its rows times the group) are taken by one kernel or the
// other, whole.
__host__ __device__ __forceinline__ bool few_rows(int64_t rows) { return rows <= kFewRows; }

// Waves that share their rows in the kernel for many (qcache_prompt.hip). A wave's registers hold
// its queries' terms, d * terms / 4 of them, and its columns of the output, d / 2. For d = 256 two
// waves share (one wave for all columns and half as many waves: 4096 queries over 16384 tokens, 8
// heads, G 4, 4.31 ms, so 4.11; short questions 72 us, so 67).
constexpr int many_halves(int d) { return d > 128 ? 2 : 1; }

// Workgroups of that kernel on a compute unit. Three terms of d = 128 take the registers of two
// waves (two waves that share rows instead: 1024 queries over 16384 tokens, 8 heads, G 4, 893 us,
// so 737).
constexpr int many_groups(int d, int terms) { return d * (terms + 1) > 256 ? 1 : 2; }

struct Item {
  int32_t r, tile, split, splits;  // request, row tile, range of its context, how many
  int32_t row0, count, len;        // the request's first row, rows, tokens up to the last row
  int32_t begin, chunk;            // where its visible context begins, tokens of a range
  int32_t any;                     // 0: the grid has more workgroups than there are items
  int32_t place, places;           // of its partial results where splits > 1; how many there are in all
};

// A request's rows that are computed and the tokens up to the last one of them, within the bounds
// that the host checked. The request's rows end at the last of its tokens: where rows past
// max_rows or past the queries' end are left out, as many tokens are (and none may be left).
__device__ __forceinline__ void request(const QAttention& a, int r, int& row0, int& count,
                                        int& len) {
  const int64_t first = a.rows ? a.rows[r] : r, next = a.rows ? a.rows[r + 1] : r + 1;
  const int64_t f = first < 0 ? 0 : first, e = next > a.n_rows ? a.n_rows : next;
  int64_t c = e > f ? e - f : 0;
  c = c < a.max_rows ? c : a.max_rows;
  const int64_t cap = a.width << a.b_shift;
  int64_t t = a.lens[r];
  t = t < 0 ? 0 : t > cap ? cap : t;
  row0 = (int)f;
  count = (int)c;
  len = c > 0 ? (int)(t - (next - f - c)) : 0;
}

constexpr int kUnit = 128;  // tokens by which contexts are cut

__device__ __forceinline__ int visible_begin(const QAttention& a, int count, int len) {
  if (a.window == 0) return 0;
  const int64_t lo = (int64_t)len - count - a.window + 1;
  return lo > 0 ? (int)(lo & ~(int64_t)63) : 0;
}

// x of another lane by a DPP move, 0 where there is none.
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROW_MASK, 0xF, false);
}
// Inclusive prefix sums over the lanes of a wave: within rows of 16, then the rows' last
// lanes to the rows after them.
template <class T>
__device__ __forceinline__ T wave_scan(T x) {
  const auto from = [](uint32_t v) { return __builtin_bit_cast(T, v); };
  const auto bits = [](T v) { return __builtin_bit_cast(uint32_t, v); };
  x += from(dpp<0x111, 0xF>(bits(x)));   // row_shr:1
  x += from(dpp<0x112, 0xF>(bits(x)));
  x += from(dpp<0x114, 0xF>(bits(x)));
  x += from(dpp<0x118, 0xF>(bits(x)));
  x += from(dpp<0x142, 0xA>(bits(x)));   // row_bcast:15 to rows 1 and 3
  x += from(dpp<0x143, 0xC>(bits(x)));   // row_bcast:31 to rows 2 and 3
  return x;
}

// Row tiles of a request for the kernel of ROWS rows; 0 where the other takes it.
template <int ROWS>
__device__ __forceinline__ int row_tiles(const QAttention& a, int count) {
  const int rows = count * a.G;                  // (n_rows * q_heads is below 2^31)
  if (few_rows(rows) != (ROWS == kFewRows)) return 0;
  return (int)((uint32_t)(rows + ROWS - 1) / ROWS);
}

// What the workgroup shares while it looks for its item.
struct FindShared {
  float cost[8], tiles[8];
  int items[8], places[8];
  Item it;
};

// What the rows of a tile see: positions see_lo .. see_hi - 1 of one row, those that
// every row of the tile sees, and those that any does.
struct Sight {
  int tok_lo, tok_hi;      // first and last row of the request in the tile
  int all_lo, all_hi, any_lo, any_hi;
};
template <int ROWS>
__device__ __forceinline__ Sight tile_sight(const QAttention& a, const Item& it) {
  Sight s;
  s.tok_lo = it.tile * ROWS / a.G;
  const int last = (it.tile * ROWS + ROWS - 1) / a.G;
  s.tok_hi = last < it.count ? last : it.count - 1;
  // (a row before the first token counts as at -1: the differences with a window stay in range)
  const int p0 = it.len - it.count;
  const int p_lo = p0 + s.tok_lo > -1 ? p0 + s.tok_lo : -1;
  const int p_hi = p0 + s.tok_hi > -1 ? p0 + s.tok_hi : -1;
  s.all_hi = p_lo + 1;   // <= 0 where the first row sees nothing
  s.all_lo = a.window && p_hi - a.window + 1 > 0 ? p_hi - a.window + 1 : 0;
  s.any_lo = a.window && p_lo - a.window + 1 > 0 ? p_lo - a.window + 1 : 0;
  s.any_hi = p_hi + 1 > 0 ? p_hi + 1 : 0;
  return s;
}

// Tokens that a tile of a request sees, on the average over its tiles: a tile's last row sees the
// rows before it, and one position more than the row before.
template <int ROWS>
__device__ __forceinline__ int tile_units(const QAttention& a, int count, int len) {
  const int own = (ROWS + a.G - 1) / a.G < count ? (ROWS + a.G - 1) / a.G : count;
  int64_t seen = (int64_t)len - (count - own) / 2;
  if (a.window && seen > (int64_t)a.window + own) seen = (int64_t)a.window + own;
  return seen > 0 ? (int)((seen + kUnit - 1) / kUnit) : 0;
}

// The workgroup's item from the lengths: what a request's tiles see is cut into as many equal
// ranges of whole units that about `items` ranges come out for all row tiles, as many as run
// together. Where there are more tiles than that, they are cut if they are longer than 3/4 of
// what a workgroup has to do in all, beyond which the longest would be what the call waits for (six
// prompts of 493 to 3975 rows over up to 300 tokens, 2 heads of d = 256, G 2: 307 us uncut, 242 so); shorter
// ones gain nothing by a cut and would cost their partial results. Every workgroup looks
// at all n <= 1024 lengths, a few a thread: two prefix sums, about 2 us, beside which other
// workgroups stream (a plan made once would be a launch of its own, 5 us and more). The grid holds
// `most` items, enough for requests that share no rows, and the workspace a.many_places of the items
// that cut tiles have, one after another; where rows_dev lays requests over one another so that
// more come out, no workgroup has an item.
template <int ROWS, int THREADS>
__device__ __forceinline__ Item find_item(const QAttention& a, int items, int most, int item,
                                          FindShared& lds) {
  constexpr int kPer = CM_QCACHE_MAX_REQUESTS / THREADS;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per = (a.n + THREADS - 1) / THREADS;   // requests of a thread
  int row0[kPer], count[kPer], len[kPer], tiles[kPer], units[kPer];
  float cost = 0.f, all = 0.f;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int r = (int)threadIdx.x * per + k;
    tiles[k] = units[k] = row0[k] = count[k] = len[k] = 0;
    if (k < per && r < a.n) {
      request(a, r, row0[k], count[k], len[k]);
      tiles[k] = row_tiles<ROWS>(a, count[k]);
      units[k] = tile_units<ROWS>(a, count[k], len[k]);
      cost += (float)tiles[k] * (float)units[k];
      all += (float)tiles[k];
    }
  }
  cost = wave_scan(cost);
  all = wave_scan(all);
  if (threadIdx.x == 0) lds.it.any = lds.it.places = 0;
  if (lane == 63) {
    lds.cost[wave] = cost;
    lds.tiles[wave] = all;
  }
  __syncthreads();
  cost = all = 0.f;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    cost += lds.cost[w];
    all += lds.tiles[w];
  }
  // Each tile's ranges round up by about half a range, so that many fewer make `items` of them
  // in all. (And a little more than the quotient: rounded sums must not make more items than
  // the grid has.)
  const float aim = all <= (float)items ? (float)items - 0.6f * all : 1.333f * (float)items;
  const float want = cost / aim * 1.0001f;
  const int chunk = !a.many_places || want > 1e9f ? 1 << 30 : want > 1.f ? (int)want + 1 : 1;
  int splits[kPer], mine = 0, kept = 0;          // items; those that have a place
  if (all > (float)most) return Item{};          // (their number might not fit an int)
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    splits[k] = (int)((uint32_t)(units[k] + chunk - 1) / (uint32_t)chunk);
    splits[k] = splits[k] < 1 ? 1 : splits[k];
    mine += tiles[k] * splits[k];
    kept += splits[k] > 1 ? tiles[k] * splits[k] : 0;
  }
  const int upto = wave_scan(mine), kept_upto = wave_scan(kept);
  if (lane == 63) {
    lds.items[wave] = upto;
    lds.places[wave] = kept_upto;
  }
  __syncthreads();
  int at = upto - mine, total = 0, place = kept_upto - kept, places = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < wave) {
      at += lds.items[w];
      place += lds.places[w];
    }
    total += lds.items[w];
    places += lds.places[w];
  }
  const bool fits = total <= most && places <= a.many_places;
  if (fits && threadIdx.x == 0) lds.it.places = places;
  if (fits && item >= at && item < at + mine) {
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int here = tiles[k] * splits[k];
      if (item >= at && item < at + here) {
        Item it;
        it.r = (int)threadIdx.x * per + k;
        it.splits = splits[k];
        // the tiles of a prompt see more tokens the later they are: the long ones first
        it.tile = tiles[k] - 1 - (item - at) / splits[k];
        it.split = (item - at) % splits[k];
        it.row0 = row0[k];
        it.count = count[k];
        it.len = len[k];
        const Sight sight = tile_sight<ROWS>(a, it);
        it.begin = sight.any_lo & ~63;
        const int own = sight.any_hi > it.begin ? (sight.any_hi - it.begin + kUnit - 1) / kUnit : 0;
        it.chunk = (int)((uint32_t)(own + splits[k] - 1) / (uint32_t)splits[k]) * kUnit;
        it.any = 1;
        it.place = place + (item - at);
        it.places = places;
        lds.it = it;
      }
      at += here;
      place += splits[k] > 1 ? here : 0;
    }
  }
  __syncthreads();
  Item it = lds.it;
  const auto same = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  it.r = same(it.r);
  it.tile = same(it.tile);
  it.split = same(it.split);
  it.splits = same(it.splits);
  it.row0 = same(it.row0);
  it.count = same(it.count);
  it.len = same(it.len);
  it.begin = same(it.begin);
  it.chunk = same(it.chunk);
  it.any = same(it.any);
  it.place = same(it.place);
  it.places = same(it.places);
  return it;
}

// KV head and item of a workgroup. Workgroups go to the eight XCDs in turn, each with a
// cache of its own; the H heads of an item read the same table entries and neighbouring
// scales, so they are workgroups of one XCD, one after another.
struct HeadItem {
  int h, item;
};
__device__ __forceinline__ HeadItem head_item(int H, int block) {
  const int x = block & 7, y = block >> 3;
  return {y % H, (y / H) * 8 + x};
}
inline int64_t head_groups(int H, int64_t items) { return (items + 7) / 8 * 8 * H; }

// Eight codes (two words) as a matrix operand.
__device__ __forceinline__ bf16x8 operand(uint32_t lo, uint32_t hi) {
  const u32x4 w = {codes_bf16<false>(lo), codes_bf16<true>(lo), codes_bf16<false>(hi),
                   codes_bf16<true>(hi)};
  return __builtin_bit_cast(bf16x8, w);
}

// Eight fp32 values as TERMS bf16 operands whose sum they are (TERMS 3) or round to.
template <int TERMS>
__device__ __forceinline__ void split_terms(const float (&x)[8], bf16x8 (&out)[TERMS]) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
  for (int t = 0; t < TERMS; ++t) {
    u32x4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      w[k] = pair_bf16(r[2 * k], r[2 * k + 1]);
      if (t + 1 < TERMS) {
        r[2 * k] -= low_bf16(w[k]);
        r[2 * k + 1] -= high_bf16(w[k]);
      }
    }
    out[t] = __builtin_bit_cast(bf16x8, w);
  }
}

// Eight elements of a query row as TERMS operands, times the sign of the softmax scale
// (a.scale_log2 is its magnitude).
template <int TERMS>
__device__ __forceinline__ void load_query(const QAttention& a, int64_t row, int head, int d0,
                                           bool live, bf16x8 (&out)[TERMS]) {
  constexpr int ES = TERMS == 1 ? 2 : 4;
  if (!live) {
#pragma unroll
    for (int t = 0; t < TERMS; ++t) out[t] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
    return;
  }
  const uint8_t* src =
      static_cast<const uint8_t*>(a.q) + (row * a.q_row + (int64_t)head * a.q_head + d0) * ES;
  if constexpr (ES == 2) {
    u32x4 w = *global_ptr<u32x4>(src);
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] ^= a.negate ? 0x80008000u : 0u;
    out[0] = __builtin_bit_cast(bf16x8, w);
  } else {
    const u32x4 w0 = *global_ptr<u32x4>(src), w1 = *(global_ptr<u32x4>(src) + 1);
    float x[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[k] = __uint_as_float(w0[k] ^ (a.negate ? 0x80000000u : 0u));
      x[4 + k] = __uint_as_float(w1[k] ^ (a.negate ? 0x80000000u : 0u));
    }
    split_terms<TERMS>(x, out);
  }
}

// Where a row's results go: row `rr` of the request's rows times the group, KV head h.
struct RowPlace {
  int64_t row;
  int head;
};
__device__ __forceinline__ RowPlace row_place(const QAttention& a, const Item& it, int h, int rr) {
  return {it.row0 + rr / a.G, h * a.G + rr % a.G};
}
template <int ES>
__device__ __forceinline__ void put_quad(const QAttention& a, const RowPlace& p, int col, f32x4 o,
                                         float l) {
  const float inv = l == 0.f ? 0.f : 1.f / l;
  f32x4 y;
#pragma unroll
  for (int c = 0; c < 4; ++c) y[c] = l == 0.f ? 0.f : o[c] * inv;
  const int64_t at = p.row * a.out_row + (int64_t)p.head * a.out_head + col;
  if constexpr (ES == 2)
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + at) =
        u32x2{pair_bf16(y[0], y[1]), pair_bf16(y[2], y[3])};
  else
    *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at) = y;
}
// low: the base-2 exponent that l is relative to (0 where nothing was seen).
__device__ __forceinline__ void put_lse(const QAttention& a, const RowPlace& p, float low, float l) {
  if (a.lse)
    a.lse[p.row * a.H * a.G + p.head] =
        l == 0.f ? kNone : (low + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// Partial results travel between workgroups of different XCDs, whose caches do not see each
// other's lines: they are stored and loaded as atomics of the GPU's scope, which go past
// those caches.
__device__ __forceinline__ void put_part(float* at, float x, float y) {
  const u32x2 w = {__float_as_uint(x), __float_as_uint(y)};
  __hip_atomic_store(reinterpret_cast<uint64_t*>(at), __builtin_bit_cast(uint64_t, w),
                     __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void get_part(const float* at, float& x, float& y) {
  const u32x2 w = __builtin_bit_cast(
      u32x2, __hip_atomic_load(reinterpret_cast<const uint64_t*>(at), __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT));
  x = __uint_as_float(w[0]);
  y = __uint_as_float(w[1]);
}

// Partial results of a segment of few rows: `rows` rows of D values, then the exponent m and the
// sum l of each row: of the segment, and of the group that it is the first of. The values are
// stored as the lanes hold them, two columns of one row after another: a store of a wave fills
// whole lines (row after row it was 8 bytes of 64 lines, which such stores write one by one).
template <int D>
struct Part {
  static constexpr int64_t kFloats = (int64_t)kFewRows * (D + 4);
  float* at;
  int rows;
  __device__ __forceinline__ void put_quad(int row, int q, f32x4 v) const {
    float* p = at + 2 * (2 * q * rows + row);
    put_part(p, v[0], v[1]);
    put_part(p + 2 * rows, v[2], v[3]);
  }
  __device__ __forceinline__ f32x4 quad(int row, int q) const {
    const float* p = at + 2 * (2 * q * rows + row);
    float x[4];
    get_part(p, x[0], x[1]);
    get_part(p + 2 * rows, x[2], x[3]);
    return f32x4{x[0], x[1], x[2], x[3]};
  }
  __device__ __forceinline__ void put_stat(int level, int row, float m, float l) const {
    put_part(at + kFewRows * D + 2 * (kFewRows * level + row), m, l);
  }
  __device__ __forceinline__ void stat(int level, int row, float& m, float& l) const {
    get_part(at + kFewRows * D + 2 * (kFewRows * level + row), m, l);
  }
};
template <int D>
__device__ __forceinline__ Part<D> part_of(const QAttention& a, const Item& it, int h, int place) {
  return {a.few_part + ((int64_t)h * a.few_max + place) * Part<D>::kFloats, it.count * a.G};
}

// x, of which the compiler does not know that it is x: what is computed from it is computed where
// it is used, not kept in registers.
__device__ __forceinline__ int anew(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// The lane's number, computed where it is asked for.
__device__ __forceinline__ int lane_anew() {
  int all = -1;
  asm volatile("" : "+s"(all));
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)all, __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0));
}

// Four columns of a row while they are joined from partial results.
struct Joined {
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float m = kNone, l = 0.f;
  // the first `there` of N results
  template <int N>
  __device__ __forceinline__ void add(f32x4 (&x)[N], float (&xm)[N], float (&xl)[N], int there) {
#pragma unroll
    for (int k = 0; k < N; ++k) {                // (what is not there weighs nothing)
      x[k] = k < there ? x[k] : f32x4{0.f, 0.f, 0.f, 0.f};
      xm[k] = k < there ? xm[k] : kNone;
      xl[k] = k < there ? xl[k] : 0.f;
    }
    float top = m;
#pragma unroll
    for (int k = 0; k < N; ++k) top = fmaxf(top, xm[k]);
    const float low = top == kNone ? 0.f : top;
    const float f = __builtin_amdgcn_exp2f(m - low);
    l *= f;
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] *= f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float w = __builtin_amdgcn_exp2f(xm[k] - low);
      l += w * xl[k];
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] += w * x[k][c];
    }
    m = top;
  }
};

// Joins `count` partial results, in the places slot(0), slot(1), ..: into the output (`whole`)
// or, as the result of a group, into the first of them. In order, by all threads, each
// several quads of columns at a time where there are few results to load for each.
template <int D, int ES, int THREADS, int BATCH, int QUADS, class Slot>
__device__ __forceinline__ void join_some(const QAttention& a, const Item& it, int h, int count,
                                          int level, bool whole, Slot slot) {
  constexpr int kQuads = D / 4;
  const Part<D> p0 = part_of<D>(a, it, h, slot(0));
  const int total = p0.rows * kQuads;
  for (int x0 = anew(threadIdx.x); x0 < total; x0 += THREADS * QUADS) {
    Joined sum[QUADS];
    for (int s = 0; s < count; s += BATCH) {
      f32x4 o[QUADS][BATCH];
      float m[QUADS][BATCH], l[QUADS][BATCH];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const Part<D> p = part_of<D>(a, it, h, slot(s + k < count ? s + k : s));
#pragma unroll
        for (int u = 0; u < QUADS; ++u) {
          const int x = x0 + u * THREADS < total ? x0 + u * THREADS : x0;
          const int quad = (int)((uint32_t)x / (uint32_t)p.rows), row = x - quad * p.rows;
          o[u][k] = p.quad(row, quad);
          p.stat(level, row, m[u][k], l[u][k]);
        }
      }
#pragma unroll
      for (int u = 0; u < QUADS; ++u) sum[u].add(o[u], m[u], l[u], count - s);
    }
#pragma unroll
    for (int u = 0; u < QUADS; ++u) {
      const int x = x0 + u * THREADS;
      if (x >= total) break;
      const int quad = (int)((uint32_t)x / (uint32_t)p0.rows), row = x - quad * p0.rows;
      if (whole) {
        const RowPlace place = row_place(a, it, h, row);
        put_quad<ES>(a, place, 4 * quad, sum[u].o, sum[u].l);
        if (quad == 0) put_lse(a, place, sum[u].m == kNone ? 0.f : sum[u].m, sum[u].l);
      } else {
        p0.put_quad(row, quad, sum[u].o);        // (read by this thread alone)
        if (quad == 0) p0.put_stat(1, row, sum[u].m, sum[u].l);
      }
    }
  }
}
constexpr int kJoin = 16;   // partial results joined at a time
template <int D, int ES, int THREADS, class Slot>
__device__ __forceinline__ void join_parts(const QAttention& a, const Item& it, int h, int count,
                                           int level, bool whole, Slot slot) {
  if (count <= 4) join_some<D, ES, THREADS, 4, 4>(a, it, h, count, level, whole, slot);
  else join_some<D, ES, THREADS, 8, 2>(a, it, h, count, level, whole, slot);
}

// Whether this workgroup is the last of `count` to come to a counter, which the last one
// leaves at zero. The partial results that the others wrote before they came are then there
// for it: every wave waits until its stores have been carried out (they are atomics of
// the GPU's scope: carried out where every XCD sees them) before the barrier, after which one
// thread counts. A release and an acquire of the whole GPU's scope would also write back
// and drop this XCD's cache: with them the 4B-large context took 122 us instead of 109.
__device__ __forceinline__ bool last_to_come(int32_t* counter, int count, int* s_flag) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const bool last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED,
                                             __HIP_MEMORY_SCOPE_AGENT) == count - 1;
    if (last) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *s_flag = last;
  }
  __syncthreads();
  return *s_flag != 0;
}

// After one of `splits` partial results, number `split`, is written: the last workgroup of
// every kJoin of them (more where there are more than kJoin^2) joins these, the last of the
// groups joins the groups. Which workgroup comes last changes nothing: the order of the sums is
// that of the ranges. slot(i) is the place of result i; a place has two counters.
template <int D, int ES, int THREADS, class Slot>
__device__ __forceinline__ void finish_split(const QAttention& a, const Item& it, int h, int split,
                                             int splits, int* s_flag, Slot slot) {
  int32_t* counters = a.few_count + 2 * (int64_t)h * a.few_max;
  int size = kJoin;
  while (size * size < splits) size += kJoin;
  const int group = split / size, groups = (splits + size - 1) / size;
  const int here = group * size, members = splits - here < size ? splits - here : size;
  if (!last_to_come(counters + 2 * slot(here), members, s_flag)) return;
  join_parts<D, ES, THREADS>(a, it, h, members, 0, groups == 1,
                             [&](int i) { return slot(here + i); });
  if (groups == 1) return;
  if (!last_to_come(counters + 2 * slot(0) + 1, groups, s_flag)) return;
  join_parts<D, ES, THREADS>(a, it, h, groups, 1, true, [&](int i) { return slot(i * size); });
}

template <int TERMS, int D>
hipError_t launch_qcache_any_rows(const QAttention& a, uint32_t many, uint32_t few,
                                  hipStream_t stream);

}  // namespace cm
