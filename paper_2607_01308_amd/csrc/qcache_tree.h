// Attention over the 8-bit paged cache for trees of drafted nodes (cm_qcache_tree_attention).
//
// A request's c nodes are its last c tokens. A node sees the context before them (with a window: the
// part within it) and the nodes whose bits its mask has. The softmax is the one-pass one of the
// decoding steps (qcache_few.h), with the same operands: codes exact in bf16, bf16 queries as they
// are and their weights as two bf16 terms, fp32 ones as three, products added in fp32; weights stay
// relative to an earlier maximum while the new one is less than 2^8 times it.
//
// A wave takes 16 R query rows (nodes times the group) at once: the codes of a step of 32 tokens are
// loaded and turned into operands once for R products of 16 rows each, so that what a step costs
// beside its matrix instructions is shared by all rows. A workgroup's four waves take equal parts of
// a range of the context, each whole steps, without a barrier until the range ends; then they
// are joined through the LDS by all threads. As many workgroups as run together take equal spans of
// all contexts, a request's once for each tile of 16 R rows, laid end to end; where a tile lies in
// several spans, the last workgroup to write its partial results joins them, in their order.
#pragma once

#include "draft.h"
#include "qcache_few.h"

namespace cm {

constexpr int kTreeWaves = 4;
constexpr int kTreeThreads = 64 * kTreeWaves;

// Row tiles of 16 that a wave takes at most: its registers hold D / 4 values of the output and
// D / 8 * terms of the queries for each (these go to the LDS where there are many).
constexpr int tree_tiles_most(int terms, int d) { return terms == 1 ? (d > 128 ? 2 : 4) : (d > 128 ? 1 : 2); }
constexpr bool tree_query_shared(int terms, int d, int tiles) { return terms * d * tiles > 256; }

struct TreeItem {
  int32_t r, tile;             // request, row tile
  int32_t row0, count, nodes;  // first row, rows that are computed, all of them
  int32_t len, held;           // tokens; tokens before the nodes (below 0: nodes without a place)
  int32_t begin, end;          // the range of the context
  int32_t splits;              // ranges of the tile
};

// A request's rows and tokens within the bounds that the host checked; rows that do not lie in
// order within the step are none.
__device__ __forceinline__ void tree_request(const TreeAttention& a, int r, TreeItem& it) {
  const int64_t first = a.a.rows ? a.a.rows[r] : r, next = a.a.rows ? a.a.rows[r + 1] : r + 1;
  const bool good = first >= 0 && next >= first && next <= a.a.n_rows;
  const int64_t cap = a.a.width << a.a.b_shift;
  int64_t t = a.a.lens[r];
  t = t < 0 ? 0 : t > cap ? cap : t;
  it.r = r;
  it.row0 = (int)first;
  it.nodes = good ? (int)(next - first) : 0;
  it.count = it.nodes < a.a.max_rows ? it.nodes : a.a.max_rows;
  it.len = (int)t;
  it.held = (int)(t - it.nodes);
}

// Where what any of a request's rows sees begins, at a multiple of 32.
__device__ __forceinline__ int tree_begin(const TreeAttention& a, const TreeItem& it) {
  if (a.a.window == 0) return 0;
  const int64_t lo = (int64_t)it.held - a.a.window + 1;
  return lo > 0 ? (int)(lo & ~(int64_t)31) : 0;
}
__device__ __forceinline__ int tree_units(const TreeAttention& a, const TreeItem& it) {
  const int units = (int)(((int64_t)it.len - tree_begin(a, it) + a.a.few_unit - 1) / a.a.few_unit);
  return units < 1 ? 1 : units;
}

template <int TERMS, int D, int R>
struct TreeShared {
  static constexpr bool kShared = tree_query_shared(TERMS, D, R);
  static constexpr int kTogether = D > 128 || R == 1 ? 1 : 2;  // row tiles joined at a time
  union {
    bf16x8 q[kShared ? R * (D / 32) * TERMS * 64 : 1];         // [tile][chunk][term][lane]
    float acc[kTreeWaves][16 * kTogether][D + 4];              // the waves' results
  };
  float m[kTreeWaves][16 * R], l[kTreeWaves][16 * R];
  int pos[CM_QCACHE_MAX_REQUESTS + 1];                         // where the requests begin, in units
  float cost[kTreeWaves];
  int sums[kTreeWaves];
  int first;
  int flag;
};

// Partial results of a range: quads of columns in two planes of pairs, row after row, so that a
// wave's stores fill whole lines; then the exponent and the sum of each row.
template <int D, int R>
struct TreePart {
  static constexpr int64_t kFloats = (int64_t)16 * R * (D + 4);
  float* at;
  __device__ __forceinline__ float* pair(int x, int plane) const {
    return at + plane * (16 * R * D / 2) + 2 * x;
  }
  __device__ __forceinline__ void put_quad(int x, f32x4 v) const {
    put_part(pair(x, 0), v[0], v[1]);
    put_part(pair(x, 1), v[2], v[3]);
  }
  __device__ __forceinline__ f32x4 quad(int x) const {
    float v[4];
    get_part(pair(x, 0), v[0], v[1]);
    get_part(pair(x, 1), v[2], v[3]);
    return f32x4{v[0], v[1], v[2], v[3]};
  }
  __device__ __forceinline__ float* stat(int level, int row) const {
    return at + 16 * R * (D + 2 * level) + 2 * row;
  }
};
template <int D, int R>
__device__ __forceinline__ TreePart<D, R> tree_part(const TreeAttention& a, int h, int place) {
  return {a.a.few_part + ((int64_t)h * a.a.few_max + place) * TreePart<D, R>::kFloats};
}

__device__ __forceinline__ RowPlace tree_place(const TreeAttention& a, const TreeItem& it, int h,
                                               int rho) {
  return {it.row0 + rho / a.a.G, h * a.a.G + rho % a.a.G};
}

// Bits lo .. hi - 1 of a word of 32 (any lo, hi).
__device__ __forceinline__ uint32_t bits_between(int64_t lo, int64_t hi) {
  lo = lo < 0 ? 0 : lo;
  hi = hi > 32 ? 32 : hi;
  if (lo >= hi) return 0;
  return (uint32_t)(((uint64_t)1 << hi) - ((uint64_t)1 << lo));
}

// Which of the 32 tokens from t on the node of row `tok` of the request sees.
__device__ __forceinline__ uint32_t tree_sees(const TreeAttention& a, const TreeItem& it, int tok,
                                              int t) {
  if (tok >= it.count) return 0;
  const int64_t row = (int64_t)it.row0 + tok;
  uint32_t sees = 0;
  if (t < it.held) {
    const int64_t lo = a.a.window ? (int64_t)a.positions[row] - a.a.window + 1 : 0;
    sees = bits_between(lo - t, (int64_t)it.held - t);
  }
  const int64_t j0 = (int64_t)t - it.held;       // the first token as a node
  if (j0 + 31 >= 0) {
    const int64_t j = j0 < 0 ? 0 : j0;
    const int64_t word = j >> 6;
    const int shift = (int)(j & 63);
    const uint64_t* mask = a.masks + row * a.words;
    uint64_t x = word < a.words ? mask[word] >> shift : 0;
    if (shift && word + 1 < a.words) x |= mask[word + 1] << (64 - shift);
    sees |= (uint32_t)(j0 < 0 ? x << -j0 : x) & bits_between(j0 < 0 ? -j0 : 0, 32);
  }
  return sees & bits_between(0, (int64_t)it.len - t);
}

// One range: all waves of the workgroup.
template <int TERMS, int D, int R>
__device__ __forceinline__ void tree_segment(const TreeAttention& ta, const TreeItem& it, int h, int slot,
                                             TreeShared<TERMS, D, R>& lds) {
  constexpr int DW = D / 16;                     // columns of a lane
  constexpr int ES = TERMS == 1 ? 2 : 4;
  constexpr int PT = TERMS == 1 ? 2 : 3;         // terms of a weight
  constexpr bool kShared = tree_query_shared(TERMS, D, R);
  const QAttention& a = ta.a;
  const int lane = anew(threadIdx.x & 63), wave = threadIdx.x >> 6;
  const int n = lane & 15, g = lane >> 4;
  const int rho0 = it.tile * 16 * R;

  // the wave's tokens: an equal part of the range, whole steps
  int begin = it.begin, end = it.end < it.len ? it.end : it.len;
  const int steps_all = end > begin ? (end - begin + kStep - 1) / kStep : 0;
  const int share = (steps_all + kTreeWaves - 1) / kTreeWaves * kStep;
  begin += wave * share;
  end = end < begin + share ? end : begin + share;
  // what every row sees
  const int64_t past = (int64_t)it.held + it.nodes - a.window;
  const int all_lo = a.window && past > 0 ? (int)past : 0, all_hi = it.held;

  const auto query = [&](int j, int c, bf16x8 (&dst)[TERMS]) {
    const int rho = rho0 + 16 * j + n, tok = rho / a.G;
    load_query<TERMS>(a, it.row0 + tok, h * a.G + rho % a.G, (c >> 1) * 64 + g * 16 + (c & 1) * 8,
                      tok < it.count, dst);
  };
  bf16x8 q[kShared ? 1 : R][kShared ? 1 : D / 32][TERMS];
  if constexpr (kShared) {
    for (int x = wave; x < R * (D / 32); x += kTreeWaves) {
      query(x / (D / 32), x % (D / 32), q[0][0]);
#pragma unroll
      for (int w = 0; w < TERMS; ++w) lds.q[(x * TERMS + w) * 64 + lane] = q[0][0][w];
    }
    __syncthreads();
  } else {
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
      for (int c = 0; c < D / 32; ++c) query(j, c, q[j][c]);
  }

  f32x4 acc[R][DW];                              // acc[.][j][i]: column (4g + i) * D / 16 + j of row n
  float ref[R], l[R];                            // exponent that acc and l are relative to
#pragma unroll
  for (int j = 0; j < R; ++j) {
    ref[j] = kNone;
    l[j] = 0.f;
#pragma unroll
    for (int c = 0; c < DW; ++c) acc[j][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const int32_t* table = a.table + (int64_t)it.r * a.width;
  const int B = 1 << a.b_shift;
  const int64_t page_codes = ((int64_t)a.H << a.b_shift) * D;
  const int64_t head_codes = ((int64_t)h << a.b_shift) * D;
  const uint32_t k_lane = n * D + g * 16, v_lane = 4 * g * D + n * DW;
  // 64 tiles of 16 tokens at a time: their pages and scales, one lane each
  for (int t0 = begin; t0 < end; t0 += 64 * 16) {
    int32_t my_page = 0;
    // (not 0, also where the softmax scale is: hidden scores are -inf times it)
    float my_ks = 0x1p-126f, my_vs = 0.f;
    const int my_t = t0 + lane * 16;
    bool there = false;
    if (my_t < end) {
      my_page = table[my_t >> a.b_shift];
      there = my_page >= 0 && my_page < a.pages;
      if (!there) my_page = 0;
      my_ks = fmaxf(a.ks[(int64_t)my_page * a.H + h] * a.scale_log2, 0x1p-126f);
      my_vs = a.vs[(int64_t)my_page * a.H + h];
    }
    const uint64_t absent = ~__ballot(there);
    const int steps = ((end < t0 + 1024 ? end : t0 + 1024) - t0 + kStep - 1) / kStep;
    Loaded<D> x;
    const auto base_of = [&](int tile) {
      const int64_t page = __builtin_amdgcn_readlane(my_page, tile);
      return page * page_codes + head_codes + (int64_t)((t0 + tile * 16) & (B - 1)) * D;
    };
    const auto load_k = [&](int s) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint8_t* kp = a.kc + base_of(2 * s + b);
#pragma unroll
        for (int c = 0; c < D / 64; ++c) x.k[b][c] = *global_ptr<u32x4>(kp + (k_lane + c * 64));
      }
    };
    const auto load_v = [&](int s) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint8_t* vp = a.vc + base_of(2 * s + b);
#pragma unroll
        for (int i = 0; i < 4; ++i) load_columns<D>(x.v[b][i], vp + (v_lane + i * D));
      }
    };
    load_k(0);
    load_v(0);
    // K of the next step is on its way from the scores on, V from the products on
    for (int s = 0; s < steps; ++s) {
      const int t = t0 + s * kStep;
      f32x4 sc[R][2];
#pragma unroll
      for (int j = 0; j < R; ++j) sc[j][0] = sc[j][1] = f32x4{0.f, 0.f, 0.f, 0.f};
      const int q_lane = kShared ? anew(lane) : lane;
#pragma unroll
      for (int c = 0; c < D / 64; ++c)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          bf16x8 k[2];
#pragma unroll
          for (int b = 0; b < 2; ++b) k[b] = operand(x.k[b][c][2 * half], x.k[b][c][2 * half + 1]);
#pragma unroll
          for (int j = 0; j < R; ++j)
#pragma unroll
            for (int w = TERMS - 1; w >= 0; --w) {
              bf16x8 qw;
              if constexpr (kShared) qw = lds.q[((j * (D / 32) + 2 * c + half) * TERMS + w) * 64 + q_lane];
              else qw = q[j][2 * c + half][w];
#pragma unroll
              for (int b = 0; b < 2; ++b)
                sc[j][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[b], qw, sc[j][b], 0, 0, 0);
            }
        }
      if (s + 1 < steps) load_k(s + 1);
      float kf[2], vs[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        kf[b] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_ks), 2 * s + b));
        vs[b] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_vs), 2 * s + b));
      }
      // steps that some row sees only in part, or with absent pages
      const bool partly = t < all_lo || t + kStep > all_hi || ((absent >> (2 * s)) & 3) != 0;
      uint32_t sees[R];                          // bit 4 b + i: the lane's tokens
#pragma unroll
      for (int j = 0; j < R; ++j) sees[j] = 0xFFu;
      if (partly) {
        uint32_t there2 = (absent >> (2 * s)) & 1 ? 0u : 0xFFFFu;
        there2 |= (absent >> (2 * s + 1)) & 1 ? 0u : 0xFFFF0000u;
        uint32_t odd = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
          for (int w = 0; w < D / 64; ++w) odd |= nan_codes(x.v[k >> 2][k & 3][w]);
        const bool any_odd = __any(odd != 0);
#pragma unroll
        for (int j = 0; j < R; ++j) {
          const uint32_t y = tree_sees(ta, it, (rho0 + 16 * j + n) / a.G, t) & there2;
          sees[j] = ((y >> (4 * g)) & 0xFu) | ((y >> (16 + 4 * g)) & 0xFu) << 4;
#pragma unroll
          for (int k = 0; k < 8; ++k)
            sc[j][k >> 2][k & 3] = (sees[j] >> k) & 1 ? sc[j][k >> 2][k & 3] : kNone;
        }
        // NaN codes of V are taken out of the product (0 * NaN would reach rows that do
        // not see them); a product of their own finds the rows that do
        if (any_odd) {
#pragma unroll
          for (int w = 0; w < D / 64; ++w) {
            uint32_t bad[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) bad[k] = nan_codes((uint32_t)anew((int)x.v[k >> 2][k & 3][w]));
#pragma unroll
            for (int o = 0; o < 4; ++o) {
              u32x4 is;                          // 1 where the code is NaN
#pragma unroll
              for (int k = 0; k < 4; ++k)
                is[k] = ((bad[2 * k] >> (8 * o)) & 1) * 0x3F80u |
                        ((bad[2 * k + 1] >> (8 * o)) & 1) * 0x3F800000u;
#pragma unroll
              for (int j = 0; j < R; ++j) {
                u32x4 by;                        // 1 where the lane's row sees the token
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  by[k] = ((sees[j] >> (2 * k)) & 1 ? 0x3F80u : 0u) |
                          ((sees[j] >> (2 * k + 1)) & 1 ? 0x3F800000u : 0u);
                f32x4 hits = {0.f, 0.f, 0.f, 0.f};
                hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, is),
                                                               __builtin_bit_cast(bf16x8, by), hits, 0,
                                                               0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  if (hits[i] > 0.f) acc[j][4 * w + o][i] = __builtin_nanf("");
              }
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) x.v[k >> 2][k & 3][w] &= ~(bad[k] * 0xFFu);
          }
        }
      }
      bf16x8 pt[R][PT];
#pragma unroll
      for (int j = 0; j < R; ++j) {
        float best = kNone;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          float y = sc[j][b][0];
#pragma unroll
          for (int i = 1; i < 4; ++i) y = fmaxf(y, sc[j][b][i]);
          best = fmaxf(best, y * kf[b]);
        }
        best = lane_max<32>(lane_max<16>(best));
        if (__any(best > ref[j] + 8.f)) {
          const float m = fmaxf(ref[j], best);
          const float shrink = m == kNone ? 1.f : __builtin_amdgcn_exp2f(ref[j] - m);
          l[j] *= shrink;
#pragma unroll
          for (int c = 0; c < DW; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[j][c][i] *= shrink;
          ref[j] = m;
        }
        const float low = ref[j] == kNone ? 0.f : ref[j];
        float pv[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float pr = __builtin_amdgcn_exp2f(fmaf(sc[j][k >> 2][k & 3], kf[k >> 2], -low));
          l[j] += pr;
          pv[k] = pr * vs[k >> 2];
        }
        if (partly) {                            // (a scale may be NaN where nothing is seen)
#pragma unroll
          for (int k = 0; k < 8; ++k) pv[k] = (sees[j] >> k) & 1 ? pv[k] : 0.f;
        }
        split_terms<PT>(pv, pt[j]);
      }
#pragma unroll
      for (int w = 0; w < D / 64; ++w) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t c[8];
#pragma unroll
          for (int k = 0; k < 8; ++k)
            c[k] = half ? codes_bf16<true>(x.v[k >> 2][k & 3][w]) : codes_bf16<false>(x.v[k >> 2][k & 3][w]);
#pragma unroll
          for (int o = 0; o < 2; ++o) {
            u32x4 vt;
#pragma unroll
            for (int k = 0; k < 4; ++k)
              vt[k] = __builtin_amdgcn_perm(c[2 * k + 1], c[2 * k], o ? 0x07060302u : 0x05040100u);
            const int col = 4 * w + 2 * half + o;
#pragma unroll
            for (int z = PT - 1; z >= 0; --z)
#pragma unroll
              for (int j = 0; j < R; ++j)
                acc[j][col] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vt),
                                                                      pt[j][z], acc[j][col], 0, 0, 0);
          }
        }
      }
      if (s + 1 < steps) load_v(s + 1);
    }
  }

  // the waves' results as one, by all threads, kTogether row tiles at a time
  constexpr int kTogether = TreeShared<TERMS, D, R>::kTogether;
  const int en = anew(n), eg = anew(g);
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const float sum = lane_sum<32>(lane_sum<16>(l[j]));
    if (eg == 0) {
      lds.m[wave][16 * j + en] = ref[j];
      lds.l[wave][16 * j + en] = sum;
    }
  }
  const int live = it.count * a.G - rho0;        // rows of the tile that there are
  const TreePart<D, R> part = tree_part<D, R>(ta, h, slot);
#pragma unroll
  for (int j0 = 0; j0 < R; j0 += kTogether) {
    __syncthreads();                             // (also: the queries in the LDS are not needed now)
#pragma unroll
    for (int jj = 0; jj < kTogether; ++jj) {
      float* row = &lds.acc[wave][16 * jj + en][4 * eg * DW];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < DW; c += 4)
          *reinterpret_cast<f32x4*>(&row[i * DW + c]) =
              f32x4{acc[j0 + jj][c][i], acc[j0 + jj][c + 1][i], acc[j0 + jj][c + 2][i],
                    acc[j0 + jj][c + 3][i]};
    }
    __syncthreads();
    constexpr int kQuads = D / 4;
    for (int y = anew(threadIdx.x); y < 16 * kTogether * kQuads; y += kTreeThreads) {
      const int quad = y % kQuads, within = y / kQuads, row = 16 * j0 + within;
      if (row >= live) break;
      float m = lds.m[0][row];
#pragma unroll
      for (int w = 1; w < kTreeWaves; ++w) m = fmaxf(m, lds.m[w][row]);
      const float low = m == kNone ? 0.f : m;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < kTreeWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(lds.m[w][row] - low);
        const f32x4 v = *reinterpret_cast<const f32x4*>(&lds.acc[w][within][4 * quad]);
        sum += f * lds.l[w][row];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] += f * v[i];
      }
      if (it.splits == 1) {
        const RowPlace place = tree_place(ta, it, h, rho0 + row);
        put_quad<ES>(a, place, 4 * quad, o, sum);
        if (quad == 0) put_lse(a, place, low, sum);
      } else {
        part.put_quad(row * kQuads + quad, o);
        if (quad == 0) put_part(part.stat(0, row), m, sum);
      }
    }
  }
  __syncthreads();                               // (the LDS is the next range's)
}

// Joins `count` partial results of a tile, in the places slot(0), slot(1), ..: into the output (`whole`)
// or, as the result of a group, into the first of them.
template <int D, int R, int ES, class Slot>
__device__ __forceinline__ void tree_join(const TreeAttention& ta, const TreeItem& it, int h, int count,
                                          int level, bool whole, Slot slot) {
  constexpr int kQuads = D / 4, kBatch = 8;
  const int rho0 = it.tile * 16 * R;
  const int live = it.count * ta.a.G - rho0;
  const int total = (live < 16 * R ? live : 16 * R) * kQuads;
  const TreePart<D, R> p0 = tree_part<D, R>(ta, h, slot(0));
  for (int x = anew(threadIdx.x); x < total; x += kTreeThreads) {
    const int row = x / kQuads;
    Joined sum;
    for (int s = 0; s < count; s += kBatch) {
      f32x4 o[kBatch];
      float m[kBatch], l[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const TreePart<D, R> p = tree_part<D, R>(ta, h, slot(s + k < count ? s + k : s));
        o[k] = p.quad(x);
        get_part(p.stat(level, row), m[k], l[k]);
      }
      sum.add(o, m, l, count - s);
    }
    if (whole) {
      const RowPlace place = tree_place(ta, it, h, rho0 + row);
      put_quad<ES>(ta.a, place, 4 * (x % kQuads), sum.o, sum.l);
      if (x % kQuads == 0) put_lse(ta.a, place, sum.m == kNone ? 0.f : sum.m, sum.l);
    } else {
      p0.put_quad(x, sum.o);                     // (read by this thread alone)
      if (x % kQuads == 0) put_part(p0.stat(1, row), sum.m, sum.l);
    }
  }
}

// After one of a tile's partial results, number `split`, is written: the last workgroup of every
// kJoin of them (more where there are more than kJoin^2) joins these, the last of the groups joins the
// groups. Which workgroup comes last changes nothing.
template <int D, int R, int ES, class Slot>
__device__ __forceinline__ void tree_finish(const TreeAttention& ta, const TreeItem& it, int h, int split,
                                            int* s_flag, Slot slot) {
  int32_t* counters = ta.a.few_count + 2 * (int64_t)h * ta.a.few_max;
  const int splits = it.splits;
  int size = kJoin;
  while (size * size < splits) size += kJoin;
  const int group = split / size, groups = (splits + size - 1) / size;
  const int here = group * size, members = splits - here < size ? splits - here : size;
  if (!last_to_come(counters + 2 * slot(here), members, s_flag)) return;
  tree_join<D, R, ES>(ta, it, h, members, 0, groups == 1, [&](int i) { return slot(here + i); });
  if (groups == 1) return;
  if (!last_to_come(counters + 2 * slot(0) + 1, groups, s_flag)) return;
  tree_join<D, R, ES>(ta, it, h, groups, 1, true, [&](int i) { return slot(i * size); });
}

// The ranges of a workgroup's span, one after another.
template <int TERMS, int D, int R>
__global__ __launch_bounds__(kTreeThreads, 2) void qcache_tree_kernel(TreeAttention ta) {
  __shared__ TreeShared<TERMS, D, R> lds;
  constexpr int ES = TERMS == 1 ? 2 : 4;
  constexpr int kPer = CM_QCACHE_MAX_REQUESTS / kTreeThreads;
  const QAttention& a = ta.a;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const HeadItem hi = head_item(a.H, blockIdx.x);
  const int h = hi.h, w = hi.item;
  if (w >= a.few_items) return;

  // where every request begins: prefix sums of the units of all its tiles
  const int per = (a.n + kTreeThreads - 1) / kTreeThreads;
  int units[kPer], mine = 0;
  float cost = 0.f;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int r = (int)threadIdx.x * per + k;
    units[k] = 0;
    if (k < per && r < a.n) {
      TreeItem it;
      tree_request(ta, r, it);
      const int tiles = (it.count * a.G + 16 * R - 1) / (16 * R);
      if (tiles) {
        units[k] = tiles * tree_units(ta, it);
        cost += (float)tiles * (float)tree_units(ta, it);
      }
    }
    mine += units[k];
  }
  const int upto = wave_scan(mine);
  cost = wave_scan(cost);
  if (lane == 63) {
    lds.sums[wave] = upto;
    lds.cost[wave] = cost;
  }
  __syncthreads();
  int at = upto - mine, total = 0;
  cost = 0.f;
#pragma unroll
  for (int v = 0; v < kTreeWaves; ++v) {
    if (v < wave) at += lds.sums[v];
    total += lds.sums[v];
    cost += lds.cost[v];
  }
  // (rows that lie over one another: more units than an int holds, which nobody takes)
  if (cost > 2e9f) return;
  total = __builtin_amdgcn_readfirstlane(total);
  int span = (total + a.few_items - 1) / a.few_items;
  span = span < ta.least ? ta.least : span;
  int u = w * span;
  const int stop = u + span < total ? u + span : total;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int r = (int)threadIdx.x * per + k;
    if (k < per && r < a.n) {
      lds.pos[r] = at;
      if (u >= at && u < at + units[k]) lds.first = r;
    }
    at += units[k];
  }
  if (threadIdx.x == 0) lds.pos[a.n] = total;
  __syncthreads();
  if (u >= total) return;

  int r = __builtin_amdgcn_readfirstlane(lds.first);
  while (u < stop) {
    const int from = __builtin_amdgcn_readfirstlane(lds.pos[r]);
    const int to = __builtin_amdgcn_readfirstlane(lds.pos[r + 1]);
    if (u >= to) {                               // (a request without rows)
      ++r;
      continue;
    }
    TreeItem it;
    tree_request(ta, r, it);
    const int each = tree_units(ta, it);
    it.tile = (u - from) / each;
    const int tile_from = from + it.tile * each, tile_to = tile_from + each;
    const int u0 = u;
    u = tile_to < stop ? tile_to : stop;
    const int begin = tree_begin(ta, it);
    it.begin = begin + (u0 - tile_from) * a.few_unit;
    const int64_t end = begin + (int64_t)(u - tile_from) * a.few_unit;
    it.end = end < it.len ? (int)end : it.len;
    const int first = tile_from / span, part = w - first;
    it.splits = (tile_to - 1) / span - first + 1;
    // (in the first of them another range may come before it)
    const auto slot = [&](int i) {
      return i == 0 ? 2 * first + (tile_from > first * span ? 1 : 0) : 2 * (first + i);
    };
    tree_segment<TERMS, D, R>(ta, it, h, slot(part), lds);
    if (it.splits > 1) tree_finish<D, R, ES>(ta, it, h, part, &lds.flag, slot);
    if (u == to) ++r;
  }
}

template <int TERMS>
hipError_t launch_tree(const TreeAttention& a, int32_t d, int32_t tiles, uint32_t groups,
                       hipStream_t stream) {
  const auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(groups), dim3(kTreeThreads), 0, stream, a);
    return hipGetLastError();
  };
  if (d == 64) {
    if constexpr (TERMS == 1)
      if (tiles == 4) return go(qcache_tree_kernel<TERMS, 64, 4>);
    return tiles == 1 ? go(qcache_tree_kernel<TERMS, 64, 1>) : go(qcache_tree_kernel<TERMS, 64, 2>);
  }
  if (d == 128) {
    if constexpr (TERMS == 1)
      if (tiles == 4) return go(qcache_tree_kernel<TERMS, 128, 4>);
    return tiles == 1 ? go(qcache_tree_kernel<TERMS, 128, 1>) : go(qcache_tree_kernel<TERMS, 128, 2>);
  }
  if constexpr (TERMS == 1)
    if (tiles == 2) return go(qcache_tree_kernel<TERMS, 256, 2>);
  return go(qcache_tree_kernel<TERMS, 256, 1>);
}
// (a file for each type of the queries: they are built side by side)
hipError_t launch_tree_bf16(const TreeAttention& a, int32_t d, int32_t tiles, uint32_t groups,
                            hipStream_t stream);
hipError_t launch_tree_fp32(const TreeAttention& a, int32_t d, int32_t tiles, uint32_t groups,
                            hipStream_t stream);

}  // namespace cm
