// Attention over the 8-bit paged cache for requests with few query rows: decoding steps.
//
// One pass over the visible keys with the running maximum m and sum l of the softmax:
// for a step of 32 tokens, x = q . k, m' = max(m, x), the accumulators and l are scaled
// by 2^(m - m'), p = 2^(x - m'), l += p, acc += p v; out = acc / l. Exponents are to the
// base 2 (log2 e is part of the score's factor). A page's K scale multiplies its scores
// and its V scale its probabilities, so the products run on the codes, which are exact
// in bf16. Queries of bf16 enter them as they are and probabilities as the sum of two
// bf16 terms (16 bits: the output's own rounding is then what is left of the error, and
// the memory, not the matrix units, is the bound); fp32 queries and their probabilities as
// the sum of three, which holds all 24 bits. Products are added in fp32.
//
// Layout of a wave's step. Both products are computed transposed, S^T = K Q^T and
// out^T = V^T P^T, by 16x16x32 matrix instructions: a lane (n = lane % 16, g = lane / 16)
// then holds of S^T the query row n and the tokens 4g .. 4g + 3 of each 16-token tile,
// which are the eight tokens that it has to supply of P^T if its k index counts
// {tile a: 4g .. 4g + 3, tile b: 4g .. 4g + 3}: the probabilities never leave their lane.
// The V operand of that lane is 8 tokens of one column; the lane loads d / 16 adjacent
// columns of its 8 tokens, so that column tile j is columns n * d / 16 + j, and transposes
// pairs of tokens by one v_perm for two values. A tile of 16 tokens never leaves its page.
//
// Work is cut along the contexts, laid end to end: as many workgroups as run together take
// equal spans of them for one KV head each, whatever the requests' lengths. A span may
// end one request, hold some whole and begin another; its waves take equal parts of each
// request's tokens in it. Where a request lies in several spans its partial results are
// joined by the last workgroups to write theirs. The spans follow from the lengths in
// device memory, which every workgroup looks at; the grid does not depend on them.
//
// Bound by HBM for long contexts: 64 ragged contexts, 8 heads of d = 128, G 4, 1.09 GB, 201 us, 5.4
// TB/s; 264 thousand tokens of one request 109 us, 5.0 TB/s, of each about 12 us at its start and
// in its joins. Pages in order instead of shuffled, pages of 128 tokens, and loads two steps ahead
// changed these by 1 to 2%; three workgroups on a compute unit made contexts of d = 64 5 to 8% faster
// and the long one of d = 128 6% slower. Below about 20 MB bound by the chain of loads from
// the lengths (twice: for the spans, and for the request) to the codes and back through the join:
// 1280 tokens 12.5 us.
#pragma once

#include "qcache_attention.h"

namespace cm {

constexpr int kStep = 32;  // tokens of a wave's step
constexpr int kSolo = 512;  // tokens up to which a wave takes a request by itself

template <int D>
struct Loaded {
  u32x4 k[2][D / 64];            // [tile][chunk]: 16 codes of token n
  uint32_t v[2][4][D / 64];      // [tile][token 4g + i][word]: D / 16 columns
};

template <int D>
__device__ __forceinline__ void load_columns(uint32_t (&dst)[D / 64], const uint8_t* p) {
  if constexpr (D == 64) {
    dst[0] = *global_ptr<uint32_t>(p);
  } else if constexpr (D == 128) {
    const u32x2 w = *global_ptr<u32x2>(p);
    dst[0] = w[0];
    dst[1] = w[1];
  } else {
    const u32x4 w = *global_ptr<u32x4>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) dst[k] = w[k];
  }
}

// Whether the queries lie in the LDS: three terms of d = 256 are 96 registers a lane, for which
// there is no room (spilled, 64 contexts of 8192 tokens of 4 heads took 261 us, not 208).
constexpr bool shared_query(int terms, int d) { return terms * d > 512; }

// What the threads of a workgroup share.
template <int TERMS, int D, int WAVES>
struct FewShared {
  bf16x8 q[shared_query(TERMS, D) ? D / 32 * TERMS * 64 : 1];  // [chunk][term][lane]
  float acc[WAVES / 2][kFewRows][D + 4];         // results of the waves, at a segment's end
  float m[WAVES / 2][kFewRows], l[WAVES / 2][kFewRows];
  int pos[CM_QCACHE_MAX_REQUESTS + 1];           // where the requests begin, in units
  int sums[WAVES];
  int first;
  int flag;
};

// Units of a request that this kernel takes; at least one, whose workgroup writes the output.
__device__ __forceinline__ int few_units(const QAttention& a, int count, int len) {
  if (count == 0 || !few_rows((int64_t)count * a.G)) return 0;
  const int units = (len - visible_begin(a, count, len) + a.few_unit - 1) / a.few_unit;
  return units < 1 ? 1 : units;
}

// solo: the segment is this wave's alone; else all waves of the workgroup come here with it.
template <int TERMS, int D, int WAVES>
__device__ __forceinline__ void few_rows_segment(const QAttention& a, const Item& it, int h, int slot,
                                                 bool solo, FewShared<TERMS, D, WAVES>& lds) {
  constexpr int DW = D / 16;                     // columns of a lane
  constexpr int ES = TERMS == 1 ? 2 : 4;         // bytes of a query element
  constexpr int PT = TERMS == 1 ? 2 : 3;         // terms of a probability
  // (The lane's numbers are made anew for each segment and for its end: addresses made from
  // them before would be kept in registers through the loop, which for d = 256 has none left.)
  const int lane = anew(threadIdx.x & 63), wave = threadIdx.x >> 6;
  const int n = lane & 15, g = lane >> 4;

  // the lane's query row
  const int rho = it.tile * kFewRows + n;
  const int tok = rho / a.G;
  const bool live = tok < it.count;
  const int head = h * a.G + rho % a.G;
  const int p = it.len - it.count + tok;         // its position
  const int see_hi = live && p >= 0 ? p + 1 : 0;
  const int see_lo = a.window && see_hi > a.window ? see_hi - a.window : 0;
  const Sight sight = tile_sight<kFewRows>(a, it);

  // the wave's tokens: an equal part of the range (solo: all of it), whole steps
  int begin = it.begin, end = begin + it.chunk;
  const int from = sight.any_lo & ~(kStep - 1);
  begin = begin > from ? begin : from;
  end = end < sight.any_hi ? end : sight.any_hi;
  const int steps_all = end > begin ? (end - begin + kStep - 1) / kStep : 0;
  const int share = (solo ? steps_all : (steps_all + WAVES - 1) / WAVES) * kStep;
  begin += solo ? 0 : wave * share;
  end = end < begin + share ? end : begin + share;

  // elements of chunk c / 2, half c % 2, in the order of the K codes that a lane holds
  const auto query = [&](int c, bf16x8 (&dst)[TERMS]) {
    load_query<TERMS>(a, it.row0 + tok, head, (c >> 1) * 64 + g * 16 + (c & 1) * 8, live, dst);
  };
  constexpr bool kShared = shared_query(TERMS, D);
  bf16x8 q[kShared ? 1 : D / 32][TERMS];
  if constexpr (kShared) {
    for (int c = wave; c < D / 32; c += WAVES) {
      query(c, q[0]);
#pragma unroll
      for (int w = 0; w < TERMS; ++w) lds.q[(c * TERMS + w) * 64 + lane] = q[0][w];
    }
    __syncthreads();                             // (its readers end at the next barrier)
  } else {
#pragma unroll
    for (int c = 0; c < D / 32; ++c) query(c, q[c]);
  }

  f32x4 acc[DW];                                 // acc[j][i]: column (4g + i) * D / 16 + j of row n
#pragma unroll
  for (int j = 0; j < DW; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  float top = kNone, l = 0.f;                    // the row's maximum; this lane's part of its sum

  const int32_t* table = a.table + (int64_t)it.r * a.width;
  const int B = 1 << a.b_shift;
  const int64_t page_codes = ((int64_t)a.H << a.b_shift) * D;
  const int64_t head_codes = ((int64_t)h << a.b_shift) * D;
  const uint32_t k_lane = n * D + g * 16, v_lane = 4 * g * D + n * DW;
  // 64 tiles at a time: their pages and scales, one lane each
  for (int t0 = begin; t0 < end; t0 += 64 * 16) {
    int32_t my_page = 0;
    float my_ks = 0.f, my_vs = 0.f;
    const int my_t = t0 + lane * 16;
    bool there = false;
    if (my_t < end) {
      my_page = table[my_t >> a.b_shift];
      there = my_page >= 0 && my_page < a.pages;
      if (!there) my_page = 0;
      my_ks = a.ks[(int64_t)my_page * a.H + h] * a.scale_log2;
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
      f32x4 sc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
      const int q_lane = kShared ? anew(lane) : lane;
      const auto of_query = [&](int c, int w) {
        if constexpr (kShared) return lds.q[(c * TERMS + w) * 64 + q_lane];
        else return q[c][w];
      };
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const bf16x8 k = operand(x.k[b][c][2 * half], x.k[b][c][2 * half + 1]);
#pragma unroll
            for (int w = TERMS - 1; w >= 0; --w)
              sc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, of_query(2 * c + half, w), sc[b],
                                                              0, 0, 0);
          }
        }
      }
      if (s + 1 < steps) load_k(s + 1);
      float vs[8], e[8];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const float f = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_ks), 2 * s + b));
        const float v = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_vs), 2 * s + b));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          e[4 * b + i] = sc[b][i] * f;
          vs[4 * b + i] = v;
        }
      }
      // steps that some row sees only in part, or with absent pages
      if (t < sight.all_lo || t + kStep > sight.all_hi || ((absent >> (2 * s)) & 3) != 0) {
        uint32_t sees = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int tt = t + 16 * (k >> 2) + 4 * g + (k & 3);
          const bool ok = tt >= see_lo && tt < see_hi && !((absent >> (2 * s + (k >> 2))) & 1);
          e[k] = ok ? e[k] : kNone;
          vs[k] = ok ? vs[k] : 0.f;              // (a scale may be NaN where nothing is seen)
          sees |= (uint32_t)ok << k;
        }
        // NaN codes of V are taken out of the product (0 * NaN would reach rows that do
        // not see them); a product of their own finds the rows that do
        uint32_t seen = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
          for (int w = 0; w < D / 64; ++w) seen |= nan_codes(x.v[k >> 2][k & 3][w]);
        if (__any(seen != 0)) {
          u32x4 by;                              // 1 where the lane's row sees the token
#pragma unroll
          for (int k = 0; k < 4; ++k)
            by[k] = ((sees >> (2 * k)) & 1 ? 0x3F80u : 0u) |
                    ((sees >> (2 * k + 1)) & 1 ? 0x3F800000u : 0u);
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
              f32x4 hits = {0.f, 0.f, 0.f, 0.f};
              hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, is),
                                                             __builtin_bit_cast(bf16x8, by), hits, 0,
                                                             0, 0);
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (hits[i] > 0.f) acc[4 * w + o][i] = __builtin_nanf("");
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) x.v[k >> 2][k & 3][w] &= ~(bad[k] * 0xFFu);
          }
        }
      }
      float best = e[0];
#pragma unroll
      for (int k = 1; k < 8; ++k) best = fmaxf(best, e[k]);
      best = lane_max<32>(lane_max<16>(best));
      const float m = fmaxf(top, best);
      const float low = m == kNone ? 0.f : m;
      if (__any(m != top)) {
        const float shrink = __builtin_amdgcn_exp2f(top - low);
        l *= shrink;
#pragma unroll
        for (int j = 0; j < DW; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[j][i] *= shrink;
        top = m;
      }
      float pv[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float pr = __builtin_amdgcn_exp2f(e[k] - low);
        l += pr;
        pv[k] = pr * vs[k];
      }
      bf16x8 pt[PT];
      split_terms<PT>(pv, pt);
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
            const int j = 4 * w + 2 * half + o;
#pragma unroll
            for (int z = PT - 1; z >= 0; --z)
              acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vt), pt[z],
                                                               acc[j], 0, 0, 0);
          }
        }
      }
      if (s + 1 < steps) load_v(s + 1);
    }
  }

  // the waves' results as one, half of the waves to the other half at a time (where they have
  // any: of up to WAVES steps a wave has one)
  l = lane_sum<32>(lane_sum<16>(l));
  const int en = anew(n), eg = anew(g);
#pragma unroll
  for (int half = WAVES / 2; half >= 1; half >>= 1) {
    if (solo || (!kShared && steps_all <= half)) continue;
    if (wave >= half && wave < 2 * half) {
      const int to = wave - half;
      float* row = &lds.acc[to][en][4 * eg * DW];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < DW; j += 4)
          *reinterpret_cast<f32x4*>(&row[i * DW + j]) =
              f32x4{acc[j][i], acc[j + 1][i], acc[j + 2][i], acc[j + 3][i]};
      if (eg == 0) {
        lds.m[to][en] = top;
        lds.l[to][en] = l;
      }
    }
    __syncthreads();
    if (wave < half) {
      const float* row = &lds.acc[wave][en][4 * eg * DW];
      const float m = fmaxf(top, lds.m[wave][en]);
      const float low = m == kNone ? 0.f : m;
      const float mine = __builtin_amdgcn_exp2f(top - low);
      const float other = __builtin_amdgcn_exp2f(lds.m[wave][en] - low);
      l = l * mine + other * lds.l[wave][en];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < DW; ++j) acc[j][i] = acc[j][i] * mine + other * row[i * DW + j];
      top = m;
    }
    __syncthreads();
  }
  if ((solo || wave == 0) && live) {
    const Part<D> part = part_of<D>(a, it, h, slot);
    const RowPlace place = row_place(a, it, h, it.tile * kFewRows + en);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < DW; j += 4) {
        const f32x4 y = {acc[j][i], acc[j + 1][i], acc[j + 2][i], acc[j + 3][i]};
        const int col = (4 * eg + i) * DW + j;
        if (it.splits == 1) put_quad<ES>(a, place, col, y, l);
        else part.put_quad(en, col / 4, y);
      }
    if (eg == 0) {
      if (it.splits == 1) put_lse(a, place, top == kNone ? 0.f : top, l);
      else part.put_stat(0, en, top, l);
    }
  }
}

// The segments of a workgroup's span, one after another.
template <int TERMS, int D, int WAVES>
__device__ __forceinline__ void few_rows_span(const QAttention& a, int block,
                                              FewShared<TERMS, D, WAVES>& lds) {
  constexpr int ES = TERMS == 1 ? 2 : 4;
  constexpr int kThreads = 64 * WAVES, kPer = CM_QCACHE_MAX_REQUESTS / kThreads;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const HeadItem hi = head_item(a.H, block);
  const int h = hi.h, w = hi.item;
  if (w >= a.few_items) return;

  // where every request begins: prefix sums of the units
  const int per = (a.n + kThreads - 1) / kThreads;
  int units[kPer], mine = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int r = (int)threadIdx.x * per + k;
    units[k] = 0;
    if (k < per && r < a.n) {
      int row0, count, len;
      request(a, r, row0, count, len);
      units[k] = few_units(a, count, len);
    }
    mine += units[k];
  }
  const int upto = wave_scan(mine);
  if (lane == 63) lds.sums[wave] = upto;
  __syncthreads();
  int at = upto - mine, total = 0;
#pragma unroll
  for (int v = 0; v < WAVES; ++v) {
    if (v < wave) at += lds.sums[v];
    total += lds.sums[v];
  }
  total = __builtin_amdgcn_readfirstlane(total);
  const int span = (total + a.few_items - 1) / a.few_items;
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

  Item it;
  it.tile = 0;
  it.any = 1;
  const int begin = u;
  const int first_r = __builtin_amdgcn_readfirstlane(lds.first);
  const int my_turn = __builtin_amdgcn_readfirstlane(wave);
  // Requests of up to kSolo tokens that lie whole in the span, two of them or more: a wave takes
  // each by itself, the next wave the next one. A segment of such a length is a chain of loads and
  // a join of the waves that no bandwidth shortens (1000 requests of 100 tokens, 8 heads of d = 128:
  // 61 us so, 108 by all waves one after another; 320 of 300 tokens 48, 55 where only 256 tokens
  // count as short). Then the others, by all waves.
  const auto short_one = [&](int from, int to) {
    return from >= begin && to <= stop && to > from && (int64_t)(to - from) * a.few_unit <= kSolo;
  };
  int pass = 1;
  if constexpr (!shared_query(TERMS, D)) {
    const int r = first_r + lane;
    const bool is = r < a.n && short_one(lds.pos[r], lds.pos[r + 1]);
    if (__builtin_popcountll(__ballot(is)) > 1) pass = 0;
  }
  const bool some_solo = pass == 0;
  int r = first_r, turn = 0;
  while (true) {
    if (u >= stop) {
      if (pass == 1) break;
      pass = 1;
      u = begin;
      r = first_r;
    }
    const int from = __builtin_amdgcn_readfirstlane(lds.pos[r]);
    const int to = __builtin_amdgcn_readfirstlane(lds.pos[r + 1]);
    if (from != to) {
      const int u0 = u;
      u = to < stop ? to : stop;
      const bool solo = some_solo && short_one(from, to);
      if (solo == (pass == 0) && (!solo || turn++ % WAVES == my_turn)) {
        request(a, r, it.row0, it.count, it.len);
        it.r = r;
        it.begin = visible_begin(a, it.count, it.len) + (u0 - from) * a.few_unit;
        it.chunk = (u - u0) * a.few_unit;
        // the spans that hold some of it
        const int first = from / span, part = w - first;
        it.splits = (to - 1) / span - first + 1;
        // (in the first of them another request may come before it)
        const auto slot = [&](int i) {
          return i == 0 ? 2 * first + (from > first * span ? 1 : 0) : 2 * (first + i);
        };
        few_rows_segment<TERMS, D, WAVES>(a, it, h, slot(part), solo, lds);
        if (it.splits > 1)
          finish_split<D, ES, kThreads>(a, it, h, part, it.splits, &lds.flag, slot);
      }
    }
    ++r;
  }
}

}  // namespace cm
