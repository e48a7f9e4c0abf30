// Attention over the 8-bit paged cache (cm_qcache_attention).
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
// Work is cut along the context: a workgroup takes one KV head and one range of one
// request's tokens for 16 query rows, its four waves a quarter each. Every wave finds
// its range from the lengths (so the grid does not depend on them); ranges of one
// request write partial results, which a second launch joins.
#include <type_traits>

#include "qcache_ops.h"

namespace cm {

namespace {

constexpr int kWaves = 4;
constexpr int kStep = 32;                       // tokens of a wave's step
constexpr int kRows = 16;                       // query rows of a tile
constexpr float kNone = -__builtin_inff();

struct Item {
  int32_t r, tile, split, splits;  // request, row tile, range of its context, how many
  int32_t row0, count, len;        // the request's first row, rows, tokens
  int32_t begin, chunk;            // where its visible context begins, tokens of a range
  bool any;
};

// A request's rows and tokens, within the bounds that the host checked.
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
  len = (int)t;
}

__device__ __forceinline__ int visible_begin(const QAttention& a, int count, int len) {
  if (a.window == 0) return 0;
  const int64_t lo = (int64_t)len - count - a.window + 1;
  return lo > 0 ? (int)(lo & ~(int64_t)(kStep - 1)) : 0;
}

__device__ __forceinline__ int64_t wave_sum(int64_t v) {
#pragma unroll
  for (int by = 1; by < 64; by <<= 1) v += __shfl_xor(v, by);
  return v;
}

// The wave's item from the lengths: every request's context is cut into ranges of
// `chunk` tokens, chunk so that about a.items ranges come out for all row tiles.
__device__ Item find_item(const QAttention& a, int item) {
  const int lane = threadIdx.x & 63;
  constexpr int64_t kUnit = kWaves * kStep;
  int64_t cost = 0;
  for (int base = 0; base < a.n; base += 64) {
    if (base + lane < a.n) {
      int row0, count, len;
      request(a, base + lane, row0, count, len);
      const int64_t tiles = ((int64_t)count * a.G + kRows - 1) / kRows;
      const int64_t ext = len - visible_begin(a, count, len);
      cost += tiles * ((ext + kUnit - 1) / kUnit);
    }
  }
  cost = wave_sum(cost);
  const int64_t chunk = (cost + a.items - 1) / a.items < 1 ? 1 : (cost + a.items - 1) / a.items;
  Item it;
  it.any = false;
  int64_t before = 0;
  for (int base = 0; base < a.n; base += 64) {
    int row0 = 0, count = 0, len = 0, begin = 0;
    int64_t mine = 0, splits = 1, range = 0;
    if (base + lane < a.n) {
      request(a, base + lane, row0, count, len);
      begin = visible_begin(a, count, len);
      const int64_t units = (len - begin + kUnit - 1) / kUnit;
      splits = (units + chunk - 1) / chunk;
      splits = splits < 1 ? 1 : splits;
      range = chunk < units ? chunk : units;
      mine = ((int64_t)count * a.G + kRows - 1) / kRows * splits;
    }
    int64_t upto = mine;
#pragma unroll
    for (int by = 1; by < 64; by <<= 1) {
      const int64_t v = __shfl_up(upto, by);
      if (lane >= by) upto += v;
    }
    const uint64_t past = __ballot(before + upto > item);
    if (past) {
      const int l = __builtin_ctzll(past);
      const int64_t first = before + __shfl(upto - mine, l);
      const int local = (int)(item - first);
      it.r = base + l;
      it.splits = (int)__shfl(splits, l);
      it.tile = local / it.splits;
      it.split = local % it.splits;
      it.row0 = __shfl(row0, l);
      it.count = __shfl(count, l);
      it.len = __shfl(len, l);
      it.begin = __shfl(begin, l);
      it.chunk = (int)(__shfl(range, l) * kUnit);
      it.any = true;
      break;
    }
    before += __shfl(upto, 63);
  }
  it.r = __builtin_amdgcn_readfirstlane(it.r);
  it.tile = __builtin_amdgcn_readfirstlane(it.tile);
  it.split = __builtin_amdgcn_readfirstlane(it.split);
  it.splits = __builtin_amdgcn_readfirstlane(it.splits);
  it.row0 = __builtin_amdgcn_readfirstlane(it.row0);
  it.count = __builtin_amdgcn_readfirstlane(it.count);
  it.len = __builtin_amdgcn_readfirstlane(it.len);
  it.begin = __builtin_amdgcn_readfirstlane(it.begin);
  it.chunk = __builtin_amdgcn_readfirstlane(it.chunk);
  return it;
}

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

// Word of four codes with NaN codes (0x7F, 0xFF) replaced by 0; *seen gathers whether
// there were any.
__device__ __forceinline__ uint32_t without_nan(uint32_t w, uint32_t* nan) {
  // a byte of (w & 0x7F..) + 1 reaches 0x80 only where it was 0x7F
  const uint32_t top = ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
  *nan = top >> 7;                               // 1 in each NaN byte
  return w & ~((top >> 7) * 0xFFu);
}

template <int D>
struct Loaded {
  u32x4 k[2][D / 64];            // [tile][chunk]: 16 codes of token n
  uint32_t v[2][4][D / 64];      // [tile][token 4g + i][word]: D / 16 columns
};

template <int D>
__device__ __forceinline__ void load_v(uint32_t (&dst)[D / 64], const uint8_t* p) {
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

// One lane's part of acc and its rows' statistics.
template <int D>
struct Acc {
  f32x4 o[D / 16];  // o[j][i]: column (4g + i) * D / 16 + j of row n
  float m, l;
};

template <int TERMS, int D>
__global__ __launch_bounds__(64 * kWaves) void qcache_attention_kernel(QAttention a) {
  constexpr int DW = D / 16;                     // columns of a lane
  constexpr int ES = TERMS == 1 ? 2 : 4;         // bytes of a query element
  constexpr int PT = TERMS == 1 ? 2 : 3;         // terms of a probability
  __shared__ float s_acc[kWaves][kRows][D + 4];
  __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = lane & 15, g = lane >> 4;
  const int h = (int)blockIdx.x % a.H, item = (int)blockIdx.x / a.H;
  const Item it = find_item(a, item);
  if (!it.any) return;

  // the lane's query row
  const int rho = it.tile * kRows + n;
  const int tok = rho / a.G;
  const bool live = tok < it.count;
  const int head = h * a.G + rho % a.G;
  const int p = it.len - it.count + tok;         // its position
  const int see_hi = live && p >= 0 ? p + 1 : 0;
  const int see_lo = a.window && p - a.window + 1 > 0 ? p - a.window + 1 : 0;
  // what every row of the tile sees, and what none does
  const int tok_lo = it.tile * kRows / a.G;
  int tok_hi = (it.tile * kRows + kRows - 1) / a.G;
  tok_hi = tok_hi < it.count ? tok_hi : it.count - 1;
  const int p_lo = it.len - it.count + tok_lo, p_hi = it.len - it.count + tok_hi;
  const int all_hi = p_lo + 1;                   // <= 0 where the first row sees nothing
  const int all_lo = a.window && p_hi - a.window + 1 > 0 ? p_hi - a.window + 1 : 0;
  const int none_lo = a.window && p_lo - a.window + 1 > 0 ? p_lo - a.window + 1 : 0;
  const int none_hi = p_hi + 1 > 0 ? p_hi + 1 : 0;

  // the wave's tokens: a quarter of the range, whole steps
  int begin = it.begin + it.split * it.chunk, end = begin + it.chunk;
  end = end < none_hi ? end : none_hi;
  const int quarter = ((end - begin + kWaves * kStep - 1) / (kWaves * kStep)) * kStep;
  begin += wave * quarter;
  end = end < begin + quarter ? end : begin + quarter;
  begin = begin < (none_lo & ~(kStep - 1)) ? (none_lo & ~(kStep - 1)) : begin;

  bf16x8 q[D / 32][TERMS];
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    // elements of chunk c / 2, half c % 2, in the order of the K codes that a lane holds
    const int d0 = (c >> 1) * 64 + g * 16 + (c & 1) * 8;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
    if (live) {
      const uint8_t* src = static_cast<const uint8_t*>(a.q) +
                           ((int64_t)(it.row0 + tok) * a.q_row + (int64_t)head * a.q_head + d0) * ES;
      if constexpr (ES == 2) {
        const u32x4 w = *global_ptr<u32x4>(src);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[2 * k] = low_bf16(w[k]);
          x[2 * k + 1] = high_bf16(w[k]);
        }
      } else {
        const u32x4 w0 = *global_ptr<u32x4>(src), w1 = *(global_ptr<u32x4>(src) + 1);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[k] = __uint_as_float(w0[k]);
          x[4 + k] = __uint_as_float(w1[k]);
        }
      }
    }
    split_terms<TERMS>(x, q[c]);
  }

  Acc<D> acc;
#pragma unroll
  for (int j = 0; j < DW; ++j) acc.o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  acc.m = kNone;
  acc.l = 0.f;

  const int32_t* table = a.table + (int64_t)it.r * a.width;
  const int B = 1 << a.b_shift;
  const int64_t page_codes = ((int64_t)a.H << a.b_shift) * D, head_codes = ((int64_t)h << a.b_shift) * D;
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
    const auto load = [&](int s, Loaded<D>& x) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int tile = 2 * s + b;
        const int64_t page = __builtin_amdgcn_readlane(my_page, tile);
        const int row = (t0 + tile * 16) & (B - 1);
        const int64_t base = page * page_codes + head_codes + (int64_t)row * D;
        const uint8_t* kp = a.kc + base + n * D + g * 16;
#pragma unroll
        for (int c = 0; c < D / 64; ++c) x.k[b][c] = *global_ptr<u32x4>(kp + c * 64);
        const uint8_t* vp = a.vc + base + (4 * g) * D + n * DW;
#pragma unroll
        for (int i = 0; i < 4; ++i) load_v<D>(x.v[b][i], vp + i * D);
      }
    };
    const auto compute = [&](int s, Loaded<D>& x) {
      const int t = t0 + s * kStep;
      f32x4 sc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const bf16x8 k = operand(x.k[b][c][2 * half], x.k[b][c][2 * half + 1]);
#pragma unroll
            for (int w = TERMS - 1; w >= 0; --w)
              sc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[2 * c + half][w], sc[b], 0, 0, 0);
          }
        }
      }
      float vs[2];
      float e[8];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const float f = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_ks), 2 * s + b));
        vs[b] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_vs), 2 * s + b));
#pragma unroll
        for (int i = 0; i < 4; ++i) e[4 * b + i] = sc[b][i] * f;
      }
      // steps that some row sees only in part, and absent pages
      const bool part = t < all_lo || t + kStep > all_hi || ((absent >> (2 * s)) & 3) != 0;
      uint32_t sees = 0xFF;
      if (part) {
        sees = 0;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int tt = t + 16 * b + 4 * g + i;
            const bool ok = tt >= see_lo && tt < see_hi && !((absent >> (2 * s + b)) & 1);
            if (!ok) e[4 * b + i] = kNone;
            sees |= (uint32_t)ok << (4 * b + i);
          }
      }
      float top = e[0];
#pragma unroll
      for (int k = 1; k < 8; ++k) top = fmaxf(top, e[k]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m = fmaxf(acc.m, top);
      const float low = m == kNone ? 0.f : m;
      if (__any(m != acc.m)) {
        const float shrink = __builtin_amdgcn_exp2f(acc.m - low);
        acc.l *= shrink;
#pragma unroll
        for (int j = 0; j < DW; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc.o[j][i] *= shrink;
        acc.m = m;
      }
      float pv[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float pr = __builtin_amdgcn_exp2f(e[k] - low);
        acc.l += pr;
        pv[k] = (sees >> k) & 1 ? pr * vs[k >> 2] : 0.f;
      }
      bf16x8 pt[PT];
      split_terms<PT>(pv, pt);
      // V: in a step that is seen in part, NaN codes are taken out of the product (0 * NaN
      // would reach rows that do not see them) and counted by a product of their own
      bool any_nan = false;
      uint32_t nan[2][4][D / 64];
      if (part) {
        uint32_t seen = 0;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int w = 0; w < D / 64; ++w) {
              x.v[b][i][w] = without_nan(x.v[b][i][w], &nan[b][i][w]);
              seen |= nan[b][i][w];
            }
        any_nan = __any(seen != 0);
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
            const int j = 4 * w + 2 * half + o;
#pragma unroll
            for (int z = PT - 1; z >= 0; --z)
              acc.o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vt),
                                                                 pt[z], acc.o[j], 0, 0, 0);
          }
        }
      }
      if (any_nan) {
        u32x4 seen_by;                           // 1 where the lane's row sees the token
#pragma unroll
        for (int k = 0; k < 4; ++k)
          seen_by[k] = ((sees >> (2 * k)) & 1 ? 0x3F80u : 0u) |
                       ((sees >> (2 * k + 1)) & 1 ? 0x3F800000u : 0u);
#pragma unroll
        for (int j = 0; j < DW; ++j) {
          u32x4 is;                              // 1 where the code is NaN
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t lo = (nan[(2 * k) >> 2][(2 * k) & 3][j >> 2] >> (8 * (j & 3))) & 1;
            const uint32_t hi = (nan[(2 * k + 1) >> 2][(2 * k + 1) & 3][j >> 2] >> (8 * (j & 3))) & 1;
            is[k] = lo * 0x3F80u | hi * 0x3F800000u;
          }
          f32x4 hits = {0.f, 0.f, 0.f, 0.f};
          hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, is),
                                                         __builtin_bit_cast(bf16x8, seen_by), hits,
                                                         0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (hits[i] > 0.f) acc.o[j][i] = __builtin_nanf("");
        }
      }
    };
    Loaded<D> x0, x1;
    load(0, x0);
    for (int s = 0; s < steps; s += 2) {
      if (s + 1 < steps) load(s + 1, x1);
      compute(s, x0);
      if (s + 1 < steps) {
        if (s + 2 < steps) load(s + 2, x0);
        compute(s + 1, x1);
      }
    }
  }

  // the waves' results as one
  acc.l += __shfl_xor(acc.l, 16);
  acc.l += __shfl_xor(acc.l, 32);
  if (g == 0) {
    s_m[wave][n] = acc.m;
    s_l[wave][n] = acc.l;
  }
  {
    float* row = &s_acc[wave][n][4 * g * DW];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < DW; ++j) row[i * DW + j] = acc.o[j][i];
  }
  __syncthreads();
  const int rows = it.count * a.G - it.tile * kRows < kRows ? it.count * a.G - it.tile * kRows : kRows;
  for (int x = threadIdx.x; x < rows * D; x += 64 * kWaves) {
    const int row = x / D, col = x % D;
    float m = kNone;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, s_m[w][row]);
    const float low = m == kNone ? 0.f : m;
    float l = 0.f, o = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(s_m[w][row] - low);
      l += f * s_l[w][row];
      o += f * s_acc[w][row][col];
    }
    if (it.splits == 1) {
      const int rr = it.tile * kRows + row;
      const int64_t at = it.row0 + rr / a.G;
      const int hd = h * a.G + rr % a.G;
      const float y = l == 0.f ? 0.f : o / l;
      const int64_t where = at * a.out_row + (int64_t)hd * a.out_head + col;
      if constexpr (ES == 2) static_cast<__bf16*>(a.out)[where] = (__bf16)y;
      else static_cast<float*>(a.out)[where] = y;
      if (col == 0 && a.lse)
        a.lse[at * a.H * a.G + hd] = l == 0.f ? kNone : (low + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
    } else {
      float* part = a.part + ((int64_t)h * a.max_items + item) * (kRows * (D + 2));
      part[row * (D + 2) + col] = o;
      if (col == 0) {
        part[row * (D + 2) + D] = m;
        part[row * (D + 2) + D + 1] = l;
      }
    }
  }
}

// The partial results of a row tile (items next to each other) as one.
template <int TERMS, int D>
__global__ __launch_bounds__(256) void qcache_join_kernel(QAttention a) {
  constexpr int ES = TERMS == 1 ? 2 : 4;
  const int h = (int)blockIdx.x % a.H, item = (int)blockIdx.x / a.H;
  const Item it = find_item(a, item);
  if (!it.any || it.split != 0 || it.splits == 1) return;
  const float* part = a.part + ((int64_t)h * a.max_items + item) * (kRows * (D + 2));
  const int rows = it.count * a.G - it.tile * kRows < kRows ? it.count * a.G - it.tile * kRows : kRows;
  for (int x = threadIdx.x; x < rows * D; x += 256) {
    const int row = x / D, col = x % D;
    float m = kNone;
    for (int s = 0; s < it.splits; ++s)
      m = fmaxf(m, part[(int64_t)s * (kRows * (D + 2)) + row * (D + 2) + D]);
    const float low = m == kNone ? 0.f : m;
    float l = 0.f, o = 0.f;
    for (int s = 0; s < it.splits; ++s) {
      const float* at = part + (int64_t)s * (kRows * (D + 2)) + row * (D + 2);
      const float f = __builtin_amdgcn_exp2f(at[D] - low);
      l += f * at[D + 1];
      o += f * at[col];
    }
    const int rr = it.tile * kRows + row;
    const int64_t to = it.row0 + rr / a.G;
    const int hd = h * a.G + rr % a.G;
    const float y = l == 0.f ? 0.f : o / l;
    const int64_t where = to * a.out_row + (int64_t)hd * a.out_head + col;
    if constexpr (ES == 2) static_cast<__bf16*>(a.out)[where] = (__bf16)y;
    else static_cast<float*>(a.out)[where] = y;
    if (col == 0 && a.lse)
      a.lse[to * a.H * a.G + hd] = l == 0.f ? kNone : (low + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
  }
}

}  // namespace

QAttentionPlan plan_qcache_attention(int32_t H, int32_t d, int32_t G, int32_t n, int64_t n_rows) {
  QAttentionPlan p;
  const int32_t groups = 2 * device_cu_count();      // workgroups that run together
  p.items = groups / H > 0 ? groups / H : 1;
  // every request's tiles round up once, every tile's ranges once
  const int64_t tiles = (n_rows * G + kRows - 1) / kRows + n;
  p.max_items = (int32_t)(tiles + p.items);
  p.bytes = sizeof(float) * (size_t)H * (size_t)p.max_items * kRows * (size_t)(d + 2);
  return p;
}

hipError_t launch_qcache_attention(const QAttention& a, int32_t d, int32_t dtype,
                                   hipStream_t stream) {
  const dim3 grid((uint32_t)((int64_t)a.max_items * a.H));
  const auto go = [&](auto terms, auto dd) {
    constexpr int TERMS = decltype(terms)::value, D = decltype(dd)::value;
    {
      ScopedTiming tm(K_QCACHE_ATTENTION, stream);
      hipLaunchKernelGGL((qcache_attention_kernel<TERMS, D>), grid, dim3(64 * kWaves), 0, stream, a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    ScopedTiming tm(K_QCACHE_JOIN, stream);
    hipLaunchKernelGGL((qcache_join_kernel<TERMS, D>), grid, dim3(256), 0, stream, a);
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
