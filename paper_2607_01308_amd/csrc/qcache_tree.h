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
// are joined through the LDS by all threads. A page's V scale is part of V's operand, which all rows of the
// wave share: one that is not finite is taken as 1 there, like K's, and the rows that see it are made NaN
// at the range's end (done among the products it cost 7% with 64 rows a wave, in registers). As many workgroups as run together take equal spans of
// all contexts, a request's once for each tile of 16 R rows, laid end to end, or begun anew with every tile
// where that is no longer; a second launch joins the tiles that lie in several spans, in their order.
//
// What bounds it with 64 rows a wave (bf16, d = 128): a step's 96 matrix instructions take 1536 clocks of
// a SIMD, its 350 vector instructions, 32 of them exponentials, about 1800; two waves share a SIMD and
// overlap in part. 128 rows over 264 thousand tokens: 249 us, 0.83 PFLOP/s of matrix instructions (a
// third of them the weights' second term), 2.2 TB/s of codes.
#pragma once

#include "draft.h"
#include "qcache_few.h"

namespace cm {

constexpr int kTreeWaves = 4;
constexpr int kTreeRange = 2;                    // what a range costs beside its units, in units
constexpr int kTreeThreads = 64 * kTreeWaves;

// Row tiles of 16 that a wave takes at most: its registers hold D / 4 values of the output and
// D / 8 * terms of the queries for each (these go to the LDS where there are many).
constexpr int tree_tiles_most(int terms, int d) { return terms == 1 ? (d > 128 ? 2 : 4) : (d > 128 ? 1 : 2); }
constexpr bool tree_query_shared(int terms, int d, int tiles) { return terms * d * tiles >= 256; }
// Workgroups of a compute unit, and steps that a wave's loads are ahead of it.
constexpr int kTreeGroups = 2;
constexpr int tree_ahead(int terms, int d, int tiles) { return d * tiles >= 512 ? 1 : d > 128 ? 1 : 2; }

// Codes of a step of 32 tokens on their way from memory, in memory's order: piece x of 16 bytes of a tile
// of 16 tokens is lane x % 64's, register x / 64. (Loaded as the products want them, a token's pieces
// 16 lanes apart, each lane's piece was a look-up of the cache of its own: three times as many, which took
// longer than the arithmetic.)
template <int D>
struct Raw {
  u32x4 k[2][D / 64], v[2][D / 64];
};

// Where chunk c of 16 bytes of a token's codes lies in the LDS: moved within its rows so that the lanes
// of a load, the same chunk of many tokens, take all banks.
template <int D>
__device__ __forceinline__ int code_place(int tok, int c) {
  return tok * D + ((c ^ (D == 64 ? (tok >> 1) & 3 : tok & 7)) << 4);
}

// Eight codes of the LDS at `p`, transposed with those of the other lanes of a row of 16: lane 2 i
// and 2 i + 1 name the first and the second eight of sixteen codes of token i, lane n gets code n of
// the eight tokens.
typedef int i32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32x2 transposed(const uint8_t* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                                       (__attribute__((address_space(3))) i32x2*)p));
}

// Two codes (the low or the high half of a word) as a bf16 pair, times the power of two in the exponent
// field of `pow`.
template <bool HI>
__device__ __forceinline__ uint32_t codes_times(uint32_t w, float pow) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, pow, HI));
}

// The greater of two values, NaN where one is (fmaxf would first make every operand canonical).
__device__ __forceinline__ float greater(float x, float y) { return __builtin_elementwise_maximum(x, y); }
template <int BY>
__device__ __forceinline__ float lane_greater(float x) {
  float a, b;
  lane_pair<BY>(x, a, b);
  return greater(a, b);
}

// split_terms<2>, the rests x - x0 as dot products (exact: one factor is 1, the other 0), so that the
// first terms are not taken apart again.
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void split_two(const float (&x)[8], bf16x8 (&out)[2]) {
  // ((-1, 0) and (0, -1), out of the compiler's sight: the first as a constant of the instruction is
  // taken for an fp32 -1, which is the second)
  uint32_t one = 0x0000BF80u, two = 0xBF800000u;
  asm("" : "+s"(one), "+s"(two));
  const bf16x2 first = __builtin_bit_cast(bf16x2, one), second = __builtin_bit_cast(bf16x2, two);
  u32x4 hi, lo;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    hi[k] = pair_bf16(x[2 * k], x[2 * k + 1]);
    const bf16x2 both = __builtin_bit_cast(bf16x2, (uint32_t)hi[k]);
    lo[k] = pair_bf16(__builtin_amdgcn_fdot2_f32_bf16(both, first, x[2 * k], false),
                      __builtin_amdgcn_fdot2_f32_bf16(both, second, x[2 * k + 1], false));
  }
  out[0] = __builtin_bit_cast(bf16x8, hi);
  out[1] = __builtin_bit_cast(bf16x8, lo);
}

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
    struct {
      bf16x8 q[kShared ? R * (D / 32) * TERMS * 64 : 1];       // [tile][chunk][term][lane]
      uint8_t codes[kTreeWaves][kStep * D];                    // of K, then of V: each wave its own
    };
    float acc[kTreeWaves][16 * kTogether][D + 4];              // the waves' results
  };
  float m[kTreeWaves][16 * R], l[kTreeWaves][16 * R];
  uint32_t spoilt[kTreeWaves][16 * R];                         // rows that see a scale that is not finite: 1 V's, 2 K's
  int pos[CM_QCACHE_MAX_REQUESTS + 1];                         // where the requests begin, in units
  float cost[kTreeWaves];
  int sums[kTreeWaves], tiles[kTreeWaves];
  int first;
};

// Partial results of a range of a cut tile: quads of columns, row after row, then the exponent and the
// sum of each row. The join is a launch of its own, so they are stored and loaded like any other data.
template <int D, int R>
struct TreePart {
  static constexpr int64_t kFloats = (int64_t)16 * R * (D + 2);
  float* at;
  __device__ __forceinline__ f32x4* quad(int x) const { return reinterpret_cast<f32x4*>(at) + x; }
  __device__ __forceinline__ f32x2v* stat(int row) const {
    return reinterpret_cast<f32x2v*>(at + 16 * R * D) + row;
  }
};
template <int D, int R>
__device__ __forceinline__ TreePart<D, R> tree_part(const TreeAttention& a, int h, int place) {
  return {a.a.few_part + ((int64_t)h * a.a.few_max + place) * TreePart<D, R>::kFloats};
}
// Where the partial results of a tile's range i are. A span has two places: for a range at its beginning,
// and for one that begins in it and goes on behind it, as the first range of a tile may.
__device__ __forceinline__ int tree_slot(int first, int mid, int i) {
  return i == 0 ? 2 * first + mid : 2 * (first + i);
}
// What the join has to know of the range in a place.
struct TreeCut {
  int32_t splits;              // ranges of its tile; 0: nothing is there
  int32_t part;                // its number among them
  int32_t first, mid;          // the span of the first of them, and its place there
  int32_t row0, rho0, live;    // the request's first row; the tile's first of its rows times the group, and how many
};

__device__ __forceinline__ RowPlace tree_place(const TreeAttention& a, int row0, int h, int rho) {
  return {row0 + rho / a.a.G, h * a.a.G + rho % a.a.G};
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
  constexpr int kAhead = tree_ahead(TERMS, D, R);
  constexpr bool kShared = tree_query_shared(TERMS, D, R);
  const QAttention& a = ta.a;
  // (the wave's number in a scalar register: its steps are the same for all lanes then, and no wait
  // for loads counts on a path on which some lanes skip a step)
  const int lane = anew(threadIdx.x & 63), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
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

  f32x4 acc[R][DW];                              // acc[.][c][i]: column 16 c + 4 g + i of row n
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
  // a lane's pieces in the LDS: as they come from memory, and as the products want them
  uint8_t* staged = lds.codes[wave];
  constexpr int kPieces = D / 16;                // of a token
  const uint32_t put = code_place<D>(lane / kPieces, lane % kPieces), lane_at = lane * 16;
  if (lane < 16 * R) lds.spoilt[wave][lane] = 0;
  // 64 tiles of 16 tokens at a time: their pages and scales, one lane each
  for (int t0 = begin; t0 < end; t0 += 64 * 16) {
    int32_t my_page = 0;
    // (not 0, also where the softmax scale is: hidden scores are -inf times it)
    float my_ks = 0x1p-126f, my_vs = 1.f;
    const int my_t = t0 + lane * 16;
    bool there = false, k_odd = false, v_odd = false;
    if (my_t < end) {
      my_page = table[my_t >> a.b_shift];
      there = my_page >= 0 && my_page < a.pages;
      if (!there) my_page = 0;
      const float ks = a.ks[(int64_t)my_page * a.H + h] * a.scale_log2;
      const float vs = a.vs[(int64_t)my_page * a.H + h];
      k_odd = there && !(ks < __builtin_inff());
      v_odd = there && !(vs < __builtin_inff());
      if (ks < __builtin_inff()) my_ks = fmaxf(ks, 0x1p-126f);
      if (there && vs < __builtin_inff()) my_vs = vs;
    }
    // (the products, which all rows share, take other scales in their place)
    if (__builtin_expect(__any(k_odd || v_odd), 0)) {
      const uint64_t k_tiles = __ballot(k_odd), v_tiles = __ballot(v_odd);
      for (uint64_t tiles = k_tiles | v_tiles; tiles; tiles &= tiles - 1) {
        const int tile = __builtin_ctzll(tiles), row = lane_anew();
        if (row < 16 * R && (tree_sees(ta, it, (rho0 + row) / a.G, t0 + tile * 16) & 0xFFFFu))
          lds.spoilt[wave][row] |= ((v_tiles >> tile) & 1) | ((k_tiles >> tile) & 1) << 1;
      }
    }
    // V's scale as a power of two, which the conversion of its codes takes, times a rest in [1, 2),
    // which the weights' exponent takes; their sum is divided by it. (An exponent field of 0 stands for
    // 2^-127 in the conversion; a scale of 0 is that. Beyond 2^119 the greatest codes would be infinite,
    // and NaN times the weight 0 of a row that does not see them: the rest takes what is above it.)
    const uint32_t vs_field = __float_as_uint(my_vs) & 0x7F800000u;
    const uint32_t vs_exponent = vs_field < 0x7B000000u ? vs_field : 0x7B000000u;
    const float my_vp = __uint_as_float(vs_exponent);
    const float rest = vs_field > vs_exponent ? my_vs * 0x1p-119f
                       : vs_exponent ? __uint_as_float((__float_as_uint(my_vs) & 0x7FFFFFu) | 0x3F800000u)
                       : my_vs == 0.f ? 1.f : fabsf(my_vs) * 0x1p127f;
    const float my_vl = __builtin_amdgcn_logf(rest), my_vi = 1.f / rest;
    const uint64_t absent = ~__ballot(there);
    const int steps = ((end < t0 + 1024 ? end : t0 + 1024) - t0 + kStep - 1) / kStep;
    Raw<D> ring[kAhead];
    const auto base_of = [&](int tile) {
      const int64_t page = __builtin_amdgcn_readlane(my_page, tile);
      return page * page_codes + head_codes + (int64_t)((t0 + tile * 16) & (B - 1)) * D;
    };
    const auto load = [&](int s, const uint8_t* codes, u32x4 (&x)[2][D / 64]) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint8_t* p = codes + base_of(2 * s + b);
#pragma unroll
        for (int c = 0; c < D / 64; ++c) x[b][c] = *global_ptr<u32x4>(p + (lane_at + c * 1024));
      }
    };
    // K of the kAhead-th next step is on its way from the scores on, V from the products on
    const auto step = [&](int s, Raw<D>& raw) {
      const int t = t0 + s * kStep;
      const int next = s + kAhead < steps ? s + kAhead : steps - 1;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int c = 0; c < D / 64; ++c)         // (1024 bytes on: 1024 / D tokens, 4 where D is 256)
          *reinterpret_cast<u32x4*>(staged + (D > 128 ? put ^ ((c & 1) << 6) : put) +
                                    (b * 16 * D + c * 1024)) = raw.k[b][c];
      load(next, a.kc, raw.k);
      f32x4 sc[R][2];
#pragma unroll
      for (int j = 0; j < R; ++j) sc[j][0] = sc[j][1] = f32x4{0.f, 0.f, 0.f, 0.f};
      const int q_lane = kShared ? anew(lane) : lane;
      const int kn = anew(n), kg = anew(g);
      u32x4 chunk[2];
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int c = 0; c < D / 64; ++c)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          bf16x8 k[2];
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            if (half == 0) chunk[b] = *reinterpret_cast<const u32x4*>(staged + code_place<D>(b * 16 + kn, 4 * c + kg));
            k[b] = operand(chunk[b][2 * half], chunk[b][2 * half + 1]);
          }
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
      __builtin_amdgcn_s_setprio(0);
      const auto of_tile = [&](float x, int b) {
        return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 2 * s + b));
      };
      // V's codes follow K's in the same place
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
          *reinterpret_cast<u32x4*>(staged + (D > 128 ? put ^ ((c & 1) << 6) : put) +
                                    (b * 16 * D + c * 1024)) = raw.v[b][c];
      load(next, a.vc, raw.v);
      // steps that some row sees only in part, or with absent pages
      const bool partly = t < all_lo || t + kStep > all_hi || ((absent >> (2 * s)) & 3) != 0;
      uint32_t seen = 0;                         // bit 8 j + 4 b + i: the lane's tokens, row tile j
      if (__builtin_expect(partly, 0)) {
        uint32_t there2 = (absent >> (2 * s)) & 1 ? 0u : 0xFFFFu;
        there2 |= (absent >> (2 * s + 1)) & 1 ? 0u : 0xFFFF0000u;
#pragma unroll
        for (int j = 0; j < R; ++j) {
          const int ln = lane_anew();            // (or what is made of it would be kept through the steps)
          const uint32_t y = tree_sees(ta, it, (rho0 + 16 * j + (ln & 15)) / a.G, t) & there2;
          const int lg = ln >> 4;
          const uint32_t mine = ((y >> (4 * lg)) & 0xFu) | ((y >> (16 + 4 * lg)) & 0xFu) << 4;
#pragma unroll
          for (int k = 0; k < 8; ++k)
            sc[j][k >> 2][k & 3] = (mine >> k) & 1 ? sc[j][k >> 2][k & 3] : kNone;
          seen |= mine << (8 * j);
        }
        // NaN codes are taken out of the product (0 * NaN would reach rows that do not see them); a
        // product of their own finds the rows that do
        uint32_t odd = 0;
#pragma unroll
        for (int x = 0; x < D / 32; ++x) {
          const u32x4 w = reinterpret_cast<const u32x4*>(staged)[64 * x + lane_anew()];
          odd |= nan_codes(w[0]) | nan_codes(w[1]) | nan_codes(w[2]) | nan_codes(w[3]);
        }
        if (__any(odd != 0)) {
          const int ln = lane_anew(), lc = ln & 15;
          const uint32_t token = 4 * (ln >> 4) + ((lc >> 1) & 3) + 16 * (lc >> 3);
#pragma unroll
          for (int c = 0; c < DW; ++c) {
            const u32x2 w = transposed(staged + code_place<D>(token, c) + 8 * (lc & 1));
            u32x4 is;                            // 1 where the code is NaN
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t y = nan_codes(w[k >> 1]) >> (16 * (k & 1));
              is[k] = (y & 1) * 0x3F80u | ((y >> 8) & 1) * 0x3F800000u;
            }
#pragma unroll
            for (int j = 0; j < R; ++j) {
              u32x4 by;                          // 1 where the lane's row sees the token
#pragma unroll
              for (int k = 0; k < 4; ++k)
                by[k] = ((seen >> (8 * j + 2 * k)) & 1) * 0x3F80u |
                        ((seen >> (8 * j + 2 * k + 1)) & 1) * 0x3F800000u;
              f32x4 hits = {0.f, 0.f, 0.f, 0.f};
              hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, is),
                                                             __builtin_bit_cast(bf16x8, by), hits, 0, 0, 0);
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (hits[i] > 0.f) acc[j][c][i] = __builtin_nanf("");
            }
          }
#pragma unroll
          for (int x = 0; x < D / 32; ++x) {
            u32x4* at = reinterpret_cast<u32x4*>(staged) + (64 * x + lane_anew());
            u32x4 w = *at;
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] &= ~(nan_codes(w[k]) * 0xFFu);
            *at = w;
          }
        }
      }
      // (each lane looks at its own tokens: that one of them has a new maximum is rare)
      float top[R];
      bool more = false;
#pragma unroll
      for (int j = 0; j < R; ++j) {
        float best[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          best[b] = sc[j][b][0];
#pragma unroll
          for (int i = 1; i < 4; ++i) best[b] = greater(best[b], sc[j][b][i]);
        }
        top[j] = greater(best[0] * of_tile(my_ks, 0), best[1] * of_tile(my_ks, 1));
        more |= top[j] > ref[j] + 8.f;
      }
      if (__any(more)) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
          if (!__any(top[j] > ref[j] + 8.f)) continue;
          // (a NaN among them: the row is NaN in any case)
          const float m = fmaxf(ref[j], lane_greater<32>(lane_greater<16>(top[j])));
          const float shrink = m == kNone ? 1.f : __builtin_amdgcn_exp2f(ref[j] - m);
          l[j] *= shrink;
#pragma unroll
          for (int c = 0; c < DW; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[j][c][i] *= shrink;
          ref[j] = m;
        }
      }
      // out^T += V^T P^T, 16 columns at a time: lane n of the operand is column n, its eight tokens
      // 4 g .. 4 g + 3 of both tiles. The products of the first columns with a row tile's weights run
      // beside the making of the next tile's.
      const uint32_t token = 4 * kg + ((kn >> 1) & 3) + 16 * (kn >> 3);
      constexpr int kFirst = R == 1 ? DW : DW / 2;
      bf16x8 pt[R][PT], vt[DW];
      const auto column = [&](int c) {
        const u32x2 w = transposed(staged + code_place<D>(token, c) + 8 * (kn & 1));
        u32x4 x;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const float pow = of_tile(my_vp, b);
          x[2 * b] = codes_times<false>(w[b], pow);
          x[2 * b + 1] = codes_times<true>(w[b], pow);
        }
        vt[c] = __builtin_bit_cast(bf16x8, x);
      };
      const auto product = [&](int j, int c, int z) {
        acc[j][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt[c], pt[j][z], acc[j][c], 0, 0, 0);
      };
#pragma unroll
      for (int c = 0; c < kFirst; ++c) column(c);
#pragma unroll
      for (int j = 0; j < R; ++j) {
        const float low = ref[j] == kNone ? 0.f : ref[j];
        float pv[8];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const float off = of_tile(my_vl, b) - low, kf = of_tile(my_ks, b);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            pv[4 * b + i] = __builtin_amdgcn_exp2f(fmaf(sc[j][b][i], kf, off));
          l[j] = fmaf((pv[4 * b] + pv[4 * b + 1]) + (pv[4 * b + 2] + pv[4 * b + 3]), of_tile(my_vi, b), l[j]);
        }
        if constexpr (PT == 2) split_two(pv, pt[j]);
        else split_terms<PT>(pv, pt[j]);
        if (j > 0) {
#pragma unroll
          for (int z = PT - 1; z >= 0; --z)
#pragma unroll
            for (int c = 0; c < kFirst; ++c) product(j - 1, c, z);
#pragma unroll
          for (int x = 0; x < PT * kFirst; ++x) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 7, 0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int z = PT - 1; z >= 0; --z)
#pragma unroll
        for (int c = 0; c < kFirst; ++c) product(R - 1, c, z);
#pragma unroll
      for (int c = kFirst; c < DW; ++c) {
        column(c);
#pragma unroll
        for (int z = PT - 1; z >= 0; --z)
#pragma unroll
          for (int j = 0; j < R; ++j) product(j, c, z);
      }
    };
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
    {
      // (in the order of the steps: a wait for the first of them is then not one for all)
      load(y < steps ? y : steps - 1, a.kc, ring[y].k);
      __builtin_amdgcn_sched_barrier(0);
      load(y < steps ? y : steps - 1, a.vc, ring[y].v);
      __builtin_amdgcn_sched_barrier(0);
    }
    // (out of the loop at once where they end: a path around a step would have every wait for
    // loads count on those that it did not issue)
    for (int s = 0;;) {
      bool over = false;
#pragma unroll
      for (int y = 0; y < kAhead; ++y) {
        if (over) break;
        step(s, ring[y]);
        over = ++s >= steps;
      }
      if (over) break;
    }
  }

  // the waves' results as one, by all threads, kTogether row tiles at a time
  constexpr int kTogether = TreeShared<TERMS, D, R>::kTogether;
  const int en = anew(n), eg = anew(g);
  uint32_t spoilt[R];
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const float sum = lane_sum<32>(lane_sum<16>(l[j]));
    spoilt[j] = lds.spoilt[wave][16 * j + en];
    if (eg == 0) {
      lds.m[wave][16 * j + en] = ref[j];
      lds.l[wave][16 * j + en] = spoilt[j] & 2 ? __builtin_nanf("") : sum;
    }
  }
  const int live = it.count * a.G - rho0;        // rows of the tile that there are
  const TreePart<D, R> part = tree_part<D, R>(ta, h, slot);
#pragma unroll
  for (int j0 = 0; j0 < R; j0 += kTogether) {
    __syncthreads();                             // (also: the queries in the LDS are not needed now)
#pragma unroll
    for (int jj = 0; jj < kTogether; ++jj) {
      float* row = &lds.acc[wave][16 * jj + en][4 * eg];
#pragma unroll
      for (int c = 0; c < DW; ++c) *reinterpret_cast<f32x4*>(&row[16 * c]) = acc[j0 + jj][c];
      if (__builtin_expect(spoilt[j0 + jj] != 0, 0))
#pragma unroll
        for (int c = 0; c < DW; ++c) *reinterpret_cast<f32x4*>(&row[16 * c]) = f32x4{} + __builtin_nanf("");
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
        const RowPlace place = tree_place(ta, it.row0, h, rho0 + row);
        put_quad<ES>(a, place, 4 * quad, o, sum);
        if (quad == 0) put_lse(a, place, low, sum);
      } else {
        *part.quad(row * kQuads + quad) = o;
        if (quad == 0) *part.stat(row) = f32x2v{m, sum};
      }
    }
  }
  __syncthreads();                               // (the LDS is the next range's)
}

// The ranges of a workgroup's span, one after another.
template <int TERMS, int D, int R>
__global__ __launch_bounds__(kTreeThreads, kTreeGroups) void qcache_tree_kernel(TreeAttention ta) {
  __shared__ TreeShared<TERMS, D, R> lds;
  constexpr int ES = TERMS == 1 ? 2 : 4;
  constexpr int kPer = CM_QCACHE_MAX_REQUESTS / kTreeThreads;
  const QAttention& a = ta.a;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const HeadItem hi = head_item(a.H, blockIdx.x);
  const int h = hi.h, w = hi.item;
  if (w >= a.few_items) return;
  // (the heads' spans are the same)
  TreeCut* cuts = static_cast<TreeCut*>(a.many_found) + 2 * w;
  const bool tells = h == 0 && threadIdx.x == 0;
  if (tells) cuts[0].splits = cuts[1].splits = 0;

  // where every request begins: prefix sums of the units of all its tiles
  const int per = (a.n + kTreeThreads - 1) / kTreeThreads;
  int units[kPer], tiles[kPer], mine = 0, my_tiles = 0;
  float cost = 0.f;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int r = (int)threadIdx.x * per + k;
    units[k] = tiles[k] = 0;
    if (k < per && r < a.n) {
      TreeItem it;
      tree_request(ta, r, it);
      tiles[k] = (it.count * a.G + 16 * R - 1) / (16 * R);
      if (tiles[k]) {
        units[k] = tree_units(ta, it);
        cost += (float)tiles[k] * (float)units[k];
      }
    }
    mine += tiles[k] * units[k];
    my_tiles += tiles[k];
  }
  const auto prefix = [&](int x) {
    const int upto = wave_scan(x);
    if (lane == 63) lds.sums[wave] = upto;
    __syncthreads();
    int before = upto - x;
#pragma unroll
    for (int v = 0; v < kTreeWaves; ++v)
      if (v < wave) before += lds.sums[v];
    return before;
  };
  my_tiles = wave_scan(my_tiles);
  cost = wave_scan(cost);
  if (lane == 63) {
    lds.tiles[wave] = my_tiles;
    lds.cost[wave] = cost;
  }
  int at = prefix(mine), total = 0, all_tiles = 0;
  cost = 0.f;
#pragma unroll
  for (int v = 0; v < kTreeWaves; ++v) {
    total += lds.sums[v];
    all_tiles += lds.tiles[v];
    cost += lds.cost[v];
  }
  // (rows that lie over one another: more units than an int holds, which nobody takes)
  if (cost > 2e9f) return;
  total = __builtin_amdgcn_readfirstlane(total);
  all_tiles = __builtin_amdgcn_readfirstlane(all_tiles);
  int span = (total + a.few_items - 1) / a.few_items;
  // Spans that begin with every tile, so that none has two ranges, whose queries, pages and sums take
  // about as long as two units: the least span s for which total + tiles (s - 1) units are no more than
  // the spans hold. (24 fp32 trees of up to 23 nodes, a window of 1000: 28.6 -> 22.2 us a call.)
  bool whole = false;
  if (all_tiles < a.few_items) {
    const int apart = (total - all_tiles + a.few_items - all_tiles - 1) / (a.few_items - all_tiles);
    whole = apart <= span + kTreeRange;
    span = whole ? apart : span;
  }
  span = span < ta.least ? ta.least : span;
  if (whole) {
    mine = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      units[k] = (units[k] + span - 1) / span * span;
      mine += tiles[k] * units[k];
    }
    __syncthreads();
    at = prefix(mine);
    total = 0;
#pragma unroll
    for (int v = 0; v < kTreeWaves; ++v) total += lds.sums[v];
    total = __builtin_amdgcn_readfirstlane(total);
  }
  int u = w * span;
  const int stop = u + span < total ? u + span : total;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int r = (int)threadIdx.x * per + k;
    if (k < per && r < a.n) {
      lds.pos[r] = at;
      if (u >= at && u < at + tiles[k] * units[k]) lds.first = r;
    }
    at += tiles[k] * units[k];
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
    const int each = tree_units(ta, it), room = whole ? (each + span - 1) / span * span : each;
    it.tile = (u - from) / room;
    const int tile_from = from + it.tile * room, tile_to = tile_from + each;
    const int u0 = u;
    u = tile_to < stop ? tile_to : stop;
    const int begin = tree_begin(ta, it);
    it.begin = begin + (u0 - tile_from) * a.few_unit;
    const int64_t end = begin + (int64_t)(u - tile_from) * a.few_unit;
    it.end = end < it.len ? (int)end : it.len;
    const int first = tile_from / span, part = w - first;
    it.splits = (tile_to - 1) / span - first + 1;
    const int mid = part == 0 && tile_from > first * span ? 1 : 0;
    if (it.splits > 1 && tells) {
      const int rho0 = it.tile * 16 * R, live = it.count * a.G - rho0;
      cuts[mid] = TreeCut{it.splits, part, first, tile_from > first * span ? 1 : 0, it.row0, rho0,
                          live < 16 * R ? live : 16 * R};
    }
    tree_segment<TERMS, D, R>(ta, it, h, 2 * w + mid, lds);
    if (whole) break;
    if (u == to) ++r;
  }
}

// Joins the partial results of the tiles that are cut: the workgroup of each range takes an equal part of
// its tile's quads of columns, over the results of all its ranges; threads that share a quad take every
// kth result, in an order that depends on their number alone. (Joined by the last workgroups of the launch
// before to come, with stores and loads past the caches of the XCDs, 64 rows over 264 thousand tokens
// took 50 us longer than their arithmetic; so 12.)
constexpr int kTreeJoin = 256;
template <int D, int R, int ES>
__global__ __launch_bounds__(kTreeJoin) void qcache_tree_join_kernel(TreeAttention ta) {
  constexpr int kQuads = D / 4, kBatch = 8;
  __shared__ f32x4 s_o[kTreeJoin];
  __shared__ float s_m[kTreeJoin], s_l[kTreeJoin];
  const QAttention& a = ta.a;
  const HeadItem hi = head_item(a.H, blockIdx.x);
  const int h = hi.h, w = hi.item, tid = threadIdx.x;
  if (w >= a.few_items) return;
  for (int mid = 0; mid < 2; ++mid) {
    const TreeCut cut = static_cast<const TreeCut*>(a.many_found)[2 * w + mid];
    if (cut.splits == 0) continue;
    const int total = cut.live * kQuads, share = (total + cut.splits - 1) / cut.splits;
    const int begin = cut.part * share, end = begin + share < total ? begin + share : total;
    // the quads of a pass, a power of two, and the threads that share one
    int width = 1;
    while (width < end - begin && width < kTreeJoin) width *= 2;
    const int sharers = kTreeJoin / width, q = tid & (width - 1), p = tid / width;
    for (int x0 = begin; x0 < end; x0 += width) {
      const int x = x0 + q < end ? x0 + q : end - 1, row = x / kQuads;
      Joined sum;
      for (int s = p; s < cut.splits; s += sharers * kBatch) {
        f32x4 o[kBatch];
        float m[kBatch], l[kBatch];
        int there = 0;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          const int i = s + k * sharers < cut.splits ? s + k * sharers : s;
          there += s + k * sharers < cut.splits;
          const TreePart<D, R> part = tree_part<D, R>(ta, h, tree_slot(cut.first, cut.mid, i));
          o[k] = *part.quad(x);
          const f32x2v st = *part.stat(row);
          m[k] = st[0];
          l[k] = st[1];
        }
        sum.add(o, m, l, there);
      }
      if (sharers > 1) {
        s_o[tid] = sum.o;
        s_m[tid] = sum.m;
        s_l[tid] = sum.l;
        __syncthreads();
        for (int half = sharers / 2; half > 0; half >>= 1) {
          if (p < half) {
            f32x4 o[1] = {s_o[tid + half * width]};
            float m[1] = {s_m[tid + half * width]}, l[1] = {s_l[tid + half * width]};
            sum.add(o, m, l, 1);
            s_o[tid] = sum.o;
            s_m[tid] = sum.m;
            s_l[tid] = sum.l;
          }
          __syncthreads();
        }
      }
      if (p == 0 && x0 + q < end) {
        const RowPlace place = tree_place(ta, cut.row0, h, cut.rho0 + row);
        put_quad<ES>(a, place, 4 * (x % kQuads), sum.o, sum.l);
        if (x % kQuads == 0) put_lse(a, place, sum.m == kNone ? 0.f : sum.m, sum.l);
      }
    }
  }
}

template <int TERMS, int D, int R>
hipError_t launch_tree_tiles(const TreeAttention& a, hipStream_t stream) {
  const dim3 groups((uint32_t)head_groups(a.a.H, a.a.few_items));
  hipLaunchKernelGGL((qcache_tree_kernel<TERMS, D, R>), groups, dim3(kTreeThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.a.few_items == 1) return e;  // (one span for each head: nothing is cut)
  hipLaunchKernelGGL((qcache_tree_join_kernel<D, R, TERMS == 1 ? 2 : 4>), groups, dim3(kTreeJoin), 0, stream, a);
  return hipGetLastError();
}
template <int TERMS>
hipError_t launch_tree(const TreeAttention& a, int32_t d, int32_t tiles, hipStream_t stream) {
  if (d == 64) {
    if constexpr (TERMS == 1)
      if (tiles == 4) return launch_tree_tiles<TERMS, 64, 4>(a, stream);
    return tiles == 1 ? launch_tree_tiles<TERMS, 64, 1>(a, stream) : launch_tree_tiles<TERMS, 64, 2>(a, stream);
  }
  if (d == 128) {
    if constexpr (TERMS == 1)
      if (tiles == 4) return launch_tree_tiles<TERMS, 128, 4>(a, stream);
    return tiles == 1 ? launch_tree_tiles<TERMS, 128, 1>(a, stream) : launch_tree_tiles<TERMS, 128, 2>(a, stream);
  }
  if constexpr (TERMS == 1)
    if (tiles == 2) return launch_tree_tiles<TERMS, 256, 2>(a, stream);
  return launch_tree_tiles<TERMS, 256, 1>(a, stream);
}
// (a file for each type of the queries: they are built side by side)
hipError_t launch_tree_bf16(const TreeAttention& a, int32_t d, int32_t tiles, hipStream_t stream);
hipError_t launch_tree_fp32(const TreeAttention& a, int32_t d, int32_t tiles, hipStream_t stream);

}  // namespace cm
