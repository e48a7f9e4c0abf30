// Attention over the 8-bit paged cache for requests with many query rows: prompts and
// questions of more rows than one 16-row tile holds.
//
// The same one-pass softmax as for few rows (qcache_few.h), with the work
// the other way round: a workgroup takes 128 query rows (a request's rows times the
// group) of one KV head, each of its four waves 32 of them, and walks the context in
// tiles of TOK tokens. A tile's codes are turned into bf16 once for all 128 rows, by 2^e of
// their page's scale on the way (the conversion takes the power of two at no cost; what is left
// of a scale that is none goes into the exponents), and staged in the LDS: K row-major, V transposed. Both products are
// computed transposed by 32x32x16 matrix instructions, S^T = K Q^T and out^T = V^T P^T, so that a
// lane holds of S^T exactly the probabilities that it has to supply of P^T; V's columns
// are laid out in that order of the tokens: element e of 16-byte chunk 2 s + k of a row is
// token 16 s + 8 (e / 4) + 4 k + e % 4. Chunks are moved within their rows by an exclusive
// or with the row's number so that the lanes of a load take all banks.
//
// Weights enter the second product as two bf16 terms (16 bits) for bf16 queries, three (24 bits) for
// fp32 ones, as in the kernel for few rows. One term would cost as much error as the
// rounding of the output does, whatever the size of the single weights, since outputs become
// smaller as their errors do: 300 queries of nearly equal weights over 4000 tokens were
// off by 1.49 times the output's own rounding, and 4096 queries over 16384 tokens took 1.33 ms
// so, 1.66 ms with two.
//
// Bound by the vector and the matrix units: for 32 rows and 64 tokens of d = 128 a wave issues 48
// products of 32 cycles and about 325 vector instructions, 33 of them exponentials. 4096
// queries over 16384 tokens, 8 heads of d = 128, G 4: 1.66 to 1.77 ms, 0.70 to 0.74 PFLOP/s, the vector
// units busy 59% of the time and the matrix units 55%.
#include <type_traits>

#include "qcache_few.h"

namespace cm {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWaveRows = 32;
constexpr int kRowWaves = kManyRows / kWaveRows;

// Codes to bf16, times the power of two in the exponent field of `pow`.
template <bool HI>
__device__ __forceinline__ uint32_t scaled_bf16(uint32_t w, float pow) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, pow, HI));
}

// Bytes of the K and V tiles, and a chunk's place in them. The rows' numbers are combined with
// the chunks' by exclusive or, so the places of a lane's chunks are its first one's with
// some bits of their numbers turned.
template <int D, int TOK>
struct Tile {
  static constexpr int kBytes = D * TOK * 2;
  // K: row = token, D / 8 chunks
  static __device__ __forceinline__ uint32_t k_at(int tok, int chunk) {
    const int x = D == 64 ? (tok >> 1) & 7 : tok & 15;
    return tok * D * 2 + ((chunk ^ x) << 4);
  }
  // V: row = column of V, TOK / 8 chunks
  static __device__ __forceinline__ uint32_t v_at(int col, int chunk) {
    const int x = TOK == 32 ? (col >> 2) & 3 : ((col >> 1) & 7) ^ ((col >> 4) & 1);
    return col * TOK * 2 + ((chunk ^ x) << 4);
  }
};

// Codes of a tile on their way from memory to the LDS: a wave stages 16 tokens of
// COLS columns.
template <int COLS>
struct Codes {
  u32x4 k[COLS / 64];
  uint32_t v[COLS / 16];
};

// 16-column chunks of its queries that a wave keeps in the LDS: where two waves share a SIMD's
// registers three terms of 128 columns leave none for the last two.
constexpr int shared_chunks(int terms, int columns, int halves) {
  return halves == 2 && terms * columns > 256 ? 2 : 0;
}

// The LDS of a workgroup.
template <int TERMS, int D, int TOK, int HALVES>
struct ManyShared {
  uint8_t k[2][D * TOK * 2];
  uint8_t v[2][D * TOK * 2];
  // halves of scores that waves exchange
  f32x4 half[HALVES == 2 ? kRowWaves * HALVES * (TOK / 32) * 4 * 64 : 1];
  static constexpr int kQuery = shared_chunks(TERMS, D / HALVES, HALVES) * TERMS;
  bf16x8 q[kQuery ? kRowWaves * HALVES * kQuery * 64 : 1];  // [wave][chunk][term][lane]
  FindShared find;
};

// Partial results of an item: quads of columns, each of the tile's rows one after another, then
// the exponent m and the sum l of each row. The join is a launch of its own, so they are stored
// and loaded like any other data.
template <int D>
struct ManyPart {
  static constexpr int64_t kFloats = (int64_t)kManyRows * (D + 4);
  float* at;
  int rows;
  __device__ __forceinline__ f32x4* quad(int row, int q) const {
    return reinterpret_cast<f32x4*>(at) + q * rows + row;
  }
  __device__ __forceinline__ f32x2v* stat(int row) const {
    return reinterpret_cast<f32x2v*>(at + kManyRows * D) + row;
  }
};
template <int D>
__device__ __forceinline__ ManyPart<D> many_part(const QAttention& a, const Item& it, int h,
                                                 int place) {
  const int rows = it.count * a.G - it.tile * kManyRows;
  return {a.many_part + ((int64_t)h * a.many_places + place) * ManyPart<D>::kFloats,
          rows < kManyRows ? rows : kManyRows};
}

// HALVES 2: two waves share 32 rows, each half of d: half of the sum of a score, which
// they exchange through the LDS, and half of the output's columns.
template <int TERMS, int D, int TOK, int HALVES>
__device__ __forceinline__ void many_rows_item(const QAttention& a, int block,
                                               ManyShared<TERMS, D, TOK, HALVES>& lds) {
  using T = Tile<D, TOK>;
  constexpr int kWaves = kRowWaves * HALVES;
  constexpr int DH = D / HALVES;                 // columns of a wave
  constexpr int ES = TERMS == 1 ? 2 : 4;
  constexpr int PT = TERMS == 1 ? 2 : 3;         // terms of a probability
  constexpr int kGroups = TOK / 16;              // 16-token groups of a tile
  constexpr int COLS = D * kGroups / kWaves;     // columns that a wave stages of its group
  constexpr int kTok32 = TOK / 32;
  constexpr int kPerLook = 64 / kGroups;         // tiles of a look-up
  static_assert(COLS == 64 || COLS == 128, "");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = lane & 31, g = lane >> 5;
  const int row_wave = wave % kRowWaves, half = wave / kRowWaves;
  const HeadItem hi = head_item(a.H, block);
  const int h = hi.h, item = hi.item;
  const Item it = find_item<kManyRows, 64 * kWaves>(a, a.many_items, a.many_max, item, lds.find);
  // (where its partial results go, for the join; a place that nobody has is marked so)
  if (h == 0 && threadIdx.x == 0) {
    Item* found = reinterpret_cast<Item*>(a.many_found);
    if (it.any && it.splits > 1) found[it.place] = it;
    if (item >= it.places && item < a.many_places) found[item].any = 0;
  }
  if (!it.any) return;

  // the lane's query row
  const int rho = it.tile * kManyRows + row_wave * kWaveRows + n;
  const int tok = rho / a.G;
  const bool live = tok < it.count;
  const int head = h * a.G + rho % a.G;
  const int p = it.len - it.count + tok;
  const int see_hi = live && p >= 0 ? p + 1 : 0;
  // (from see_hi where it is asked for: one register less through the tiles)
  const auto see_from = [&] { return a.window && see_hi > a.window ? see_hi - a.window : 0; };
  const Sight sight = tile_sight<kManyRows>(a, it);
  const bool wave_live = it.tile * kManyRows + row_wave * kWaveRows < it.count * a.G;

  int begin = it.begin + it.split * it.chunk, end = begin + it.chunk;
  const int from = sight.any_lo & ~(TOK - 1);
  begin = begin > from ? begin : from;
  end = end < sight.any_hi ? end : sight.any_hi;
  const int tiles = end > begin ? (end - begin + TOK - 1) / TOK : 0;

  constexpr int kKept = DH / 16 - shared_chunks(TERMS, DH, HALVES);
  bf16x8 q[kKept][TERMS];
#pragma unroll
  for (int c = 0; c < kKept; ++c)
    load_query<TERMS>(a, it.row0 + tok, head, half * DH + c * 16 + g * 8, live, q[c]);
  const uint32_t q_place = wave * lds.kQuery * 64 + lane;
#pragma unroll
  for (int c = kKept; c < DH / 16; ++c) {
    bf16x8 x[TERMS];
    load_query<TERMS>(a, it.row0 + tok, head, half * DH + c * 16 + g * 8, live, x);
#pragma unroll
    for (int w = 0; w < TERMS; ++w) lds.q[q_place + ((c - kKept) * TERMS + w) * 64] = x[w];
  }

  f32x16 acc[DH / 32];
#pragma unroll
  for (int j = 0; j < DH / 32; ++j)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[j][i] = 0.f;
  float ref = kNone, top = kNone, l = 0.f;       // exponent that acc and l are relative to; maximum

  const int32_t* table = a.table + (int64_t)it.r * a.width;
  const int B = 1 << a.b_shift;
  const int64_t page_codes = ((int64_t)a.H << a.b_shift) * D;
  const int64_t head_codes = ((int64_t)h << a.b_shift) * D;

  // 64 groups at a time: their pages and scales, one lane each. A scale is a power of two,
  // which the conversion to bf16 takes, times a rest in [1, 2), which the scores' factor
  // takes for K and the exponent of the probabilities for V: 2^(x - ref + log2 rest) goes into
  // the product, and its sum over a group divided by the rest into l.
  int32_t my_page = 0;
  float my_ks = 0.f, my_vs = 0.f;                // the powers of two
  float my_kf = 0.f, my_vl = 0.f, my_vi = 1.f;   // scores' factor; log2 and inverse of V's rest
  uint64_t absent = 0;
  const auto look_up = [&](int t0) {
    const int my_t = t0 + lane_anew() * 16;
    bool there = false;
    my_page = 0;
    float ks = 1.f, vs = 1.f;
    if (my_t < end) {
      my_page = table[my_t >> a.b_shift];
      there = my_page >= 0 && my_page < a.pages;
      if (!there) my_page = 0;
      ks = a.ks[(int64_t)my_page * a.H + h];
      vs = a.vs[(int64_t)my_page * a.H + h];
    }
    const auto split = [](float s, float& pow) {
      const uint32_t e = __float_as_uint(s) & 0x7F800000u;
      pow = __uint_as_float(e);
      // (an exponent field of 0 stands for 2^-127 in the conversion; a scale of 0 is that)
      if (e == 0) return s == 0.f ? 1.f : fabsf(s) * 0x1p127f;
      return __uint_as_float((__float_as_uint(s) & 0x7FFFFFu) | 0x3F800000u);
    };
    // (not 0, also where the softmax scale is: hidden scores are -inf times it)
    my_kf = fmaxf(split(ks, my_ks) * a.scale_log2, 0x1p-126f);
    const float rest = split(vs, my_vs);
    my_vl = __builtin_amdgcn_logf(rest);
    my_vi = 1.f / rest;
    absent = ~__ballot(there);
  };
  // The wave's share of a tile: group `wave % kGroups`, columns from wave / kGroups * COLS.
  const int my_group = __builtin_amdgcn_readfirstlane(wave % kGroups);
  const int col0 = __builtin_amdgcn_readfirstlane(wave / kGroups * COLS);
  // K: lane = (token lane / 4, quarter of the columns). V: lane = (tokens 4 g + i and 8 + 4 g + i,
  // four columns) or, for 64 columns, (tokens 4 (lane / 16) + i, four columns).
  const uint32_t k_load = (lane >> 2) * D + (lane & 3) * (COLS / 4) + col0;
  const uint32_t v_load = (COLS == 128 ? 4 * g * D + 4 * n : 4 * (lane >> 4) * D + 4 * (lane & 15)) + col0;
  // (what is made of it is computed again for each tile, not kept for all of them in registers)
  const auto fresh = [](uint32_t x) { return (uint32_t)anew((int)x); };
  const auto load = [&](int tile, Codes<COLS>& x) {
    const uint32_t kl = fresh(k_load), vl = fresh(v_load);
    const int gi = (tile * kGroups + my_group) & 63;
    const int64_t page = __builtin_amdgcn_readlane(my_page, gi);
    const int row = __builtin_amdgcn_readfirstlane((begin + tile * TOK + my_group * 16) & (B - 1));
    const int64_t base = page * page_codes + head_codes + (int64_t)row * D;
    const uint8_t* kp = a.kc + base;
#pragma unroll
    for (int w = 0; w < COLS / 64; ++w) x.k[w] = *global_ptr<u32x4>(kp + (kl + 16 * w));
    const uint8_t* vp = a.vc + base;
#pragma unroll
    for (int i = 0; i < COLS / 16; ++i)
      x.v[i] = *global_ptr<uint32_t>(vp + (vl + ((i & 3) + 8 * (i >> 2)) * D));
  };
  // A lane's places in the LDS: what it reads of K and V, what it stages of them.
  const uint32_t k_read = T::k_at(n, half * (DH / 8) + g);
  const uint32_t v_read = T::v_at(half * DH + n, g);
  const uint32_t k_write =
      T::k_at(my_group * 16 + (lane >> 2), (col0 + (lane & 3) * (COLS / 4)) / 8);
  const uint32_t v_write =
      COLS == 128 ? T::v_at(col0 + 4 * n, 2 * my_group + g)
                  : T::v_at(col0 + 4 * (lane & 15), 2 * my_group + ((lane >> 4) & 1)) +
                        8 * (lane >> 5);
  const auto stage = [&](int tile, const Codes<COLS>& x, int buf) {
    const int gi = (tile * kGroups + my_group) & 63;
    const float ks = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_ks), gi));
    const float vs = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_vs), gi));
    const uint32_t kw = fresh(k_write), vw = fresh(v_write);
#pragma unroll
    for (int w = 0; w < COLS / 32; ++w) {
      const uint32_t lo = x.k[w >> 1][2 * (w & 1)], hi2 = x.k[w >> 1][2 * (w & 1) + 1];
      const u32x4 o = {scaled_bf16<false>(lo, ks), scaled_bf16<true>(lo, ks),
                       scaled_bf16<false>(hi2, ks), scaled_bf16<true>(hi2, ks)};
      *reinterpret_cast<u32x4*>(&lds.k[buf][kw ^ (w << 4)]) = o;
    }
    constexpr int NV = COLS / 16;                // tokens of a lane
    uint32_t lo[NV], hi2[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      lo[i] = scaled_bf16<false>(x.v[i], vs);
      hi2[i] = scaled_bf16<true>(x.v[i], vs);
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint32_t sel = c & 1 ? 0x07060302u : 0x05040100u;
      uint32_t o[NV / 2];
#pragma unroll
      for (int k = 0; k < NV / 2; ++k)
        o[k] = c < 2 ? __builtin_amdgcn_perm(lo[2 * k + 1], lo[2 * k], sel)
                     : __builtin_amdgcn_perm(hi2[2 * k + 1], hi2[2 * k], sel);
      // column 4 n + c: its row's number differs from that of c = 0 in c / 2 (TOK 64)
      uint8_t* at = &lds.v[buf][(vw ^ (TOK == 64 ? (c >> 1) << 4 : 0)) + c * TOK * 2];
      if constexpr (COLS == 128) *reinterpret_cast<u32x4*>(at) = u32x4{o[0], o[1], o[2], o[3]};
      else *reinterpret_cast<u32x2*>(at) = u32x2{o[0], o[1]};
    }
  };

  // Operands come from the LDS four products ahead; where an operand has three, six.
  constexpr int kAhead = TERMS == 3 ? 2 : 4;
  const auto k_operand = [&](uint32_t kr, int buf, int e) {  // product e = c * kTok32 + b of the scores
    const int b = e % kTok32, c = e / kTok32;
    return *reinterpret_cast<const u32x4*>(&lds.k[buf][(kr ^ (c << 5)) + b * 32 * D * 2]);
  };
  const auto v_operand = [&](uint32_t vr, int buf, int e) {  // product e = s * DH / 32 + j of the output
    const int s = e / (DH / 32), j = e % (DH / 32);
    return *reinterpret_cast<const u32x4*>(&lds.v[buf][(vr ^ (s << 5)) + j * 32 * TOK * 2]);
  };
  constexpr int kScoreOps = kTok32 * (DH / 16), kOutOps = kGroups * (DH / 32);
  static_assert(kScoreOps >= kAhead && kOutOps >= kAhead, "");
  // The tile's scores, of this wave's half of d; leaves the first operands of V in f.
  const auto scores = [&](f32x16 (&sc)[kTok32], u32x4 (&f)[kAhead], int buf) {
    const uint32_t kr = fresh(k_read), vr = fresh(v_read);
    const uint32_t qr = kKept < DH / 16 ? fresh(q_place) : 0;
#pragma unroll
    for (int b = 0; b < kTok32; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[b][i] = 0.f;
#pragma unroll
    for (int e = 0; e < kAhead; ++e) f[e] = k_operand(kr, buf, e);
#pragma unroll
    for (int e = 0; e < kScoreOps; ++e) {
      const bf16x8 k = __builtin_bit_cast(bf16x8, f[e % kAhead]);
      const int b = e % kTok32, c = e / kTok32;
#pragma unroll
      for (int w = TERMS - 1; w >= 0; --w) {
        const bf16x8 qw = c < kKept ? q[c < kKept ? c : 0][w]
                                    : lds.q[qr + ((c - kKept) * TERMS + w) * 64];
        sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qw, sc[b], 0, 0, 0);
      }
      f[e % kAhead] = e + kAhead < kScoreOps ? k_operand(kr, buf, e + kAhead)
                                             : v_operand(vr, buf, e + kAhead - kScoreOps);

    }
  };
  // The rest of a tile; register i of sc[b] is token 32 b + 8 (i / 4) + 4 g + i % 4 of row n.
  // seen: every row sees every token of the tile.
  const auto compute = [&](f32x16 (&sc)[kTok32], u32x4 (&f)[kAhead], bool seen, int tile, int buf) {
    const int t = begin + tile * TOK;
    const int g0 = (tile * kGroups) & 63;        // the tile's first group among those looked up
    const auto of_group = [&](float x, int s) {
      return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), g0 + s));
    };
    if (!seen) {
      const int lo = see_from() - t - 4 * g, hi = see_hi - t - 4 * g;
#pragma unroll
      for (int b = 0; b < kTok32; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int tt = 32 * b + 8 * (i >> 2) + (i & 3);
          const bool gone = (absent >> (g0 + 2 * b + (i >> 3))) & 1;
          sc[b][i] = tt >= lo && tt < hi && !gone ? sc[b][i] : kNone;
        }
    }
    float best = kNone;
#pragma unroll
    for (int s = 0; s < kGroups; ++s) {
      float x = sc[s >> 1][8 * (s & 1)];
#pragma unroll
      for (int i = 1; i < 8; ++i) x = fmaxf(x, sc[s >> 1][8 * (s & 1) + i]);
      best = fmaxf(best, x * of_group(my_kf, s));
    }
    best = lane_max<32>(best);
    top = fmaxf(top, best);
    // acc and l stay relative to an earlier maximum while the new one is less than 2^8 times it
    if (__any(top > ref + 8.f)) {
      const float shrink = top == kNone ? 1.f : __builtin_amdgcn_exp2f(ref - top);
      l *= shrink;
#pragma unroll
      for (int j = 0; j < DH / 32; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[j][i] *= shrink;
      ref = top;
    }
    const float low = ref == kNone ? 0.f : ref;
    const uint32_t vr = fresh(v_read);
    // out^T += V^T P^T, 16 tokens at a time: registers 8 (s % 2) .. of sc[s / 2], as the sum of
    // PT bf16 terms, each the rounding of what the ones before have left
    const auto products = [&](int s) {
      bf16x8 pt[PT];
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = sc[s >> 1][8 * (s & 1) + i];
      split_terms<PT>(x, pt);
#pragma unroll
      for (int j = 0; j < DH / 32; ++j) {
        const int e = s * (DH / 32) + j;
#pragma unroll
        for (int w = 0; w < PT; ++w)
          acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f[e % kAhead]),
                                                           pt[w], acc[j], 0, 0, 0);
        if (e + kAhead < kOutOps) f[e % kAhead] = v_operand(vr, buf, e + kAhead);
      }
    };
    const auto exponents = [&](int s) {
      const float kf = of_group(my_kf, s), off = of_group(my_vl, s) - low;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = __builtin_amdgcn_exp2f(fmaf(sc[s >> 1][8 * (s & 1) + i], kf, off));
        sc[s >> 1][8 * (s & 1) + i] = x;
        sum += x;
      }
      l = fmaf(sum, of_group(my_vi, s), l);
    };
    exponents(0);
#pragma unroll
    for (int s = 0; s < kGroups; ++s) {
      if (s + 1 < kGroups) exponents(s + 1);
      products(s);
    }
  };

  // In a tile that some row sees only in part, values of V that are not finite: a product of
  // their places with what each row sees finds the rows and columns that become NaN; then
  // they are taken out of the tile, since 0 * NaN would reach the other rows. (All waves come
  // here together.)
  const auto take_out = [&](int tile, int buf) {
    const int tl = lane_anew(), tn = tl & 31, tg = tl >> 5, thread = anew(threadIdx.x);
    int odd = 0;
    for (int x = thread; x < T::kBytes / 16; x += 64 * kWaves) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(&lds.v[buf][16 * x]);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        odd |= (v[k] & 0x7F80u) == 0x7F80u || (v[k] & 0x7F800000u) == 0x7F800000u;
    }
    if (!__syncthreads_or(odd)) return;
    const int t = begin + tile * TOK, see_lo = see_from();
    const int g0 = (tile * kGroups) & 63;
#pragma unroll 1
    for (int s = 0; s < kGroups; ++s) {
      u32x4 by;                                  // 1 where the row sees the token
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int tt = t + 16 * s + 8 * (k >> 1) + 4 * tg + 2 * (k & 1);
        const bool here = !((absent >> (g0 + s)) & 1);
        by[k] = (here && tt >= see_lo && tt < see_hi ? 0x3F80u : 0u) |
                (here && tt + 1 >= see_lo && tt + 1 < see_hi ? 0x3F800000u : 0u);
      }
#pragma unroll
      for (int j = 0; j < DH / 32; ++j) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(
            &lds.v[buf][T::v_at(half * DH + 32 * j + tn, 2 * s + tg)]);
        u32x4 is;                                // 1 where the value is not finite
#pragma unroll
        for (int k = 0; k < 4; ++k)
          is[k] = ((v[k] & 0x7F80u) == 0x7F80u ? 0x3F80u : 0u) |
                  ((v[k] & 0x7F800000u) == 0x7F800000u ? 0x3F800000u : 0u);
        f32x16 hits;
#pragma unroll
        for (int i = 0; i < 16; ++i) hits[i] = 0.f;
        hits = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, is),
                                                       __builtin_bit_cast(bf16x8, by), hits, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (hits[i] > 0.f) acc[j][i] = __builtin_nanf("");
      }
    }
    __syncthreads();
    for (int x = thread; x < T::kBytes / 16; x += 64 * kWaves) {
      u32x4* at = reinterpret_cast<u32x4*>(&lds.v[buf][16 * x]);
      u32x4 v = *at;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        v[k] &= ((v[k] & 0x7F80u) == 0x7F80u ? 0u : 0xFFFFu) |
                ((v[k] & 0x7F800000u) == 0x7F800000u ? 0u : 0xFFFF0000u);
      *at = v;
    }
    __syncthreads();
  };

  // One tile: its scores; the next tile staged and a later one loaded, which the matrix
  // instructions of the scores leave time for; the softmax and the second product. Loads are
  // one or two tiles ahead of the staging, as registers allow.
  // (Past the end of the look-up a tile is staged that nobody reads, and the last one
  // loaded again.)
  constexpr int kLoads = COLS == 128 ? 1 : 2;
  const auto tile_step = [&](int i, int stop, int buf, Codes<COLS>& x) {
    const int t = begin + i * TOK;
    const uint64_t mask = ((1ull << kGroups) - 1) << ((i * kGroups) & 63);
    const bool seen = t >= sight.all_lo && t + TOK <= sight.all_hi && (absent & mask) == 0;
    if (!seen) take_out(i, buf);
    const int ahead = i + 1 + kLoads < stop ? i + 1 + kLoads : stop - 1;
    f32x16 sc[kTok32];
    u32x4 f[kAhead];
    if (wave_live) {
      scores(sc, f, buf);
      stage(i + 1, x, buf ^ 1);
      load(ahead, x);
    } else {
      stage(i + 1, x, buf ^ 1);
      load(ahead, x);
    }
    if constexpr (HALVES == 2) {
      const auto place = [&](int h2, int x) {
        return &lds.half[((row_wave + h2 * kRowWaves) * (4 * kTok32) + x) * 64 + lane];
      };
      if (wave_live) {
#pragma unroll
        for (int x = 0; x < 4 * kTok32; ++x)
          *place(half, x) = f32x4{sc[x >> 2][4 * (x & 3)], sc[x >> 2][4 * (x & 3) + 1],
                                  sc[x >> 2][4 * (x & 3) + 2], sc[x >> 2][4 * (x & 3) + 3]};
      }
      __syncthreads();
      if (wave_live) {
#pragma unroll
        for (int x = 0; x < 4 * kTok32; ++x) {
          const f32x4 o = *place(1 - half, x);
#pragma unroll
          for (int y = 0; y < 4; ++y) sc[x >> 2][4 * (x & 3) + y] += o[y];
        }
      }
    }
    if (wave_live) compute(sc, f, seen, i, buf);
    __syncthreads();
  };
  // Look-ups are for 64 groups; a tile's groups never straddle two of them.
  for (int base = 0; base < tiles; base += kPerLook) {
    look_up(begin + base * TOK);
    const int stop = tiles - base < kPerLook ? tiles : base + kPerLook;
    const auto last = [&](int i) { return i < stop ? i : stop - 1; };
    Codes<COLS> x[kLoads];
    load(base, x[0]);
    if constexpr (kLoads == 2) load(last(base + 1), x[1]);
    __syncthreads();
    stage(base, x[0], 0);
    load(last(base + kLoads), x[0]);
    __syncthreads();
    for (int i = base; i < stop; i += 2) {
      tile_step(i, stop, 0, x[kLoads - 1]);
      if (i + 1 < stop) tile_step(i + 1, stop, 1, x[0]);
    }
  }

  // results: the lane's columns 32 j + 8 b + 4 g + (0 .. 3) of row n
  // (the lane's and the wave's numbers anew: no registers are kept for them through the tiles)
  l = lane_sum<32>(l);
  const int el = lane_anew(), en = el & 31, eg = el >> 5;
  const int ew = my_group + col0 / COLS * kGroups, end_half = ew / kRowWaves;
  const int end_row = ew % kRowWaves * kWaveRows + en;
  if (live) {
    const RowPlace place = row_place(a, it, h, it.tile * kManyRows + end_row);
    const ManyPart<D> part = many_part<D>(a, it, h, it.place);
#pragma unroll
    for (int j = 0; j < DH / 32; ++j)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const f32x4 y = {acc[j][4 * b], acc[j][4 * b + 1], acc[j][4 * b + 2], acc[j][4 * b + 3]};
        const int col = end_half * DH + 32 * j + 8 * b + 4 * eg;
        if (it.splits == 1) put_quad<ES>(a, place, col, y, l);
        else *part.quad(end_row, col / 4) = y;
      }
    if (eg == 0 && end_half == 0) {
      if (it.splits == 1) {
        put_lse(a, place, ref == kNone ? 0.f : ref, l);
      } else {
        *part.stat(end_row) = f32x2v{ref, l};
      }
    }
  }
}

// Requests of many rows in the first `many` workgroups, of few in the others.
template <int TERMS, int D, int TOK, int HALVES>
__global__ __launch_bounds__(64 * kRowWaves * HALVES, many_groups(D, TERMS) * HALVES) void qcache_any_rows_kernel(
    QAttention a, uint32_t many) {
  __shared__ union Shared {
    ManyShared<TERMS, D, TOK, HALVES> many;
    FewShared<TERMS, D, kRowWaves * HALVES> few;
  } lds;
  if (blockIdx.x < many) many_rows_item<TERMS, D, TOK, HALVES>(a, blockIdx.x, lds.many);
  else few_rows_span<TERMS, D, kRowWaves * HALVES>(a, blockIdx.x - many, lds.few);
}

// Joins the partial results of the tiles whose context is cut: kJoinGroups workgroups for each of
// a tile's s items take equal parts of its quads of columns, over all s results, in their order.
// The items are those that the launch before has found. (Joined by the last of a tile's workgroups
// in that launch, 16 questions of 84 rows of d = 256 kept 32 of the 256 compute units busy while
// 18 MB came back, 40 us.)
constexpr int kJoinGroups = 4, kJoinThreads = 256;
template <int D, int ES>
__global__ __launch_bounds__(kJoinThreads) void qcache_join_kernel(QAttention a) {
  const HeadItem hi = head_item(a.H, blockIdx.x);
  if (hi.item >= a.many_places) return;
  const Item it = reinterpret_cast<const Item*>(a.many_found)[hi.item];
  if (!it.any) return;
  const ManyPart<D> p0 = many_part<D>(a, it, hi.h, hi.item - it.split);
  const int total = p0.rows * (D / 4);
  const int parts = it.splits * kJoinGroups, part = it.split * kJoinGroups + (int)blockIdx.y;
  const int share = (total + parts - 1) / parts;
  const int begin = part * share, end = begin + share < total ? begin + share : total;
  const auto join = [&](auto batch) {
    constexpr int BATCH = decltype(batch)::value;
    for (int x = begin + (int)threadIdx.x; x < end; x += kJoinThreads) {
      const int quad = (int)((uint32_t)x / (uint32_t)p0.rows), row = x - quad * p0.rows;
      Joined sum;
      for (int s = 0; s < it.splits; s += BATCH) {
        f32x4 o[BATCH];
        float m[BATCH], l[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
          ManyPart<D> p = p0;
          p.at += (int64_t)(s + k < it.splits ? s + k : s) * ManyPart<D>::kFloats;
          o[k] = *p.quad(row, quad);
          const f32x2v st = *p.stat(row);
          m[k] = st[0];
          l[k] = st[1];
        }
        sum.add(o, m, l, it.splits - s);
      }
      const RowPlace place = row_place(a, it, hi.h, it.tile * kManyRows + row);
      put_quad<ES>(a, place, 4 * quad, sum.o, sum.l);
      if (quad == 0) put_lse(a, place, sum.m == kNone ? 0.f : sum.m, sum.l);
    }
  };
  if (it.splits <= 4) join(std::integral_constant<int, 4>{});
  else if (it.splits <= 8) join(std::integral_constant<int, 8>{});
  else join(std::integral_constant<int, 16>{});
}

}  // namespace

template <int TERMS, int D>
hipError_t launch_qcache_any_rows(const QAttention& a, uint32_t many, uint32_t few,
                                  hipStream_t stream) {
  constexpr int TOK = D == 256 ? 32 : 64;
  constexpr int HALVES = many_halves(D);
  hipLaunchKernelGGL((qcache_any_rows_kernel<TERMS, D, TOK, HALVES>), dim3(many + few),
                     dim3(64 * kRowWaves * HALVES), 0, stream, a, many);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.many_places) return e;
  hipLaunchKernelGGL((qcache_join_kernel<D, TERMS == 1 ? 2 : 4>),
                     dim3((uint32_t)head_groups(a.H, a.many_places), kJoinGroups), dim3(kJoinThreads), 0,
                     stream, a);
  return hipGetLastError();
}

template hipError_t launch_qcache_any_rows<1, 64>(const QAttention&, uint32_t, uint32_t, hipStream_t);
template hipError_t launch_qcache_any_rows<1, 128>(const QAttention&, uint32_t, uint32_t, hipStream_t);
template hipError_t launch_qcache_any_rows<1, 256>(const QAttention&, uint32_t, uint32_t, hipStream_t);
template hipError_t launch_qcache_any_rows<3, 64>(const QAttention&, uint32_t, uint32_t, hipStream_t);
template hipError_t launch_qcache_any_rows<3, 128>(const QAttention&, uint32_t, uint32_t, hipStream_t);
template hipError_t launch_qcache_any_rows<3, 256>(const QAttention&, uint32_t, uint32_t, hipStream_t);

}  // namespace cm
