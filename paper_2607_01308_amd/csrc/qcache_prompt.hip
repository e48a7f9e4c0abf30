// Attention over the 8-bit paged cache for requests with many query rows: prompts and
// questions of more rows than one 16-row tile holds.
//
// The same one-pass softmax as for few rows (qcache_attention.hip), with the work
// the other way round: a workgroup takes 128 query rows (a request's rows times the
// group) of one KV head, each of its four waves 32 of them, and walks the context in
// tiles of TOK tokens. A tile's codes are turned into bf16 once for all 128 rows, by 2^e of
// their page's scale on the way (the conversion takes the power of two at no cost; scales
// that are no powers of two leave a factor in [1, 2) for the scores and the
// probabilities), and staged in the LDS: K row-major, V transposed. Both products are
// computed transposed by 32x32x16 matrix instructions, S^T = K Q^T and out^T = V^T P^T, so that a
// lane holds of S^T exactly the probabilities that it has to supply of P^T; V's columns
// are laid out in that order of the tokens: element e of 16-byte chunk 2 s + k of a row is
// token 16 s + 8 (e / 4) + 4 k + e % 4. Chunks are moved within their rows by an exclusive
// or with the row's number so that the lanes of a load take all banks.
//
// Bound by the matrix and the vector units in about equal parts: for 32 rows and 64 tokens of
// d = 128 a wave issues 32 products of 32 cycles and about 250 vector instructions.
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

// Bytes of the K and V tiles, and a chunk's place in them.
template <int D, int TOK>
struct Tile {
  static constexpr int kBytes = D * TOK * 2;
  // K: row = token, D / 8 chunks
  static __device__ __forceinline__ int k_at(int tok, int chunk) {
    const int x = D == 64 ? (tok >> 1) & 7 : tok & 15;
    return tok * D * 2 + ((chunk ^ x) << 4);
  }
  // V: row = column of V, TOK / 8 chunks
  static __device__ __forceinline__ int v_at(int col, int chunk) {
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

// The LDS of a workgroup.
template <int D, int TOK, int HALVES>
struct ManyShared {
  uint8_t k[2][D * TOK * 2];
  uint8_t v[2][D * TOK * 2];
  // halves of scores that waves exchange
  f32x4 half[HALVES == 2 ? kRowWaves * HALVES * (TOK / 32) * 4 * 64 : 1];
  int odd[64 / (TOK / 16)];                      // a value that is not finite among a tile's V
  FindShared find;
  int flag;
};

// HALVES 2: two waves share 32 rows, each half of d: half of the sum of a score, which
// they exchange through the LDS, and half of the output's columns.
template <int TERMS, int D, int TOK, int HALVES>
__device__ __forceinline__ void many_rows_item(const QAttention& a, int block,
                                               ManyShared<D, TOK, HALVES>& lds) {
  using T = Tile<D, TOK>;
  constexpr int kWaves = kRowWaves * HALVES;
  constexpr int DH = D / HALVES;                 // columns of a wave
  constexpr int ES = TERMS == 1 ? 2 : 4;
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
  const Item it = find_item<kManyRows, 64 * kWaves>(a, a.many_items, item, lds.find);
  if (!it.any) return;

  // the lane's query row
  const int rho = it.tile * kManyRows + row_wave * kWaveRows + n;
  const int tok = rho / a.G;
  const bool live = tok < it.count;
  const int head = h * a.G + rho % a.G;
  const int p = it.len - it.count + tok;
  const int see_hi = live && p >= 0 ? p + 1 : 0;
  const int see_lo = a.window && p - a.window + 1 > 0 ? p - a.window + 1 : 0;
  const Sight sight = tile_sight<kManyRows>(a, it);
  const bool wave_live = it.tile * kManyRows + row_wave * kWaveRows < it.count * a.G;

  int begin = it.begin + it.split * it.chunk, end = begin + it.chunk;
  const int from = sight.any_lo & ~(TOK - 1);
  begin = begin > from ? begin : from;
  end = end < sight.any_hi ? end : sight.any_hi;
  const int tiles = end > begin ? (end - begin + TOK - 1) / TOK : 0;

  bf16x8 q[DH / 16][TERMS];
#pragma unroll
  for (int c = 0; c < DH / 16; ++c)
    load_query<TERMS>(a, it.row0 + tok, head, half * DH + c * 16 + g * 8, live, q[c]);

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

  // 64 groups at a time: their pages and scales, one lane each
  int32_t my_page = 0;
  float my_ks = 0.f, my_vs = 0.f;                // the powers of two
  float my_kf = 1.f, my_vf = 1.f;                // what is left of the scales
  uint64_t absent = 0, uneven = 0;
  const auto look_up = [&](int t0) {
    const int my_t = t0 + lane * 16;
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
    const auto split = [](float s, float& pow, float& rest) {
      const uint32_t e = __float_as_uint(s) & 0x7F800000u;
      pow = __uint_as_float(e);
      // (an exponent field of 0 stands for 2^-127 in the conversion)
      rest = e == 0 ? s * 0x1p127f : __uint_as_float((__float_as_uint(s) & 0x807FFFFFu) | 0x3F800000u);
    };
    split(ks, my_ks, my_kf);
    split(vs, my_vs, my_vf);
    absent = ~__ballot(there);
    uneven = __ballot(my_kf != 1.f || my_vf != 1.f);
  };
  // The wave's share of a tile: group `wave % kGroups`, columns from wave / kGroups * COLS.
  const int my_group = wave % kGroups, col0 = wave / kGroups * COLS;
  const auto load = [&](int tile, Codes<COLS>& x) {
    const int gi = (tile * kGroups + my_group) & 63;
    const int64_t page = __builtin_amdgcn_readlane(my_page, gi);
    const int row = (begin + tile * TOK + my_group * 16) & (B - 1);
    const int64_t base = page * page_codes + head_codes + (int64_t)row * D + col0;
    // K: lane = (token lane / 4, quarter of the columns)
    const uint8_t* kp = a.kc + base + (lane >> 2) * D + (lane & 3) * (COLS / 4);
#pragma unroll
    for (int w = 0; w < COLS / 64; ++w) x.k[w] = *(global_ptr<u32x4>(kp) + w);
    const uint8_t* vp = a.vc + base;
    if constexpr (COLS == 128) {
      // V: lane = (tokens 4 g + i and 8 + 4 g + i, four columns)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        x.v[i] = *global_ptr<uint32_t>(vp + ((i & 3) + 4 * g + 8 * (i >> 2)) * D + 4 * n);
    } else {
      // V: lane = (tokens 4 (lane / 16) + i, four columns)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        x.v[i] = *global_ptr<uint32_t>(vp + (4 * (lane >> 4) + i) * D + 4 * (lane & 15));
    }
  };
  const auto stage = [&](int tile, const Codes<COLS>& x, int buf) {
    const int gi = (tile * kGroups + my_group) & 63;
    const float ks = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_ks), gi));
    const float vs = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_vs), gi));
    {
      const int t = my_group * 16 + (lane >> 2);
#pragma unroll
      for (int w = 0; w < COLS / 64; ++w)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint32_t lo = x.k[w][2 * half], hi2 = x.k[w][2 * half + 1];
          const u32x4 o = {scaled_bf16<false>(lo, ks), scaled_bf16<true>(lo, ks),
                           scaled_bf16<false>(hi2, ks), scaled_bf16<true>(hi2, ks)};
          const int chunk = (col0 + (lane & 3) * (COLS / 4)) / 8 + 2 * w + half;
          *reinterpret_cast<u32x4*>(&lds.k[buf][T::k_at(t, chunk)]) = o;
        }
    }
    bool odd = false;
    constexpr int NV = COLS / 16;                // tokens of a lane
    uint32_t lo[NV], hi2[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      odd |= nan_codes(x.v[i]) != 0;
      lo[i] = scaled_bf16<false>(x.v[i], vs);
      hi2[i] = scaled_bf16<true>(x.v[i], vs);
    }
    odd |= (__float_as_uint(vs) & 0x7F800000u) == 0x7F800000u;
    if (odd) lds.odd[tile & (kPerLook - 1)] = 1;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint32_t sel = c & 1 ? 0x07060302u : 0x05040100u;
      uint32_t o[NV / 2];
#pragma unroll
      for (int k = 0; k < NV / 2; ++k)
        o[k] = c < 2 ? __builtin_amdgcn_perm(lo[2 * k + 1], lo[2 * k], sel)
                     : __builtin_amdgcn_perm(hi2[2 * k + 1], hi2[2 * k], sel);
      if constexpr (COLS == 128) {
        *reinterpret_cast<u32x4*>(&lds.v[buf][T::v_at(col0 + 4 * n + c, 2 * my_group + g)]) =
            u32x4{o[0], o[1], o[2], o[3]};
      } else {
        // tokens 4 quad + i: chunk 2 group + quad % 2, half quad / 2
        const int quad = lane >> 4;
        *reinterpret_cast<u32x2*>(
            &lds.v[buf][T::v_at(col0 + 4 * (lane & 15) + c, 2 * my_group + (quad & 1)) +
                      8 * (quad >> 1)]) = u32x2{o[0], o[1]};
      }
    }
  };

  // The tile's scores, of this wave's half of d.
  const auto scores = [&](f32x16 (&sc)[kTok32], int buf) {
#pragma unroll
    for (int b = 0; b < kTok32; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[b][i] = 0.f;
#pragma unroll
    for (int c = 0; c < DH / 16; ++c) {
#pragma unroll
      for (int b = 0; b < kTok32; ++b) {
        const bf16x8 k = __builtin_bit_cast(
            bf16x8, *reinterpret_cast<const u32x4*>(
                        &lds.k[buf][T::k_at(32 * b + n, half * (DH / 8) + 2 * c + g)]));
#pragma unroll
        for (int w = TERMS - 1; w >= 0; --w)
          sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[c][w], sc[b], 0, 0, 0);
      }
    }
  };
  // The rest of a tile; register i of sc[b] is token 32 b + 8 (i / 4) + 4 g + i % 4 of row n.
  // seen: every row sees every token of the tile.
  const auto compute = [&](f32x16 (&sc)[kTok32], bool seen, int tile, int buf) {
    const int t = begin + tile * TOK;
    const int g0 = (tile * kGroups) & 63;        // the tile's first group among those looked up
    const bool plain = ((uneven >> g0) & ((1ull << kGroups) - 1)) == 0;
    if (!plain) {
#pragma unroll
      for (int s = 0; s < kGroups; ++s) {
        const float f = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_kf), g0 + s));
#pragma unroll
        for (int i = 0; i < 8; ++i) sc[s >> 1][8 * (s & 1) + i] *= f;
      }
    }
    if (!seen) {
      const int lo = see_lo - t - 4 * g, hi = see_hi - t - 4 * g;
#pragma unroll
      for (int b = 0; b < kTok32; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int tt = 32 * b + 8 * (i >> 2) + (i & 3);
          const bool gone = (absent >> (g0 + 2 * b + (i >> 3))) & 1;
          sc[b][i] = tt >= lo && tt < hi && !gone ? sc[b][i] : kNone;
        }
    }
    float best = sc[0][0];
#pragma unroll
    for (int b = 0; b < kTok32; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) best = fmaxf(best, sc[b][i]);
    best = fmaxf(best, __shfl_xor(best, 32));
    top = fmaxf(top, best * a.scale_log2);
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
    // terms of a probability: fp32 queries take three; bf16 queries two while a single
    // weight may be more than 1/32 of a row's sum, then one (an error of 2^-8 of 2^-5)
    bool fine = TERMS == 3;
    if constexpr (TERMS == 1) {
      const float whole = l + __shfl_xor(l, 32);
      fine = __any(live && !(whole >= 32.f * __builtin_amdgcn_exp2f(top - low)));
    }
#pragma unroll
    for (int b = 0; b < kTok32; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        sc[b][i] = __builtin_amdgcn_exp2f(fmaf(sc[b][i], a.scale_log2, -low));
        l += sc[b][i];
      }
    if (!plain) {
#pragma unroll
      for (int s = 0; s < kGroups; ++s) {
        const float f = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_vf), g0 + s));
#pragma unroll
        for (int i = 0; i < 8; ++i) {            // (the scale may be NaN where nothing is seen)
          const float x = sc[s >> 1][8 * (s & 1) + i];
          sc[s >> 1][8 * (s & 1) + i] = x == 0.f ? 0.f : x * f;
        }
      }
    }
    // out^T += V^T P^T, one term of the probabilities after the other
    for (int more = TERMS == 3 ? 2 : fine ? 1 : 0;; --more) {
#pragma unroll
      for (int s = 0; s < kGroups; ++s) {        // 16 tokens: registers 8 (s % 2) .. of sc[s / 2]
        u32x4 w;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          w[k] = pair_bf16(sc[s >> 1][8 * (s & 1) + 2 * k], sc[s >> 1][8 * (s & 1) + 2 * k + 1]);
        const bf16x8 pt = __builtin_bit_cast(bf16x8, w);
#pragma unroll
        for (int j = 0; j < DH / 32; ++j) {
          const u32x4 v = *reinterpret_cast<const u32x4*>(
              &lds.v[buf][T::v_at(half * DH + 32 * j + n, 2 * s + g)]);
          acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), pt, acc[j],
                                                           0, 0, 0);
        }
      }
      if (more == 0) break;
      // (what follows belongs to the next term alone: nothing of it, nor the loads of V,
      // is to move before the branch)
      asm volatile("" ::: "memory");
#pragma unroll
      for (int b = 0; b < kTok32; ++b) asm volatile("" : "+v"(sc[b]));
#pragma unroll
      for (int b = 0; b < kTok32; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          const uint32_t w = pair_bf16(sc[b][i], sc[b][i + 1]);
          sc[b][i] -= low_bf16(w);
          sc[b][i + 1] -= high_bf16(w);
        }
    }
  };

  // Values of V that are not finite, in a tile that some row sees only in part: a product
  // of their places with what each row sees finds the rows and columns that become NaN;
  // then they are taken out of the tile, since 0 * NaN would reach the other rows. (Rare,
  // and all waves come here together.)
  const auto take_out = [&](int tile, int buf) {
    const int t = begin + tile * TOK;
    const int g0 = (tile * kGroups) & 63;
#pragma unroll 1
    for (int s = 0; s < kGroups; ++s) {
      u32x4 by;                                  // 1 where the row sees the token
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int tt = t + 16 * s + 8 * (k >> 1) + 4 * g + 2 * (k & 1);
        const bool here = !((absent >> (g0 + s)) & 1);
        by[k] = (here && tt >= see_lo && tt < see_hi ? 0x3F80u : 0u) |
                (here && tt + 1 >= see_lo && tt + 1 < see_hi ? 0x3F800000u : 0u);
      }
#pragma unroll
      for (int j = 0; j < DH / 32; ++j) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(
            &lds.v[buf][T::v_at(half * DH + 32 * j + n, 2 * s + g)]);
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
    for (int x = threadIdx.x; x < T::kBytes / 16; x += 64 * kWaves) {
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

  // Tiles: loaded two ahead, staged one ahead, one barrier each. Look-ups are for 64
  // groups; a tile's groups never straddle two of them.
  for (int base = 0; base < tiles; base += kPerLook) {
    if (threadIdx.x < kPerLook) lds.odd[threadIdx.x] = 0;
    look_up(begin + base * TOK);
    const int stop = tiles - base < kPerLook ? tiles : base + kPerLook;
    Codes<COLS> x;
    load(base, x);
    __syncthreads();
    stage(base, x, base & 1);
    if (base + 1 < stop) load(base + 1, x);
    __syncthreads();
    for (int i = base; i < stop; ++i) {
      const int t = begin + i * TOK;
      const uint64_t mask = ((1ull << kGroups) - 1) << ((i * kGroups) & 63);
      const bool seen = t >= sight.all_lo && t + TOK <= sight.all_hi && (absent & mask) == 0;
      if (!seen && lds.odd[i & (kPerLook - 1)] != 0) take_out(i, i & 1);
      f32x16 sc[kTok32];
      if constexpr (HALVES == 1) {
        if (wave_live) {
          scores(sc, i & 1);
          compute(sc, seen, i, i & 1);
        }
      } else {
        if (wave_live) scores(sc, i & 1);
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
          compute(sc, seen, i, i & 1);
        }
      }
      if (i + 1 < stop) {
        stage(i + 1, x, (i + 1) & 1);
        if (i + 2 < stop) load(i + 2, x);
      }
      __syncthreads();
    }
  }

  // results: the lane's columns 32 j + 8 b + 4 g + (0 .. 3) of row n
  l += __shfl_xor(l, 32);
  if (live) {
    const RowPlace place = row_place(a, it, h, rho);
    const Part<kManyRows, D> part = part_of<kManyRows, D>(a, h, item);
    const int row = row_wave * kWaveRows + n;
#pragma unroll
    for (int j = 0; j < DH / 32; ++j)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const f32x4 y = {acc[j][4 * b], acc[j][4 * b + 1], acc[j][4 * b + 2], acc[j][4 * b + 3]};
        const int col = half * DH + 32 * j + 8 * b + 4 * g;
        if (it.splits == 1) put_quad<ES>(a, place, col, y, l);
        else part.put_quad(row, col / 4, y);
      }
    if (g == 0 && half == 0) {
      if (it.splits == 1) {
        put_lse(a, place, ref == kNone ? 0.f : ref, l);
      } else {
        part.put_stat(0, row, ref, l);
      }
    }
  }
  if (it.splits > 1)
    finish_split<kManyRows, D, ES, 64 * kWaves>(a, it, h, it.split, it.splits, &lds.flag,
                                                [&](int i) { return item - it.split + i; });
}

// Requests of many rows in the first `many` workgroups, of few in the others.
template <int TERMS, int D, int TOK, int HALVES>
__global__ __launch_bounds__(64 * kRowWaves * HALVES, 2) void qcache_any_rows_kernel(
    QAttention a, uint32_t many) {
  __shared__ union Shared {
    ManyShared<D, TOK, HALVES> many;
    FewShared<D, kRowWaves * HALVES> few;
  } lds;
  if (blockIdx.x < many) many_rows_item<TERMS, D, TOK, HALVES>(a, blockIdx.x, lds.many);
  else few_rows_span<TERMS, D, kRowWaves * HALVES>(a, blockIdx.x - many, lds.few);
}

}  // namespace

template <int TERMS, int D>
hipError_t launch_qcache_any_rows(const QAttention& a, uint32_t many, uint32_t few,
                                  hipStream_t stream) {
  // a wave's registers hold its queries' terms, d TERMS / 4 of them, and its columns of the output,
  // d / 2; beyond 96 two waves share the rows
  constexpr int TOK = D == 256 ? 32 : 64;
  constexpr int HALVES = D * (TERMS + 1) > 256 ? 2 : 1;
  hipLaunchKernelGGL((qcache_any_rows_kernel<TERMS, D, TOK, HALVES>), dim3(many + few),
                     dim3(64 * kRowWaves * HALVES), 0, stream, a, many);
  return hipGetLastError();
}

template hipError_t launch_qcache_any_rows<1, 64>(const QAttention&, uint32_t, uint32_t, hipStream_t);
template hipError_t launch_qcache_any_rows<1, 128>(const QAttention&, uint32_t, uint32_t, hipStream_t);
template hipError_t launch_qcache_any_rows<1, 256>(const QAttention&, uint32_t, uint32_t, hipStream_t);
template hipError_t launch_qcache_any_rows<3, 64>(const QAttention&, uint32_t, uint32_t, hipStream_t);
template hipError_t launch_qcache_any_rows<3, 128>(const QAttention&, uint32_t, uint32_t, hipStream_t);
template hipError_t launch_qcache_any_rows<3, 256>(const QAttention&, uint32_t, uint32_t, hipStream_t);

}  // namespace cm
