// K and V rows into the 8-bit paged cache (cm_qcache_write).
//
// The unit of work is a tile: the new rows of one page, for one head, layer and K/V.
// Its scale is the least power of two s with max |x| <= 448 s, so x / s is exact and each
// value is rounded once; e4m3 is a floating format, so the up to one bit of range that a
// power of two leaves unused costs no precision. One pass: a tile's rows are loaded
// into registers, their maximum is taken over the waves that hold them, the codes
// are made from the same registers. A page entered in its middle keeps its scale unless
// the new rows need a greater one; then its earlier rows are read, scaled by a power of
// two and rounded again.
//
// Bound by bandwidth: each row is read once and its codes are written once. All 36 layers of a
// merged cache of 16384 tokens, 8 heads of d = 128 (2.4 GB of bf16 read, 1.2 GB of codes written):
// 652 us, 5.6 TB/s; 32 tokens of one layer 4.0 us.
#include <algorithm>
#include <type_traits>

#include "qcache_ops.h"

namespace cm {

namespace {

struct WriteArgs {
  QRows k, v;
  uint8_t* codes;   // of the first layer written
  float* scales;
  int64_t slice_codes, slice_scales;  // of one (layer, K/V)
  int64_t pages, n_tokens;
  int64_t from;                       // first token of the launch's windows
  const int64_t* slots;
  int32_t H, b_shift, tiles;          // tiles: layers * 2 * H of a page
};

// max over the lanes of a wave, of magnitudes as integers (their order is the values')
__device__ __forceinline__ uint32_t wave_max(uint32_t m) {
#pragma unroll
  for (int by = 1; by < 64; by <<= 1) {
    const uint32_t o = __shfl_xor(m, by);
    m = o > m ? o : m;
  }
  return m;
}

// Largest magnitude of a 16-byte piece, as fp32 bits; FINITE: of its finite values.
template <int ESIZE, bool FINITE>
__device__ __forceinline__ uint32_t piece_max(u32x4 v, uint32_t m) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if constexpr (ESIZE == 4) {
      const uint32_t a = v[w] & 0x7FFFFFFFu;
      if (!FINITE || a < 0x7F800000u) m = a > m ? a : m;
    } else {
      const uint32_t hi = v[w] & 0x7FFF0000u, lo = (v[w] << 16) & 0x7FFF0000u;
      if (!FINITE || hi < 0x7F800000u) m = hi > m ? hi : m;
      if (!FINITE || lo < 0x7F800000u) m = lo > m ? lo : m;
    }
  }
  return m;
}

// Sixteen values (ESIZE 16-byte pieces) times `inv` as sixteen codes.
template <int ESIZE>
__device__ __forceinline__ u32x4 unit_codes(const u32x4 (&v)[ESIZE], float inv) {
  u32x4 out;
  if constexpr (ESIZE == 4) {
#pragma unroll
    for (int w = 0; w < 4; ++w)
      out[w] = codes_of(__uint_as_float(v[w][0]) * inv, __uint_as_float(v[w][1]) * inv,
                        __uint_as_float(v[w][2]) * inv, __uint_as_float(v[w][3]) * inv);
  } else {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t a = v[w >> 1][2 * (w & 1)], b = v[w >> 1][2 * (w & 1) + 1];
      out[w] = codes_of(low_bf16(a) * inv, high_bf16(a) * inv, low_bf16(b) * inv,
                        high_bf16(b) * inv);
    }
  }
  return out;
}

// One workgroup of four waves: 4 / TW tiles of TW waves, at the pages that begin in window
// blockIdx.x of `window` tokens, a.from on. UNITS: 16-element units of a lane.
template <int ESIZE, int D, int TW, int UNITS>
__global__ __launch_bounds__(256) void qcache_write_kernel(WriteArgs a, int32_t window) {
  __shared__ uint32_t s_max[2][4];
  constexpr int kUnitsPerRow = D / 16;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tl = threadIdx.x & (64 * TW - 1);   // thread of the tile
  const int tile = __builtin_amdgcn_readfirstlane((int)blockIdx.y * (4 / TW) + wave / TW);
  if (tile >= a.tiles) return;                  // (TW == 1: whole waves, no barrier below)
  const int h = tile % a.H, kv = (tile / a.H) & 1, layer = tile / (2 * a.H);
  const QRows rows = kv ? a.v : a.k;
  const int64_t slice = 2 * (int64_t)layer + kv;
  const uint8_t* src = rows.data + layer * rows.layer + h * rows.head;
  const int64_t B = (int64_t)1 << a.b_shift, n_slots = a.pages << a.b_shift;
  int turn = 0;

  // The `count` tokens of one page from i on, the first in row `begin` of it, token t in row
  // row_of(t): loaded, their scale, their codes.
  const auto write_page = [&](int64_t i, int64_t page, int count, int begin, auto row_of) {
    float* scale_at = a.scales + slice * a.slice_scales + page * a.H + h;
    uint8_t* codes = a.codes + slice * a.slice_codes + ((page * a.H + h) << a.b_shift) * D;
    u32x4 v[UNITS][ESIZE];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int unit = u * 64 * TW + tl;
      const int t = unit / kUnitsPerRow, col = (unit % kUnitsPerRow) * 16;
      const uint8_t* at = src + (i + t) * rows.token + col * ESIZE;
#pragma unroll
      for (int w = 0; w < ESIZE; ++w) {
        if (t < count) v[u][w] = *(global_ptr<u32x4>(at) + w);
        else v[u][w] = u32x4{0, 0, 0, 0};
      }
    }
    const auto tile_max = [&](bool finite) -> uint32_t {
      uint32_t m = 0;
#pragma unroll
      for (int u = 0; u < UNITS; ++u)
#pragma unroll
        for (int w = 0; w < ESIZE; ++w)
          m = finite ? piece_max<ESIZE, true>(v[u][w], m) : piece_max<ESIZE, false>(v[u][w], m);
      m = wave_max(m);
      if constexpr (TW > 1) {
        uint32_t(&box)[4] = s_max[turn & 1];    // two boxes: a wave may be one turn ahead
        ++turn;
        if (lane == 0) box[wave] = m;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < TW; ++k) {
          const uint32_t o = box[(wave / TW) * TW + k];
          m = o > m ? o : m;
        }
      }
      return m;
    };
    uint32_t top = tile_max(false);
    if constexpr (TW == 2) {
      // two tiles share the workgroup's barriers: both look again if either has to
      bool again = false;
#pragma unroll
      for (int k = 0; k < 4; ++k) again |= s_max[(turn - 1) & 1][k] >= 0x7F800000u;
      if (again) top = tile_max(true);
    } else {
      if (top >= 0x7F800000u) top = tile_max(true);
    }
    float scale = __uint_as_float(scale_bits(top));
    if (begin > 0) {
      const float old = *scale_at;
      const float grown = fmaxf(scale, old);
      if (grown > old) {
        const float ratio = old / grown;
        for (int unit = tl; unit < begin * kUnitsPerRow; unit += 64 * TW) {
          u32x4* at = reinterpret_cast<u32x4*>(codes) + unit;
          u32x4 c = *at;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[w], false);
            const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[w], true);
            c[w] = codes_of(lo[0] * ratio, lo[1] * ratio, hi[0] * ratio, hi[1] * ratio);
          }
          *at = c;
        }
      }
      scale = grown;
    }
    const float inv = 1.0f / scale;
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int unit = u * 64 * TW + tl;
      const int t = unit / kUnitsPerRow, col = (unit % kUnitsPerRow) * 16;
      const int row = row_of(t);
      if (t < count)
        *reinterpret_cast<u32x4*>(codes + row * D + col) = unit_codes<ESIZE>(v[u], inv);
    }
    if constexpr (TW > 1) __syncthreads();      // every wave has read the old scale
    if (tl == 0) *scale_at = scale;
  };

  const int64_t w0 = a.from + (int64_t)blockIdx.x * window;
  // Lanes look at the tokens from the one before the window on: with pages of at most 32
  // tokens 64 of them hold every page that begins in the window, unless tokens are skipped.
  if (B <= 32) {
    const int64_t at = w0 - 1 + lane;
    const int64_t s = at >= 0 && at < a.n_tokens ? a.slots[at] : -1;
    const int page = s >= 0 && s < n_slots ? (int)(s >> a.b_shift) : -1;
    const int row = (int)(s & (B - 1));
    const int before = __shfl_up(page, 1);
    const uint64_t skipped = __ballot(at >= 0 && at < a.n_tokens && page < 0);
    uint64_t first = __ballot(lane >= 1 && lane <= window && page >= 0 && page != before);
    bool simple = skipped == 0;
    for (uint64_t f = first; f && simple; f &= f - 1) {
      const int l = __builtin_ctzll(f);
      const uint64_t other = ~__ballot(page == __builtin_amdgcn_readlane(page, l)) >> l;
      simple = other && __builtin_ctzll(other) <= B;
    }
    if (simple) {
      for (; first; first &= first - 1) {
        const int l = __builtin_ctzll(first);
        const int here = __builtin_amdgcn_readlane(page, l);
        const uint64_t other = ~__ballot(page == here) >> l;
        write_page(w0 - 1 + l, here, __builtin_ctzll(other), __builtin_amdgcn_readlane(row, l),
                   [&](int t) { return __shfl(row, (l + t) & 63); });
      }
      return;
    }
  }

  // Pages of any length, with skipped tokens.
  const auto page_of = [&](int64_t i) -> int64_t {
    const int64_t s = i >= 0 && i < a.n_tokens ? a.slots[i] : -1;
    return s >= 0 && s < n_slots ? s >> a.b_shift : -1;
  };
  // the window's tokens that are the first of their page, skipped tokens aside
  bool first = false;
  if (lane < window) {
    const int64_t p = page_of(w0 + lane);
    if (p >= 0) {
      int64_t j = w0 + lane - 1;
      while (j >= 0 && page_of(j) < 0) --j;
      first = page_of(j) != p;
    }
  }
  uint64_t todo = __ballot(first);
  int64_t next = -1;                            // where the page goes on after skipped tokens
  while (todo || next >= 0) {
    const int64_t i = next >= 0 ? next : w0 + __builtin_ctzll(todo);
    if (next < 0) todo &= todo - 1;
    // the run of tokens in this page: lanes look at the next 128
    const int64_t page = page_of(i);
    const int row_lo = i + lane < a.n_tokens ? (int)(a.slots[i + lane] & (B - 1)) : 0;
    const uint64_t same_lo = __ballot(page_of(i + lane) == page);
    int count = ~same_lo ? __builtin_ctzll(~same_lo) : 64;
    int row_hi = 0;
    if (count == 64) {
      const int64_t j = i + 64 + lane;
      row_hi = j < a.n_tokens ? (int)(a.slots[j] & (B - 1)) : 0;
      const uint64_t same_hi = __ballot(page_of(j) == page);
      count += ~same_hi ? __builtin_ctzll(~same_hi) : 64;
    }
    count = count < B ? count : (int)B;
    const int begin = __builtin_amdgcn_readfirstlane(row_lo);
    next = i + count;
    while (next < a.n_tokens && page_of(next) < 0) ++next;
    if (next >= a.n_tokens || page_of(next) != page) next = -1;
    write_page(i, page, count, begin, [&](int t) {
      const int lo = __shfl(row_lo, t & 63), hi = __shfl(row_hi, t & 63);
      return t < 64 ? lo : hi;
    });
    if (next >= 0) {                            // the tiles are read again
      __threadfence_block();
      if constexpr (TW > 1) __syncthreads();
    }
  }
}

}  // namespace

hipError_t launch_qcache_write(const QCacheDesc& c, int32_t first_layer, int32_t n_layers,
                               int32_t dtype, const QRows& k, const QRows& v, int64_t n_tokens,
                               const int64_t* slots, hipStream_t stream) {
  if (n_tokens == 0 || n_layers == 0) return hipSuccess;
  WriteArgs a;
  a.k = k;
  a.v = v;
  a.slice_codes = c.slice_codes();
  a.slice_scales = c.slice_scales();
  a.codes = c.codes + 2 * (int64_t)first_layer * a.slice_codes;
  a.scales = c.scales + 2 * (int64_t)first_layer * a.slice_scales;
  a.pages = c.pages;
  a.n_tokens = n_tokens;
  a.slots = slots;
  a.H = c.H;
  a.b_shift = c.b_shift;
  a.tiles = n_layers * 2 * c.H;
  const int32_t B = 1 << c.b_shift;
  // Few rows (decoding steps): a window of one token, so that every page has waves of its own.
  // Many: as many tokens as the lanes can look at with the pages that begin among them, at
  // most 32, since a wave without a page would only be in the way (the 4B-N4 merged
  // cache by windows of 16 tokens 709 us, of 32 668; its pages by one token 880).
  const bool bulk = n_tokens * a.tiles > (1 << 14);
  const int32_t window = !bulk ? 1 : B == 32 ? 31 : 32;
  const int64_t windows = (n_tokens + window - 1) / window;
  ScopedTiming tm(K_QCACHE_WRITE, stream);
  const auto go = [&](auto e, auto dd, auto tw, auto units) {
    constexpr int ESIZE = decltype(e)::value, D = decltype(dd)::value, TW = decltype(tw)::value,
                  UNITS = decltype(units)::value;
    // a launch holds at most 2^24 - 1 workgroups of 256 threads a row of the grid
    for (int64_t done = 0; done < windows; done += (1 << 24) - 1) {
      const int64_t some = std::min<int64_t>(windows - done, (1 << 24) - 1);
      const dim3 grid((uint32_t)some, (uint32_t)((a.tiles + 4 / TW - 1) / (4 / TW)));
      a.from = done * window;
      hipLaunchKernelGGL((qcache_write_kernel<ESIZE, D, TW, UNITS>), grid, dim3(256), 0, stream,
                         a, window);
    }
  };
  const auto by_type = [&](auto dd, auto tw, auto units) {
    if (dtype == CM_BF16) go(std::integral_constant<int, 2>{}, dd, tw, units);
    else go(std::integral_constant<int, 4>{}, dd, tw, units);
  };
#define CM_INT(x) std::integral_constant<int, x>{}
  // a tile of B * d elements: up to 32 a lane by waves, then by lanes
  const auto by_tile = [&](auto dd) {
    switch ((B * decltype(dd)::value) >> 10) {
      case 1: by_type(dd, CM_INT(1), CM_INT(1)); break;
      case 2: by_type(dd, CM_INT(1), CM_INT(2)); break;
      case 4: by_type(dd, CM_INT(2), CM_INT(2)); break;
      case 8: by_type(dd, CM_INT(4), CM_INT(2)); break;
      case 16: by_type(dd, CM_INT(4), CM_INT(4)); break;
      default: by_type(dd, CM_INT(4), CM_INT(8)); break;
    }
  };
  switch (c.d) {
    case 64: by_tile(CM_INT(64)); break;
    case 128: by_tile(CM_INT(128)); break;
    default: by_tile(CM_INT(256)); break;
  }
#undef CM_INT
  return hipGetLastError();
}

}  // namespace cm
