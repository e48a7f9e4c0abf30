// Norms of queries and keys for each head, with the rotation for their positions in the same
// pass (cm_norm_rotate).
//
// Of a row x of d elements: y = x / sqrt(mean x^2 + eps) * w, then pair i of y is turned by the
// angle p * base^(-2i/d). The angle is made in revolutions: the frequency base^(-2i/d) / 2 pi and its
// product with the position in fp64, whose whole turns are taken off before the rest is
// rounded to fp32, so that far positions lose nothing; sine and cosine, the mean and the
// products are in fp32, and a result is rounded once.
//
// A lane holds two 16-byte pieces of a row, one of each half of it at the same place, so that the
// pairs of either style are its own; d / (2 * elements of a piece) lanes share a row and sum its
// squares within the wave. A wave takes several heads of one token, for which its angles are
// the same. A row whose squares leave the range of fp32 downwards is taken times 2^96 where eps does not
// cover what is lost. As many waves as run together take the tokens one after another, so that each reads the weights
// and makes its frequencies once (twice as many waves, weights read one by one: 78 us). 16384
// tokens of 40 heads of 128, bf16: 67 us, 4.9 TB/s, what a copy reaches, vector instructions in 69% of the SIMDs' time.
#include <cmath>
#include <type_traits>

#include "draft.h"
#include "qcache_ops.h"

namespace cm {

namespace {

constexpr int kThreads = 256;
constexpr int kGroups = 4;             // workgroups of a compute unit (111 registers a lane)

template <int CTRL>
__device__ __forceinline__ float moved(float x) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, true));
}
// Sum over the N lanes that share a row, aligned groups of 4 to 32.
template <int N>
__device__ __forceinline__ float row_sum(float x) {
  x += moved<0xB1>(x);                   // quad_perm [1, 0, 3, 2]
  x += moved<0x4E>(x);                   // quad_perm [2, 3, 0, 1]
  if constexpr (N >= 8) x += moved<0x141>(x);   // row_half_mirror
  if constexpr (N >= 16) x += moved<0x140>(x);  // row_mirror
  if constexpr (N >= 32) x = lane_sum<16>(x);
  return x;
}

// A 16-byte piece as fp32 values, and back.
template <int ES>
__device__ __forceinline__ void unpack(u32x4 v, float (&x)[16 / ES]) {
  if constexpr (ES == 4) {
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = __uint_as_float(v[k]);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[2 * k] = low_bf16(v[k]);
      x[2 * k + 1] = high_bf16(v[k]);
    }
  }
}
template <int ES>
__device__ __forceinline__ u32x4 pack(const float (&x)[16 / ES]) {
  u32x4 v;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (ES == 4) v[k] = __float_as_uint(x[k]);
    else v[k] = pair_bf16(x[2 * k], x[2 * k + 1]);
  }
  return v;
}

// E weights from element i on (at any address of their type's), 1 where there are none.
typedef uint32_t words4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t words2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t half_words2 __attribute__((ext_vector_type(2), aligned(2)));
template <int E>
__device__ __forceinline__ void weights(const HeadRows& r, int i, float (&w)[E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) w[e] = 1.f;
  if (!r.weight) return;
  if (r.weight_dtype == CM_F32) {
#pragma unroll
    for (int k = 0; k < E / 4; ++k) {
      const words4 x = *(const CM_GLOBAL words4*)(global_ptr<float>(r.weight) + i + 4 * k);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[4 * k + e] = __uint_as_float(x[e]);
    }
  } else {
    const CM_GLOBAL uint16_t* at = global_ptr<uint16_t>(r.weight) + i;
    uint32_t x[E / 2];
    if constexpr (E == 8) {
      const words2 y = *(const CM_GLOBAL words2*)at;
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = y[k];
    } else {
      const half_words2 y = *(const CM_GLOBAL half_words2*)at;
#pragma unroll
      for (int k = 0; k < 2; ++k) x[k] = y[k];
    }
#pragma unroll
    for (int k = 0; k < E / 2; ++k) {
      w[2 * k] = low_bf16(x[k]);
      w[2 * k + 1] = high_bf16(x[k]);
    }
  }
}

// parts: waves that share a token's heads; groups: row groups of a wave's width that a token has.
template <int ES, int D, bool HALF>
__global__ __launch_bounds__(kThreads, kGroups) void norm_rotate_kernel(RotateArgs a, int32_t parts,
                                                               int32_t groups, int64_t units) {
  constexpr int E = 16 / ES;             // elements of a piece
  constexpr int kLanes = D / (2 * E);    // lanes of a row
  constexpr int kRows = 64 / kLanes;     // rows of a wave
  const int lane = threadIdx.x & 63;
  const int within = lane % kLanes, c0 = within * E;
  const int64_t waves = (int64_t)gridDim.x * (kThreads / 64);
  const int per = (groups + parts - 1) / parts;
  float qw[2][E], kw[2][E];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    weights(a.q, c0 + s * (D / 2), qw[s]);
    weights(a.k, c0 + s * (D / 2), kw[s]);
  }
  // revolutions a position, of the lane's pairs: those of its first one times the powers of the base
  // between them, which the host made (an exp2 in fp64 for each pair took as long as a token's heads)
  double freq[E];
  const double first = 0.15915494309189535 * exp2(-(2.0 / D) * (HALF ? c0 : c0 / 2) * a.log2_base);
#pragma unroll
  for (int e = 0; e < E; ++e) {
    freq[e] = first * a.between[e];
  }
  for (int64_t u = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); u < units; u += waves) {
    const int64_t t = parts == 1 ? u : u / parts;
    const int part = parts == 1 ? 0 : (int)(u - t * parts);
    const double p = a.positions[t];
    float cs[E], sn[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const double turns = p * freq[e];
      sincospif((float)(2.0 * (turns - rint(turns))), &sn[e], &cs[e]);
    }
    const int end = (part + 1) * per < groups ? (part + 1) * per : groups;
    for (int group = part * per; group < end; ++group) {
      const int row = group * kRows + lane / kLanes;
      const bool is_k = row >= a.q.heads;
      const int head = is_k ? row - a.q.heads : row;
      if (is_k && head >= a.k.heads) continue;  // (whole rows: the lanes of a row stay together)
      const uint8_t* in = is_k ? a.k.in + t * a.k.in_token + head * a.k.in_head
                               : a.q.in + t * a.q.in_token + head * a.q.in_head;
      uint8_t* out = is_k ? a.k.out + t * a.k.out_token + head * a.k.out_head
                          : a.q.out + t * a.q.out_token + head * a.q.out_head;
      in += within * 16;
      out += within * 16;
      float x[2][E];
      unpack<ES>(*global_ptr<u32x4>(in), x[0]);
      unpack<ES>(*global_ptr<u32x4>(in + D / 2 * ES), x[1]);
      if (is_k ? a.k.weight != nullptr : a.q.weight != nullptr) {
        const auto squares = [&] {
          float sum = 0.f;
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int e = 0; e < E; ++e) sum = fmaf(x[s][e], x[s][e], sum);
          return row_sum<kLanes>(sum);
        };
        float sum = squares(), eps = a.eps;
        // (rows whose squares leave the range of fp32 downwards, times 2^96, where eps does not cover that)
        if (a.eps < 0x1p-66f && __any(sum < 0x1p-96f)) {
          const float up = sum < 0x1p-96f ? 0x1p96f : 1.f;
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int e = 0; e < E; ++e) x[s][e] *= up;
          sum = squares();
          eps = eps * up * up;
        }
        const float inv = 1.f / sqrtf(sum * (1.f / D) + eps);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int e = 0; e < E; ++e) x[s][e] = x[s][e] * inv * (is_k ? kw[s][e] : qw[s][e]);
      }
      float y[2][E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        // the pair's places: across the pieces, or side by side in one
        const int s0 = HALF ? 0 : e / (E / 2), e0 = HALF ? e : 2 * (e % (E / 2));
        const int s1 = HALF ? 1 : s0, e1 = HALF ? e : e0 + 1;
        const float u0 = x[s0][e0], u1 = x[s1][e1];
        y[s0][e0] = fmaf(u0, cs[e], -(u1 * sn[e]));
        y[s1][e1] = fmaf(u1, cs[e], u0 * sn[e]);
      }
      *reinterpret_cast<u32x4*>(out) = pack<ES>(y[0]);
      *reinterpret_cast<u32x4*>(out + D / 2 * ES) = pack<ES>(y[1]);
    }
  }
}

}  // namespace

hipError_t launch_norm_rotate(RotateArgs a, int32_t d, int32_t dtype, int32_t style,
                              hipStream_t stream) {
  if (a.n_tokens == 0 || a.q.heads + a.k.heads == 0) return hipSuccess;
  const auto go = [&](auto es, auto dd, auto half) -> hipError_t {
    constexpr int ES = decltype(es)::value, D = decltype(dd)::value;
    constexpr bool HALF = decltype(half)::value;
    constexpr int kRows = 64 / (D / (2 * (16 / ES)));
    constexpr int E = 16 / ES;
    for (int e = 0; e < E; ++e)
      a.between[e] = std::exp2(-(2.0 / D) * (HALF || e < E / 2 ? e : D / 4 + e - E / 2) * a.log2_base);
    const int32_t groups = (a.q.heads + a.k.heads + kRows - 1) / kRows;
    // a token's heads by as many waves as fill the GPU
    const int64_t fill = (int64_t)device_cu_count() * 16;
    int32_t parts = (int32_t)(fill / a.n_tokens < 1 ? 1 : fill / a.n_tokens > groups ? groups : fill / a.n_tokens);
    const int32_t per = (groups + parts - 1) / parts;
    parts = (groups + per - 1) / per;
    const int64_t units = a.n_tokens * parts, most = (int64_t)device_cu_count() * kGroups;
    const int64_t blocks = (units + kThreads / 64 - 1) / (kThreads / 64);
    ScopedTiming tm(K_NORM_ROTATE, stream);
    hipLaunchKernelGGL((norm_rotate_kernel<ES, D, HALF>), dim3((uint32_t)(blocks < most ? blocks : most)),
                       dim3(kThreads), 0, stream, a, parts, groups, units);
    return hipGetLastError();
  };
  const auto by_style = [&](auto es, auto dd) {
    return style == CM_ROPE_HALF ? go(es, dd, std::true_type{}) : go(es, dd, std::false_type{});
  };
  const auto by_d = [&](auto es) {
    switch (d) {
      case 64: return by_style(es, std::integral_constant<int, 64>{});
      case 128: return by_style(es, std::integral_constant<int, 128>{});
      default: return by_style(es, std::integral_constant<int, 256>{});
    }
  };
  return dtype == CM_BF16 ? by_d(std::integral_constant<int, 2>{}) : by_d(std::integral_constant<int, 4>{});
}

}  // namespace cm
