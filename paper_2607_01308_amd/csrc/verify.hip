// Drafted tokens verified against the target's probabilities, from given random numbers
// (cm_verify_drafts).
//
// A walk from a request's node 0: the children x of a node are tried in order. With the node's row
// p and the row q of probabilities that its children were sampled from, child x of token t is
// accepted if u q(t) m < r(t); r = p and m = 1 at first, and a rejection leaves
// r' = max(r - m q, 0), m' = sum r'. Since max(max(a - b, 0) - c, 0) = max(a - (b + c), 0) for
// b, c >= 0, r after any number of rejections is max(p - M q, 0) with M the sum of their m:
// one number is all that is kept. Without q a drafted token counts as certain: a rejection takes it
// out of r, and its probability off m. Where no child is accepted the next token is the first v with
// r_0 + .. + r_v > s sum r. Sums and comparisons are in fp64: u q(t) is then exact, and sums of a
// hundred thousand terms are off by 1e-14 of themselves, not by 1e-6, beside which the borders of
// a sampled token lie close.
//
// A workgroup takes a request: its walk looks at single probabilities, which it has read at once into
// the LDS, and a pass over a row sums r where a rejected child has a sibling after it or the token is
// to be sampled. A pass is bound by the vector instructions of its compute unit, 9 for an element (two
// conversions and three operations in fp64, the check of its bits): 100003 tokens about 6 us. So
// other workgroups help where few requests leave the GPU idle: each sums its parts of the row for the
// passes that it is told of, through memory, in about 4 us with all trips; nobody waits for another for
// longer than verify_waits says. 32 trees of up to 25 nodes over 100003 tokens: 33 us (47 us alone), as long as
// the request with the most rejections takes. Without q every child that was rejected is looked for in every
// eight elements: 32 requests of 63 children 87 us, 22 where they are up to three of a node.
#include "draft.h"
#include "qcache_ops.h"

namespace cm {

namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kGroups = 2;           // workgroups of a compute unit
constexpr int kParts = 64;           // parts of a row at most
constexpr int64_t kPart = 8192;      // elements of one, or a multiple
constexpr int kVec = 8;              // elements of a lane's load
constexpr int kStep = 64 * kVec;     // and of a wave's

// What is not a probability counts as none.
__device__ __forceinline__ double clean(float x) {
  return x > 0.f && x < __builtin_inff() ? (double)x : 0.0;
}

template <int ES>
__device__ __forceinline__ float element(const void* row, int64_t v) {
  if constexpr (ES == 4) return *(global_ptr<float>(row) + v);
  else return __uint_as_float((uint32_t) * (global_ptr<uint16_t>(row) + v) << 16);
}

// kVec elements from v on as they are in memory; rows begin at any element.
typedef uint32_t words_f32 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t words_bf16 __attribute__((ext_vector_type(4), aligned(2)));
template <int ES>
struct Raw {
  u32x4 w[ES / 2];
};
template <int ES>
__device__ __forceinline__ Raw<ES> load_raw(const void* row, int64_t v) {
  Raw<ES> x;
  if constexpr (ES == 4) {
    const CM_GLOBAL float* at = global_ptr<float>(row) + v;
    x.w[0] = *(const CM_GLOBAL words_f32*)at;
    x.w[1] = *(const CM_GLOBAL words_f32*)(at + 4);
  } else {
    x.w[0] = *(const CM_GLOBAL words_bf16*)(global_ptr<uint16_t>(row) + v);
  }
  return x;
}
template <int ES>
__device__ __forceinline__ void unpack(const Raw<ES>& raw, float (&x)[kVec]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (ES == 4) {
      x[k] = __uint_as_float(raw.w[0][k]);
      x[4 + k] = __uint_as_float(raw.w[1][k]);
    } else {
      x[2 * k] = low_bf16(raw.w[0][k]);
      x[2 * k + 1] = high_bf16(raw.w[0][k]);
    }
  }
}
// The same as fp32; what lies behind V is 0.
template <int ES>
__device__ __forceinline__ void load(const void* row, int64_t v, int64_t V, float (&x)[kVec]) {
  if (v + kVec <= V) {
    unpack<ES>(load_raw<ES>(row, v), x);
  } else {
#pragma unroll
    for (int k = 0; k < kVec; ++k) x[k] = v + k < V ? element<ES>(row, v + k) : 0.f;
  }
}
// The greatest of the values' bits: 0x7F800000 or more where one is no probability (or -0).
__device__ __forceinline__ uint32_t greatest_bits(uint32_t top, const float (&x)[kVec]) {
#pragma unroll
  for (int k = 0; k < kVec; ++k) {
    const uint32_t y = __float_as_uint(x[k]);
    top = top > y ? top : y;
  }
  return top;
}

// What the workgroups of a request tell one another, all zero between calls. Words are stored and loaded
// one by one, in no order; a reader takes them when the last one fits the others.
struct VerifyTalk {
  uint64_t pass[3];                    // the first one's: M's bits, the pass, both mixed
  uint64_t left;                       // workgroups that are done
  struct { uint64_t sum, mixed; } part[kParts];
};
__device__ __forceinline__ void tell(uint64_t* at, uint64_t x) {
  __hip_atomic_store(at, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t told(const uint64_t* at) {
  return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// Bits that two passes, or two parts of one, share by chance alone; never 0.
__device__ __forceinline__ uint64_t mark(uint64_t x) {
  x = (x + 1) * 0x9E3779B97F4A7C15ull;
  x = (x ^ (x >> 29)) * 0xBF58476D1CE4E5B9ull;
  return (x ^ (x >> 32)) | 1;
}
// A pass: its number in the call, whether drafted tokens are taken out, the node.
constexpr uint64_t kOver = 0x3FFFFFFF;
__device__ __forceinline__ uint64_t pass_of(uint32_t number, bool gone, uint32_t node) {
  return (uint64_t)number << 32 | (uint64_t)gone << 31 | node;
}

struct VerifyShared {
  double part[kParts];                 // sums of the parts of the row
  double waves[kParts][kWaves];        // and of the waves' shares of them
  uint64_t missing, pass, M;
  double sub[kWaves];                  // and of their steps
  int64_t hit[kWaves], any[kWaves];
  int64_t gone[CM_DRAFT_MAX_NODES];    // tokens taken out of r
  int64_t drafts[CM_DRAFT_MAX_NODES];  // the request's nodes
  int32_t parents[CM_DRAFT_MAX_NODES];
  float accept[CM_DRAFT_MAX_NODES];
  float p[CM_DRAFT_MAX_NODES], q[CM_DRAFT_MAX_NODES];  // their tokens' in the rows of their parents
  int32_t n_gone;
};

// The first n workgroups take a request each; of the others every n-th helps one: it sums its parts of the
// row in the passes that it is told of. A part's sum is the same whoever makes it.
template <int ES>
__global__ __launch_bounds__(kThreads, kGroups * kWaves / 4) void verify_kernel(VerifyArgs a) {
  __shared__ VerifyShared lds;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int req = blockIdx.x % a.n, mine = blockIdx.x / a.n;
  const int64_t first = a.rows[req], next = a.rows[req + 1];
  const bool fits = first >= 0 && next >= first && next <= a.n_rows;
  const int c = fits && next - first <= CM_DRAFT_MAX_NODES ? (int)(next - first) : 0;
  if (c == 0) {
    if (mine > 0) return;
    if (threadIdx.x == 0) {
      a.counts[req] = 0;
      a.tokens[req] = -1;
    }
    if (fits)
      for (int64_t i = first + threadIdx.x; i < next; i += kThreads) a.path[i] = -1;
    return;
  }
  VerifyTalk* talk = static_cast<VerifyTalk*>(a.talk) + req;
  // (what the walk looks at, at once: a look-up in memory for each node on its way took as long as a pass)
  for (int i = threadIdx.x; i < c; i += kThreads) {
    const int64_t t = a.drafts[first + i];
    const int32_t of = a.parents[first + i];
    const bool in = of >= 0 && of < i && t >= 0 && t < a.V;
    lds.drafts[i] = t;
    lds.parents[i] = of;
    lds.accept[i] = a.accept[first + i];
    lds.p[i] = in ? element<ES>(static_cast<const uint8_t*>(a.p) + (first + of) * a.p_row * ES, t) : 0.f;
    lds.q[i] = in && a.q ? element<ES>(static_cast<const uint8_t*>(a.q) + (first + of) * a.q_row * ES, t) : 0.f;
  }
  if (threadIdx.x == 0) lds.n_gone = 0;
  __syncthreads();
  const int32_t* parents = lds.parents;
  const int64_t* drafts = lds.drafts;
  const float* accept = lds.accept;
  int32_t* path = a.path + first;

  // The next child of node `of` after node `after`, c where there is none. (All waves look.)
  const auto child = [&](int of, int after) {
    for (int i0 = after + 1; i0 < c; i0 += 64) {
      const int i = i0 + lane;
      const uint64_t hit = __ballot(i < c && parents[i] == of);
      if (hit) return i0 + __builtin_ctzll(hit);
    }
    return c;
  };
  // Whether one of the children of `of` up to node `end` has token t.
  const auto tried = [&](int of, int end, int64_t t) {
    for (int i0 = of + 1; i0 < end; i0 += 64) {
      const int i = i0 + lane;
      if (__any(i < end && parents[i] == of && drafts[i] == t)) return true;
    }
    return false;
  };

  int node = 0, count = 0;
  const uint8_t *p = nullptr, *q = nullptr;
  const int64_t V = a.V;
  const bool sampled = a.q != nullptr;
  // parts of the row, and a wave's share of one: whole steps
  const int64_t part = (V + kParts * kPart - 1) / (kParts * kPart) * kPart, share = part / kWaves;
  const int parts = (int)((V + part - 1) / part);

  // r of kVec elements, from v on, with the probabilities x and y
  const auto rest_of = [&](float (&x)[kVec], float (&y)[kVec], int64_t v, double M, double (&r)[kVec]) {
    uint32_t top = greatest_bits(0, x);
    if (sampled) top = greatest_bits(top, y);
    if (__builtin_expect(__any(top >= 0x7F800000u), 0)) {
#pragma unroll
      for (int k = 0; k < kVec; ++k) {
        x[k] = (float)clean(x[k]);
        if (sampled) y[k] = (float)clean(y[k]);
      }
    }
    if (sampled) {
#pragma unroll
      for (int k = 0; k < kVec; ++k) r[k] = fmax(fma(-M, (double)y[k], (double)x[k]), 0.0);
    } else {
#pragma unroll
      for (int k = 0; k < kVec; ++k) r[k] = x[k];
      const int gone = lds.n_gone;
      for (int i = 0; i < gone; ++i) {
        const int64_t t = lds.gone[i] - v;
#pragma unroll
        for (int k = 0; k < kVec; ++k) r[k] = t == k ? 0.0 : r[k];
      }
    }
  };
  const auto rest = [&](int64_t v, double M, double (&r)[kVec]) {
    float x[kVec], y[kVec];
    load<ES>(p, v, V, x);
    if (sampled) load<ES>(q, v, V, y);
    rest_of(x, y, v, M, r);
  };
  const auto sum_of = [](const double (&r)[kVec]) {
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < kVec; ++k) s += r[k];
    return s;
  };
  const auto wave_sum = [&](double x) {
#pragma unroll
    for (int by = 1; by < 64; by <<= 1) x += __shfl_xor(x, by);
    return x;
  };
  // sums of the wave's shares of parts from, from + step, ..
  const auto sum_parts = [&](int from, int step, double M) {
    for (int i = from; i < parts; i += step) {
      double s = 0.0;
      const int64_t begin = i * part + wave * share, end = begin + share < V ? begin + share : V;
      int64_t v0 = begin;
      for (; v0 + 2 * kStep <= end; v0 += 2 * kStep) {
        Raw<ES> x[2], y[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          x[b] = load_raw<ES>(p, v0 + b * kStep + lane * kVec);
          if (sampled) y[b] = load_raw<ES>(q, v0 + b * kStep + lane * kVec);
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          float xs[kVec], ys[kVec];
          double r[kVec];
          unpack<ES>(x[b], xs);
          if (sampled) unpack<ES>(y[b], ys);
          rest_of(xs, ys, v0 + b * kStep + lane * kVec, M, r);
          s += sum_of(r);
        }
      }
      for (int64_t v = v0 + lane * kVec; v < end; v += kStep) {
        double r[kVec];
        rest(v, M, r);
        s += sum_of(r);
      }
      s = wave_sum(s);
      if (lane == 0) lds.waves[i][wave] = s;
    }
  };
  // The sum of part i, from its waves' (behind a barrier).
  const auto part_sum = [&](int i) {
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s += lds.waves[i][w];
    return s;
  };
  // The tokens that children of node `of` drafted, taken out of r.
  const auto take_out = [&](int of) {
    __syncthreads();
    if (threadIdx.x == 0) lds.n_gone = 0;
    __syncthreads();
    for (int i = of + 1 + (int)threadIdx.x; i < c; i += kThreads)
      if (parents[i] == of) lds.gone[atomicAdd(&lds.n_gone, 1)] = drafts[i];
    __syncthreads();
  };
  // Done with the request's talk: the last one clears it.
  const auto leave = [&] {
    if (threadIdx.x != 0) return;
    if (__hip_atomic_fetch_add(&talk->left, 1ull, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) !=
        (uint64_t)a.groups - 1)
      return;
    for (int i = 0; i < 3; ++i) tell(&talk->pass[i], 0);
    for (int i = 0; i < parts; ++i) {
      tell(&talk->part[i].sum, 0);
      tell(&talk->part[i].mixed, 0);
    }
    tell(&talk->left, 0);
  };

  if (mine > 0) {
    uint32_t done = 0;
    while (true) {
      if (threadIdx.x == 0) {
        const uint64_t start = wall_clock64(), wait = a.helper_wait * (uint64_t)(part / kPart);
        uint64_t M = 0, pass = kOver;
        for (uint64_t now = start; now - start < wait; now = wall_clock64()) {
          M = told(&talk->pass[0]);
          pass = told(&talk->pass[1]);
          const bool whole = told(&talk->pass[2]) == (M ^ mark(pass));
          if (whole && (uint32_t)(pass >> 32) > done) break;
          pass = kOver;
          __builtin_amdgcn_s_sleep(1);
        }
        lds.M = M;
        lds.pass = pass;
      }
      __syncthreads();
      const uint64_t pass = lds.pass;
      const double M = __longlong_as_double((long long)lds.M);
      const uint32_t node = (uint32_t)pass & 0x7FFFFFFFu;
      if (node >= (uint32_t)c) break;            // (kOver)
      done = (uint32_t)(pass >> 32);
      p = static_cast<const uint8_t*>(a.p) + (first + node) * a.p_row * ES;
      if (sampled) q = static_cast<const uint8_t*>(a.q) + (first + node) * a.q_row * ES;
      if ((pass >> 31) & 1) take_out((int)node);
      else if (threadIdx.x == 0) lds.n_gone = 0;
      __syncthreads();
      sum_parts(mine, a.groups, M);
      __syncthreads();
      if (threadIdx.x == 0)
        for (int i = mine; i < parts; i += a.groups) {
          const uint64_t x = (uint64_t)__double_as_longlong(part_sum(i));
          tell(&talk->part[i].sum, x);
          tell(&talk->part[i].mixed, x ^ mark(pass * kParts + i));
        }
    }
    leave();
    return;
  }

  // sum r over the row of `node`; the parts' sums stay in lds.part
  uint32_t passes = 0;
  int helpers = a.groups;
  const auto tell_pass = [&](double M, uint64_t pass) {
    if (threadIdx.x != 0) return;
    const uint64_t x = (uint64_t)__double_as_longlong(M);
    tell(&talk->pass[0], x);
    tell(&talk->pass[1], pass);
    tell(&talk->pass[2], x ^ mark(pass));
  };
  const auto total = [&](double M) {
    const uint64_t pass = pass_of(++passes, !sampled && lds.n_gone > 0, (uint32_t)node);
    __syncthreads();                             // (the sums before are not needed now)
    if (helpers > 1) tell_pass(M, pass);
    sum_parts(0, helpers, M);
    __syncthreads();
    for (int i = (int)threadIdx.x * helpers; i < parts; i += kThreads * helpers) lds.part[i] = part_sum(i);
    if (helpers > 1) {
      if (wave == 0) {
        const uint64_t start = wall_clock64(), wait = a.sums_wait * (uint64_t)(part / kPart);
        bool wants = lane < parts && lane % helpers != 0;
        for (uint64_t now = start; now - start < wait; now = wall_clock64()) {
          if (wants) {
            const uint64_t x = told(&talk->part[lane].sum);
            if (told(&talk->part[lane].mixed) == (x ^ mark(pass * kParts + lane))) {
              lds.part[lane] = __longlong_as_double((long long)x);
              wants = false;
            }
          }
          if (!__any(wants)) break;
        }
        const uint64_t missing = __ballot(wants);
        if (lane == 0) lds.missing = missing;
      }
      __syncthreads();
      const uint64_t missing = lds.missing;
      if (missing) {                             // (none of them is waited for again)
        helpers = 1;
        for (int i = 0; i < parts; ++i)
          if ((missing >> i) & 1) sum_parts(i, kParts, M);
        __syncthreads();
        for (int i = threadIdx.x; i < parts; i += kThreads)
          if ((missing >> i) & 1) lds.part[i] = part_sum(i);
      }
    }
    __syncthreads();
    double all = 0.0;
    for (int i = 0; i < parts; ++i) all += lds.part[i];
    return all;
  };

  double M = 0.0, m = 1.0;
  while (true) {
    if (threadIdx.x == 0) path[count] = node;
    ++count;
    p = static_cast<const uint8_t*>(a.p) + (first + node) * a.p_row * ES;
    if (sampled) q = static_cast<const uint8_t*>(a.q) + (first + node) * a.q_row * ES;
    M = 0.0;
    m = 1.0;
    int x = child(node, node);
    for (; x < c; x = child(node, x)) {
      const double pt = clean(lds.p[x]), u = accept[x];
      double r, want = u;
      if (sampled) {
        const double qt = clean(lds.q[x]);
        r = fmax(fma(-M, qt, pt), 0.0);
        want *= qt;
      } else {
        r = tried(node, x, drafts[x]) ? 0.0 : pt;
      }
      if (want * m < r) break;
      if (sampled) {
        M += m;
        if (child(node, x) < c) m = total(M);    // (else the sum is made below)
      } else {
        m -= r;
      }
    }
    if (x == c) break;
    node = x;
  }
  for (int i = count + (int)threadIdx.x; i < c; i += kThreads) path[i] = -1;

  // the token after `node`
  if (!sampled) take_out(node);
  double all = total(M);
  if (!(all > 0.0)) {                            // nothing is left: as if no child had been tried
    M = 0.0;
    __syncthreads();
    if (threadIdx.x == 0) lds.n_gone = 0;
    __syncthreads();
    all = total(M);
  }
  if (a.groups > 1) {
    tell_pass(0.0, pass_of(passes + 1, false, (uint32_t)kOver));
    leave();
  }
  const double want = (double)a.sample[req] * all;
  // the first part that passes it, else the last that holds anything
  int w0 = -1;
  double before = 0.0, run = 0.0, before_last = 0.0;
  int last = 0;
  for (int w = 0; w < parts; ++w) {
    if (lds.part[w] > 0.0) {
      last = w;
      before_last = run;
    }
    if (w0 < 0 && run + lds.part[w] > want) {
      w0 = w;
      before = run;
    }
    run += lds.part[w];
  }
  if (w0 < 0) {
    w0 = last;
    before = before_last;
  }
  // that part's steps, in order: each wave's sum of one step at a time
  const int64_t begin = w0 * part, end = begin + part < V ? begin + part : V;
  __syncthreads();
  int64_t found = -1, final_one = -1;            // the token; the last one so far that has any
  for (int64_t v0 = begin; v0 < end && found < 0; v0 += (int64_t)kWaves * kStep) {
    const int64_t v = v0 + wave * kStep + lane * kVec;
    double r[kVec];
    if (v < end) rest(v, M, r);
    else {
#pragma unroll
      for (int k = 0; k < kVec; ++k) r[k] = 0.0;
    }
    const double mine = sum_of(r);
    double upto = mine;
#pragma unroll
    for (int by = 1; by < 64; by <<= 1) {
      const double o = __shfl_up(upto, by);
      if (lane >= by) upto += o;
    }
    if (lane == 63) lds.sub[wave] = upto;
    __syncthreads();
    double at = before;
    for (int w = 0; w < wave; ++w) at += lds.sub[w];
    at += upto - mine;
    // the lane's first element that passes, and its last that has any
    int hit = -1, any = -1;
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      at += r[k];
      if (r[k] > 0.0) any = k;
      if (hit < 0 && r[k] > 0.0 && at > want) hit = k;
    }
    // the first lane of the first wave: through the LDS
    const uint64_t hits = __ballot(hit >= 0), anys = __ballot(any >= 0);
    if (lane == 0) {
      lds.hit[wave] = -1;
      lds.any[wave] = -1;
    }
    if (hits && lane == __builtin_ctzll(hits)) lds.hit[wave] = v + hit;
    if (anys && lane == 63 - __builtin_clzll(anys)) lds.any[wave] = v + any;
    __syncthreads();
    for (int w = kWaves - 1; w >= 0; --w)
      if (lds.hit[w] >= 0) found = lds.hit[w];
    for (int w = 0; w < kWaves; ++w) {
      if (lds.any[w] >= 0) final_one = lds.any[w];
      before += lds.sub[w];
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    a.counts[req] = count;
    a.tokens[req] = found >= 0 ? found : final_one;
  }
}

}  // namespace

// Workgroups of a request: as many as run together, none without a part of the row, where the row has four parts
// and eight or more run together. (Trees of 16 over 200000 tokens, bf16: one request 35.5 us alone, 14.9
// shared, 32 of them 91 and 36; 32 over 32768 tokens 23.7 and 20.7, over 16384 17.5 and 20.1; with four
// workgroups each, 128 requests over 32768 tokens 19.7 and 23.4, over 50000 27.1 and 29.3.)
int32_t verify_groups(int32_t n, int64_t V) {
  const int64_t part = (V + kParts * kPart - 1) / (kParts * kPart) * kPart, parts = (V + part - 1) / part;
  const int64_t groups = (int64_t)kGroups * device_cu_count() / n;
  return (int32_t)(groups < 8 || parts < 4 ? 1 : groups > parts ? parts : groups);
}
size_t verify_workspace(int32_t n, int64_t V) {
  return verify_groups(n, V) > 1 ? sizeof(VerifyTalk) * (size_t)n : 0;
}

uint64_t verify_waits[2] = {100000, 3000};

hipError_t launch_verify_drafts(VerifyArgs a, int32_t dtype, hipStream_t stream) {
  a.helper_wait = verify_waits[0];
  a.sums_wait = verify_waits[1];
  a.groups = a.talk ? verify_groups(a.n, a.V) : 1;
  const dim3 grid((uint32_t)(a.n * a.groups));
  ScopedTiming tm(K_VERIFY_DRAFTS, stream);
  if (dtype == CM_BF16)
    hipLaunchKernelGGL(verify_kernel<2>, grid, dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(verify_kernel<4>, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace cm
