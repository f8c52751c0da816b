// Log probabilities (mcd.h, mcd_logprobs): of a vector x of V logits
//
//   m = max x;  S = sum over the others of e^(x - m);  U = sum of e^(x - m) (m - x)
//   log p[t] = (x[t] - m) - log1p(S);  entropy = log1p(S) + U / (1 + S)
//
// and the ids of the T largest logits, ties to the lower id.  The largest logit's own
// 1 is kept out of S: the log probability of a token that is nearly certain keeps its
// leading digits.
//
// A vector goes through once, in parts that a wave or a workgroup holds in registers:
// the part's maximum first, then its sums against it, so nothing is scaled again.
// Sums and log probabilities are in fp32.  Parts meet in a second launch, in their
// order: the same inputs give the same bits.
#include "gemm_common.h"

#include "logprobs.h"

namespace mcd {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// Logits as whole numbers in the same order, -0 and 0 alike; NaN: 0, below all.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  if (x != x) return 0u;
  return u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t order) {
  return __uint_as_float(order ^ (order >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}
constexpr uint32_t kMaskedOrder = 0x007FFFFFu;       // order_of(-infinity)

// (order, id): the larger first, ties to the lower id
struct Entry {
  uint32_t order, id;
};
__device__ __forceinline__ bool before(const Entry &a, const Entry &b) {
  return a.order > b.order || (a.order == b.order && a.id < b.id);
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

// The wave's LDS accesses so far are done before those that follow (of the same wave).
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

constexpr int kRoom = 128;                           // candidates that a wave sorts

// The T (1..kMostTop) first of the wave's entries order[i], id(i) (i < E, every lane's
// own) into list[0..T), {0, ~0} past the last; orders up to kMaskedOrder are no
// entries.  room: kRoom entries of LDS of the wave's own.
//
// T lanes hold a largest entry of at least `least`, so the T first are among the entries
// from `least` on: usually little more than T of them, which are compared each with all.
// Where ties make them more than kRoom, they are taken one by one.
template <int E, class Id>
__device__ __forceinline__ void wave_top(const uint32_t (&order)[E], Id &&id, int T, Entry *room,
                                         Entry *list) {
  const int lane = threadIdx.x & 63;
  uint32_t mine = order[0];
#pragma unroll
  for (int i = 1; i < E; ++i) mine = max(mine, order[i]);
  uint32_t least = 0;
#pragma unroll 1
  for (uint32_t bit = 1u << 31; bit; bit >>= 1)
    if (__popcll(__ballot(mine >= (least | bit))) >= T) least |= bit;
  least = max(least, kMaskedOrder + 1);
  int count = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const bool in = order[i] >= least;
    const uint64_t all = __ballot(in);
    const int at = count + __popcll(all & ((1ull << lane) - 1));
    if (in && at < kRoom) room[at] = Entry{order[i], id(i)};
    count += __popcll(all);
  }
  if (lane < T) list[lane] = Entry{0u, ~0u};
  wave_lds_sync();
  if (count <= kRoom) {
    for (int c = lane; c < count; c += 64) {
      const Entry e = room[c];
      int rank = 0;
      for (int k = 0; k < count; ++k) rank += before(room[k], e);
      if (rank < T) list[rank] = e;
    }
  } else {
    Entry last = {~0u, 0u};
    for (int n = 0; n < T; ++n) {
      Entry best = {0u, ~0u};
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const Entry e = {order[i], id(i)};
        // (count > kRoom >= T: there is one every time)
        if (e.order >= least && (n == 0 || before(last, e)) && before(e, best)) best = e;
      }
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) {
        const Entry o = {(uint32_t)__shfl_xor((int)best.order, d),
                         (uint32_t)__shfl_xor((int)best.id, d)};
        if (before(o, best)) best = o;
      }
      if (lane == 0) list[n] = best;
      last = best;
    }
  }
  wave_lds_sync();
}

// 16 bytes of logits from any element on.
template <bool BF16>
struct Group;
template <>
struct Group<false> {
  static constexpr int N = 4;
  typedef float raw __attribute__((ext_vector_type(4), aligned(4)));
  static __device__ __forceinline__ void get(raw w, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = w[i];
  }
  static __device__ __forceinline__ float one(const void *p, int64_t at) {
    return static_cast<const float *>(p)[at];
  }
};
template <>
struct Group<true> {
  static constexpr int N = 8;
  typedef uint32_t raw __attribute__((ext_vector_type(4), aligned(2)));
  static __device__ __forceinline__ void get(raw w, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ float one(const void *p, int64_t at) {
    return __uint_as_float((uint32_t)static_cast<const uint16_t *>(p)[at] << 16);
  }
};

// Where vector (row, k) begins and its ids.
struct Vector {
  int row, k, V;
  int64_t at;
};
__device__ __forceinline__ Vector vector_of(const LogprobView &lv, uint32_t v) {
  Vector x;
  x.row = (int)(v / (uint32_t)lv.K);
  x.k = (int)(v - (uint32_t)x.row * (uint32_t)lv.K);
  x.at = (int64_t)x.row * lv.stride + lv.off.o[x.k];
  x.V = lv.off.o[x.k + 1] - lv.off.o[x.k];
  return x;
}

// A vector's results, by a wave: from m, S, U and its first T entries (order of each).
template <bool BF16>
__device__ __forceinline__ void write_vector(const LogprobView &lv, const Vector &x, float m,
                                             float S, float U, const Entry *list) {
  const int lane = threadIdx.x & 63;
  const int64_t out = (int64_t)x.row * lv.K + x.k;
  // no distribution: a NaN, infinity or nothing but -infinity among the logits
  const bool none = S != S || m == INFINITY || m == -INFINITY;
  const float nan = __builtin_nanf(""), log_sum = log1pf(S);
  if (lane == 0) {
    const int row = lv.token_row ? lv.token_row[x.row] : x.row;
    const bool has = row >= 0 && row < lv.token_rows;
    const int t = has ? lv.tokens[(int64_t)row * lv.K + x.k] : 0;
    float lp;
    if (has && t == lv.pad_id) {
      lp = 0.0f;                                     // no choice: certain
    } else if (!has || t < 0 || t >= x.V) {
      lp = nan;
      atomicOr(lv.status, (uint32_t)MCD_DEV_BAD_TOKEN);
    } else {
      lp = none ? nan : (Group<BF16>::one(lv.logits, x.at + t) - m) - log_sum;
    }
    lv.logprob[out] = lp;
    if (lv.entropy) lv.entropy[out] = none ? nan : log_sum + U / (1.0f + S);
  }
  if (lane < lv.T) {
    const Entry e = list[lane];
    const bool is = !none && e.order > kMaskedOrder;
    if (lv.top_ids) lv.top_ids[out * lv.T + lane] = is ? (int)e.id : -1;
    if (lv.top_logprobs)
      lv.top_logprobs[out * lv.T + lane] =
          none ? nan : is ? (logit_of(e.order) - m) - log_sum : -INFINITY;
  }
}

// WAVES waves to a part of E * 64 WAVES logits of a vector.
template <bool BF16, int WAVES, int E, bool TOP>
__global__ __launch_bounds__(256) void part_kernel(LogprobView lv) {
  typedef Group<BF16> G;
  constexpr int PART = 64 * WAVES * E;
  __shared__ Entry room[TOP ? 4 * kRoom : 1], list[TOP ? 4 * kMostTop : 1];
  __shared__ float sh_m[4], sh_s[4], sh_u[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // (below 2^31)
  const uint32_t item = blockIdx.x * (4 / WAVES) + wave / WAVES;
  if (WAVES == 1 && item >= (uint32_t)lv.vectors * lv.parts) return;
  const uint32_t vec = item / (uint32_t)lv.parts;
  const int part = (int)(item - vec * lv.parts);
  const Vector v = vector_of(lv, vec);
  const int first = part * PART;                     // (below 2^20)
  const int tid = WAVES == 1 ? lane : threadIdx.x;

  float x[E];
  const char *base = static_cast<const char *>(lv.logits) + v.at * (BF16 ? 2 : 4);
  // id of register i
  auto id = [&](int i) __attribute__((always_inline)) {
    return (uint32_t)(first + (i / G::N * 64 * WAVES + tid) * G::N + i % G::N);
  };
  typename G::raw raw[E / G::N];
#pragma unroll
  for (int i = 0; i < E / G::N; ++i) {
    const int at = (int)id(i * G::N);
    if (at + G::N <= v.V)
      raw[i] = *reinterpret_cast<const typename G::raw *>(base + (int64_t)at * (BF16 ? 2 : 4));
  }
#pragma unroll
  for (int i = 0; i < E / G::N; ++i) {
    const int at = (int)id(i * G::N);
    if (at + G::N <= v.V) {
      G::get(raw[i], x + i * G::N);
    } else {
#pragma unroll
      for (int j = 0; j < G::N; ++j)
        x[i * G::N + j] = at + j < v.V ? G::one(base, at + j) : -INFINITY;
    }
  }
  float mine = x[0];
#pragma unroll
  for (int i = 1; i < E; ++i) mine = fmaxf(mine, x[i]);
  const float wave_m = wave_max(mine);
  float m = wave_m;
  if constexpr (WAVES > 1) {
    if (lane == 0) sh_m[wave] = wave_m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, sh_m[w]);
  }
  float S = 0.0f, U = 0.0f;
  if (m == -INFINITY) {                              // nothing, or NaN
#pragma unroll
    for (int i = 0; i < E; ++i) S += x[i] != x[i] ? x[i] : 0.0f;
    S = wave_sum(S);
  } else {
    int ones = 0;
    const bool at_m = wave_m == m;                   // (uniform)
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float d = x[i] - m;
      float e = __builtin_amdgcn_exp2f(d * kLog2e);
      if (at_m) {                                    // 1 for every logit of m's size, counted
        ones += __popcll(__ballot(d == 0.0f));
        e = d == 0.0f ? 0.0f : e;
      }
      S += e;
      // (e is 0 from there on, and 0 times infinity is not)
      U = fmaf(e, fmaxf(d, -256.0f), U);
    }
    S = wave_sum(S) + (float)max(ones - 1, 0);
    U = wave_sum(-U);
    // m of other waves too: their ones are not the vector's first
    if constexpr (WAVES > 1) {
      bool earlier = false;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) earlier |= w < wave && sh_m[w] == m;
      if (at_m && earlier && ones) S += 1.0f;
    }
  }
  if constexpr (TOP) {
    uint32_t order[E];
#pragma unroll
    for (int i = 0; i < E; ++i) order[i] = order_of(x[i]);
    wave_top<E>(order, id, lv.T, room + wave * kRoom, list + wave * kMostTop);
  }
  if constexpr (WAVES > 1) {
    if (lane == 0) {
      sh_s[wave] = S;
      sh_u[wave] = U;
    }
    __syncthreads();
    if (wave) return;
    S = U = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      S += sh_s[w];
      U += sh_u[w];
    }
    if constexpr (TOP) {
      // the waves' lists: two entries a lane
      uint32_t order[2], ids[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int at = i * 64 + lane;
        const bool in = at % kMostTop < lv.T;
        order[i] = in ? list[at].order : 0u;
        ids[i] = in ? list[at].id : ~0u;
      }
      wave_lds_sync();
      wave_top<2>(order, [&](int i) __attribute__((always_inline)) { return ids[i]; }, lv.T, room,
                  list);
    }
  }
  const Entry *mine_list = list + (TOP && WAVES == 1 ? wave * kMostTop : 0);
  if (lv.parts == 1) {
    write_vector<BF16>(lv, v, m, S, U, mine_list);
    return;
  }
  if (lane == 0) lv.part_sums[item] = make_float4(m, S, U, 0.0f);
  if constexpr (TOP) {
    if (lane < lv.T)
      lv.part_top[(int64_t)item * lv.T + lane] = make_uint2(mine_list[lane].order, mine_list[lane].id);
  }
}

// A wave for each vector joins its parts (at most 64, one a lane).
template <bool BF16>
__global__ __launch_bounds__(256) void join_kernel(LogprobView lv) {
  __shared__ Entry room[4 * kRoom], list[4 * kMostTop];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t vec = (int64_t)blockIdx.x * 4 + wave;
  if (vec >= lv.vectors) return;
  const Vector v = vector_of(lv, (uint32_t)vec);
  const float4 p = lane < lv.parts ? lv.part_sums[vec * lv.parts + lane]
                                   : make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
  const float m = wave_max(p.x);
  float S, U = 0.0f;
  if (p.x == m) {                                    // (also where all are -infinity)
    S = p.y;
    U = p.z;
  } else if (p.x == -INFINITY) {
    S = p.y;                                         // 0, or NaN
  } else {
    const float d = p.x - m, f = __builtin_amdgcn_exp2f(d * kLog2e);
    S = (1.0f + p.y) * f;
    U = (p.z - (1.0f + p.y) * fmaxf(d, -256.0f)) * f;
  }
  const int ones = __popcll(__ballot(p.x == m && lane < lv.parts));
  S = wave_sum(S) + (float)max(ones - 1, 0);
  U = wave_sum(U);
  Entry *mine_list = list + wave * kMostTop;
  if (lv.T) {
    constexpr int E = 64 * kMostTop / 64;
    uint32_t order[E], ids[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int at = i * 64 + lane;
      uint2 e = make_uint2(0u, ~0u);
      if (at < lv.parts * lv.T) e = lv.part_top[vec * lv.parts * lv.T + at];
      order[i] = e.x;
      ids[i] = e.y;
    }
    wave_top<E>(order, [&](int i) __attribute__((always_inline)) { return ids[i]; }, lv.T,
                room + wave * kRoom, mine_list);
  }
  write_vector<BF16>(lv, v, m, S, U, mine_list);
}

template <bool BF16, int WAVES, int E>
void part_launch(const LogprobView &lv, hipStream_t st) {
  const int64_t items = lv.vectors * lv.parts;
  const dim3 grid((unsigned)(WAVES == 1 ? (items + 3) / 4 : items));
  if (lv.T)
    hipLaunchKernelGGL((part_kernel<BF16, WAVES, E, true>), grid, dim3(256), 0, st, lv);
  else
    hipLaunchKernelGGL((part_kernel<BF16, WAVES, E, false>), grid, dim3(256), 0, st, lv);
}

template <bool BF16>
void logprobs_launch(const LogprobView &lv, const LogprobPlan &p, hipStream_t st) {
  if (p.part == 1024) part_launch<BF16, 1, 16>(lv, st);
  else if (p.part == 4096) part_launch<BF16, 4, 16>(lv, st);
  else part_launch<BF16, 4, 32>(lv, st);
  if (p.parts > 1)
    hipLaunchKernelGGL(join_kernel<BF16>, dim3((unsigned)((lv.vectors + 3) / 4)), dim3(256), 0, st,
                       lv);
}

}  // namespace

LogprobPlan logprob_plan(int64_t vectors, int32_t V) {
  LogprobPlan p;
  p.part = V <= 1024 ? 1024 : 4096;
  if (V > 4096 && (vectors * ((V + 4095) / 4096) > 2048 || V > 64 * 4096)) p.part = 8192;
  p.parts = (V + p.part - 1) / p.part;
  return p;
}

hipError_t launch_logprobs(const LogprobView &lv, const LogprobPlan &p, bool bf16,
                           hipStream_t st) {
  if (bf16) logprobs_launch<true>(lv, p, st);
  else logprobs_launch<false>(lv, p, st);
  return hipGetLastError();
}

}  // namespace mcd
