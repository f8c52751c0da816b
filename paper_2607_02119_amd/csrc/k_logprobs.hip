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
//
// 1024 vectors of 151936 bf16 logits with the first alternative: 63 us, 4.9 TB/s; the vector
// units are busy all the time, at 13 instructions a logit.  Parts of 4096 logits took 78.
// Small calls are a launch and one chain of loads: 64 rows of 8 x 4096 fp32 logits 4.0 us,
// with the first alternative 4.4, with 5 7.2, with 32 9.7.
#include "gemm_common.h"

#include "logprobs.h"

namespace mcd {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
// The maximum from which differences are taken first.  Up to here its product with log2 e is
// rounded by 2^-8 at most; the rounding grows with the product, 128 powers of two (more than
// fp32 holds, to be taken out again) from 2^31 on.
constexpr float kLargeLogit = 0x1p16f;

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

// Over the 64 lanes, on the vector units: within rows of 16 lanes by rotation, across them
// by swaps.
template <int CTRL>
__device__ __forceinline__ uint32_t row_move(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false);
}
template <class F>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t x, F &&f) {
  x = f(x, row_move<0x128>(x));                      // row_ror 8, 4, 2, 1
  x = f(x, row_move<0x124>(x));
  x = f(x, row_move<0x122>(x));
  x = f(x, row_move<0x121>(x));
  const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = f(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return f(b[0], b[1]);
}
__device__ __forceinline__ float wave_max(float x) {
  return __uint_as_float(wave_reduce(__float_as_uint(x), [](uint32_t a, uint32_t b)
                                         __attribute__((always_inline)) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }));
}
__device__ __forceinline__ float wave_sum(float x) {
  return __uint_as_float(wave_reduce(__float_as_uint(x), [](uint32_t a, uint32_t b)
                                         __attribute__((always_inline)) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}
__device__ __forceinline__ uint32_t wave_min(uint32_t x) {
  return wave_reduce(x, [](uint32_t a, uint32_t b) __attribute__((always_inline)) {
    return min(a, b);
  });
}

// x of the lane whose number differs in bit D alone, on the vector units.
template <int D>
__device__ __forceinline__ uint32_t lane_xor(uint32_t x) {
  const bool upper = threadIdx.x & D;
  if constexpr (D == 1) return row_move<0xB1>(x);    // quad_perm 1 0 3 2
  if constexpr (D == 2) return row_move<0x4E>(x);    // quad_perm 2 3 0 1
  if constexpr (D == 4) {                            // row_shl 4 and row_shr 4, by fours of lanes
    const int down = __builtin_amdgcn_update_dpp((int)x, (int)x, 0x104, 0xF, 0x5, false);
    return (uint32_t)__builtin_amdgcn_update_dpp(down, (int)x, 0x114, 0xF, 0xA, false);
  }
  if constexpr (D == 8) return row_move<0x128>(x);   // row_ror 8
  if constexpr (D == 16) {
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return upper ? a[0] : a[1];
  }
  if constexpr (D == 32) {
    const auto a = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return upper ? a[0] : a[1];
  }
}

// The wave's LDS accesses so far are done before those that follow (of the same wave).
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

constexpr int kRoom = 128;                           // candidates that a wave sorts

__device__ __forceinline__ uint64_t key_of(const Entry &e) {
  return (uint64_t)e.order << 32 | ~e.id;            // larger: before
}
__device__ __forceinline__ Entry entry_of(uint64_t key) {
  return Entry{(uint32_t)(key >> 32), ~(uint32_t)key};
}

// The lanes' keys in descending order, in blocks of N lanes (the first of them: other blocks the
// other way in turn).
template <int SIZE, int D>
__device__ __forceinline__ void exchange(uint64_t &key) {
  const int lane = threadIdx.x & 63;
  const uint64_t other = (uint64_t)lane_xor<D>((uint32_t)(key >> 32)) << 32 |
                         lane_xor<D>((uint32_t)key);
  // the larger to the lower lane, the other way in every second block
  const bool larger = ((lane & D) == 0) == ((lane & SIZE) == 0);
  key = (other > key) == larger ? other : key;
  if constexpr (D > 1) exchange<SIZE, D / 2>(key);
}
template <int N, int SIZE = 2>
__device__ __forceinline__ uint64_t sort_lanes(uint64_t key) {
  exchange<SIZE, SIZE / 2>(key);
  if constexpr (SIZE < N) return sort_lanes<N, 2 * SIZE>(key);
  return key;
}

// The first T of `count` (at most kRoom) entries of LDS into list, in order: sorted by the lanes,
// in 10 or 21 exchanges; of more than 64 the first 32 of each half are merged in 6 more.
// (Comparing 24 to 44 entries each with all took 1.5 to 3 us.)
__device__ __forceinline__ void sort_entries(const Entry *room, int count, int T, Entry *list) {
  static_assert(kRoom == 128 && kMostTop <= 32, "two halves");
  const int lane = threadIdx.x & 63;
  uint64_t key = lane < count ? key_of(room[lane]) : 0;
  if (count <= 16) key = sort_lanes<16>(key);
  else key = sort_lanes<64>(key);
  if (count > 64) {
    const uint64_t more =
        sort_lanes<64>(64 + lane < count ? key_of(room[64 + lane]) : 0);
    const uint64_t turned = __shfl((unsigned long long)more, 63 - lane);
    key = lane < 32 ? key : turned;                  // down, then up
    exchange<64, 32>(key);
  }
  if (lane < T && lane < count) list[lane] = entry_of(key);
}

// The first T of four sorted lists of T entries, kMostTop apart, into `to` (apart from them), by
// a wave: an entry's place is its own in its list and, for each other list, how many there
// come before it.
__device__ __forceinline__ void merge_lists(const Entry *lists, int T, Entry *to) {
  const int step = 1 << (31 - __clz(T));
  for (int i = threadIdx.x & 63; i < 4 * T; i += 64) {
    const int mine = i / T;
    const Entry e = lists[mine * kMostTop + i % T];
    int n[3] = {0, 0, 0};                            // of the others', before e
    for (int d = step; d > 0; d >>= 1) {
#pragma unroll
      for (int w = 0; w < 3; ++w) {
        const Entry o = lists[((mine + 1 + w) & 3) * kMostTop + min(n[w] + d, T) - 1];
        if ((n[w] + d <= T) & before(o, e)) n[w] += d;
      }
    }
    const int rank = i % T + n[0] + n[1] + n[2];
    // (entries that are none are before no other, and equal: any of them may stay)
    if (rank < T) to[rank] = e;
  }
}

// The T (2..kMostTop) first of the wave's logits x[i] with ids id(i) (i < E, every lane's own)
// into list[0..T), {0, ~0} past the last; -infinity and NaN are none.  room: kRoom entries of
// LDS of the wave's own.
//
// T lanes hold a largest logit of at least `least`, so the T first are among the logits
// from `least` on.  It is found bit by bit from the lanes' largest, until little more than T
// lanes are left or 16 bits are known; where more than kRoom logits lie there the other
// bits follow, and where ties leave more even so, the first are taken one by one.
template <int E, class Id>
__device__ __forceinline__ void wave_top(const float (&x)[E], Id &&id, int T, Entry *room,
                                         Entry *list) {
  const int lane = threadIdx.x & 63;
  float most = x[0];
#pragma unroll
  for (int i = 1; i < E; ++i) most = fmaxf(most, x[i]);
  const uint32_t mine = order_of(most);
  // the bits that all of the lanes' largest have in common are its too
  const uint32_t low = wave_min(mine), differ = low ^ ~wave_min(~mine);
  const int bits = 32 - __clz((int)differ);
  uint32_t least = differ ? low >> (bits - 1) >> 1 << (bits - 1) << 1 : low;
  // (of more lanes there would soon be more than the 64 candidates that are sorted at once)
  const int enough = T + (T < 8 ? 2 : 0);
  int count = 0, next = bits - 1;
#pragma unroll 1
  for (int half = 0; half < 2; ++half) {
    for (const int end = half ? 0 : max(bits - 16, 0); next >= end; --next) {
      const uint32_t more = least | 1u << next;
      const int lanes = __popcll(__ballot(mine >= more));
      if (lanes >= T) least = more;
      if (lanes >= T && lanes <= enough && !half) break;
    }
    const float from = logit_of(max(least, kMaskedOrder + 1));
    count = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const bool in = x[i] >= from;
      const uint64_t all = __ballot(in);
      if (!all) continue;
      const int at = count + (int)__popcll(all & ((1ull << lane) - 1));
      if (in && at < kRoom) room[at] = Entry{order_of(x[i]), id(i)};
      count += (int)__popcll(all);
    }
    if (count <= kRoom) break;
  }
  if (lane < T) list[lane] = Entry{0u, ~0u};
  wave_lds_sync();
  if (count == 0) {
  } else if (count <= kRoom) {
    sort_entries(room, count, T, list);
  } else {
    Entry last = {~0u, 0u};
    for (int n = 0; n < T; ++n) {
      Entry best = {0u, ~0u};
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const Entry e = {order_of(x[i]), id(i)};
        // (count > kRoom >= T: there is one every time)
        if (e.order > kMaskedOrder && (n == 0 || before(last, e)) && before(e, best)) best = e;
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

// A vector's token and its logit, loaded before the sums are known.
struct Given {
  int token;
  float logit;
  bool has;                    // a row of tokens that is there
};
template <bool BF16>
__device__ __forceinline__ Given given_of(const LogprobView &lv, const Vector &x) {
  Given g;
  const int row = lv.token_row ? lv.token_row[x.row] : x.row;
  g.has = row >= 0 && row < lv.token_rows;
  g.token = g.has ? lv.tokens[(int64_t)row * lv.K + x.k] : 0;
  g.logit = Group<BF16>::one(lv.logits, x.at + min(max(g.token, 0), x.V - 1));
  return g;
}

// A vector's results, by a wave: from m, S, U and its first T entries.
__device__ __forceinline__ void write_vector(const LogprobView &lv, const Vector &x,
                                             const Given &g, float m, float S, float U,
                                             const Entry *list) {
  const int lane = threadIdx.x & 63;
  const int64_t out = (int64_t)x.row * lv.K + x.k;
  // no distribution: a NaN, infinity or nothing but -infinity among the logits
  const bool none = S != S || m == INFINITY || m == -INFINITY;
  const float nan = __builtin_nanf(""), log_sum = log1pf(S);
  if (lane == 0) {
    float lp = none ? nan : (g.logit - m) - log_sum;
    if (g.has && g.token == lv.pad_id) {
      lp = 0.0f;                                     // no choice: certain
    } else if (!g.has || g.token < 0 || g.token >= x.V) {
      lp = nan;
      atomicOr(lv.status, (uint32_t)MCD_DEV_BAD_TOKEN);
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

enum { kNoTop, kFirst, kTop };   // alternatives: none, the first alone, more

// WAVES waves to a part of E * 64 WAVES logits of a vector.
//
// Exponents are y = x log2 e - m', m' = m log2 e rounded to fp32: one operation for a logit,
// whose error is y's own rounding and a shift that all share.  The shift, m' less what it
// stands for, is known (fma), and taken out of S and U at the end.  Of maxima beyond kLargeLogit
// y = (x - m) log2 e, an operation more.
template <bool BF16, int WAVES, int E, int TOP>
__global__ __launch_bounds__(256) void part_kernel(LogprobView lv) {
  typedef Group<BF16> G;
  constexpr int PART = 64 * WAVES * E;
  __shared__ Entry room[TOP == kTop ? 4 * kRoom : 1], list[TOP ? 4 * kMostTop : 1];
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
  Given given = {};
  if (first + PART <= v.V) {                         // (uniform) all there
    typename G::raw raw[E / G::N];
#pragma unroll
    for (int i = 0; i < E / G::N; ++i)
      raw[i] = *reinterpret_cast<const typename G::raw *>(base +
                                                          (int64_t)id(i * G::N) * (BF16 ? 2 : 4));
    if (lv.parts == 1 && (WAVES == 1 || wave == 0)) given = given_of<BF16>(lv, v);
#pragma unroll
    for (int i = 0; i < E / G::N; ++i) G::get(raw[i], x + i * G::N);
  } else {
    if (lv.parts == 1 && (WAVES == 1 || wave == 0)) given = given_of<BF16>(lv, v);
    // the group across the end, the same for all lanes
    const int end = v.V / G::N * G::N;
    float rest[G::N];
#pragma unroll
    for (int j = 0; j < G::N; ++j) rest[j] = end + j < v.V ? G::one(base, end + j) : -INFINITY;
#pragma unroll
    for (int i = 0; i < E / G::N; ++i) {
      const int at = (int)id(i * G::N);
      float y[G::N];
#pragma unroll
      for (int j = 0; j < G::N; ++j) y[j] = at == end ? rest[j] : -INFINITY;
      if (at < end)
        G::get(*reinterpret_cast<const typename G::raw *>(base + (int64_t)at * (BF16 ? 2 : 4)), y);
#pragma unroll
      for (int j = 0; j < G::N; ++j) x[i * G::N + j] = y[j];
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
    const bool large = fabsf(m) > kLargeLogit;
    const float top = large ? 0.0f : __fmul_rn(m, kLog2e), shift = large ? m : 0.0f;
    const float gap = large ? 0.0f : fmaf(m, kLog2e, -top);   // what top falls short of m log2 e by
    int ones = 0;
    auto sums = [&](auto at_m, auto far) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float z = decltype(far)::value ? x[i] - shift : x[i];
        const float y = fmaf(z, kLog2e, -top);
        float e = __builtin_amdgcn_exp2f(y);
        if constexpr (decltype(at_m)::value) {       // 1 for every logit of m's size, counted
          const bool is = x[i] == m;
          ones += (int)__popcll(__ballot(is));
          e = is ? 0.0f : e;
        }
        S += e;
        // (e is 0 from there on, and 0 times infinity is not)
        U = fmaf(e, fmaxf(y, -300.0f), U);
      }
    };
    const std::integral_constant<bool, true> yes{};
    const std::integral_constant<bool, false> no{};
    if (large) sums(yes, yes);
    else if (wave_m == m) sums(yes, no);
    else sums(no, no);
    S = wave_sum(S);
    U = wave_sum(U);
    // 2^y = 2^(true exponent + gap): both sums carry 2^gap
    const float f = __builtin_amdgcn_exp2f(-gap);
    U = (gap * S - U) * f * 0.6931471805599453f;
    S = S * f + (float)max(ones - 1, 0);
    // m of other waves too: their ones are not the vector's first
    if constexpr (WAVES > 1) {
      bool earlier = false;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) earlier |= w < wave && sh_m[w] == m;
      if (ones && earlier) S += 1.0f;
    }
  }
  if constexpr (TOP == kTop)
    wave_top<E>(x, id, lv.T, room + wave * kRoom, list + wave * kMostTop);
  if constexpr (TOP == kFirst) {
    uint32_t at = ~0u;
    if (wave_m == m && m > -INFINITY) {
#pragma unroll
      for (int i = E - 1; i >= 0; --i) at = x[i] == m ? id(i) : at;
      at = wave_min(at);
    }
    if (lane == 0) list[wave * kMostTop] = Entry{at == ~0u ? 0u : order_of(m), at};
    if constexpr (WAVES == 1) wave_lds_sync();
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
    if constexpr (TOP == kFirst) {
      Entry best = list[0];
#pragma unroll
      for (int w = 1; w < WAVES; ++w)
        if (before(list[w * kMostTop], best)) best = list[w * kMostTop];
      wave_lds_sync();
      if (lane == 0) list[0] = best;
      wave_lds_sync();
    }
    if constexpr (TOP == kTop) {
      if (lane < lv.T) room[lane] = Entry{0u, ~0u};
      wave_lds_sync();
      merge_lists(list, lv.T, room);
      wave_lds_sync();
    }
  }
  const Entry *mine_list = TOP == kTop && WAVES > 1 ? room
                                                    : list + (TOP && WAVES == 1 ? wave * kMostTop : 0);
  if (lv.parts == 1) {
    write_vector(lv, v, given, m, S, U, mine_list);
    return;
  }
  if (lane == 0) lv.part_sums[item] = make_float4(m, S, U, 0.0f);
  if constexpr (TOP) {
    if (lane < lv.T)
      lv.part_top[(int64_t)item * lv.T + lane] =
          make_uint2(mine_list[lane].order, mine_list[lane].id);
  }
}

// A wave for each vector joins its parts (at most 64, one a lane).  (Joined by the last of the
// vector's workgroups in the first launch, 24 vectors took 20 us without alternatives
// instead of 6.3: the fences between the parts and their count write the caches back.)
// E: entries of the alternatives a lane.
template <bool BF16, int TOP, int E = 1>
__global__ __launch_bounds__(256) void join_kernel(LogprobView lv) {
  __shared__ Entry rooms[TOP == kTop ? 4 * kRoom : 1], lists[4 * kMostTop];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t vec = (int64_t)blockIdx.x * 4 + wave;
  if (vec >= lv.vectors) return;
  Entry *list = lists + wave * kMostTop;
  const Vector v = vector_of(lv, (uint32_t)vec);
  const int64_t first = vec * lv.parts;
  const float4 p = lane < lv.parts ? lv.part_sums[first + lane]
                                   : make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
  const uint2 *top = lv.part_top + first * lv.T;
  const Given given = given_of<BF16>(lv, v);
  if constexpr (TOP == kFirst) {
    const uint2 e = lane < lv.parts ? top[lane] : make_uint2(0u, ~0u);
    const uint32_t most = ~wave_min(~e.x), id = wave_min(e.x == most ? e.y : ~0u);
    if (lane == 0) *list = Entry{most, id};
    wave_lds_sync();
  } else if constexpr (TOP == kTop) {
    float x[E];
    uint32_t ids[E];
    // (the parts' first entries, then their second, ...: spread over the lanes)
    const int parts = lv.parts, skip = 64 / parts, rest = 64 % parts;
    int rank = lane / parts, part = lane - rank * parts;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      uint2 e = make_uint2(0u, ~0u);
      if (rank < lv.T) e = top[part * lv.T + rank];
      x[i] = e.x > kMaskedOrder ? logit_of(e.x) : -INFINITY;
      ids[i] = e.y;
      rank += skip;
      part += rest;
      if (part >= parts) {
        part -= parts;
        ++rank;
      }
    }
    wave_top<E>(x, [&](int i) __attribute__((always_inline)) { return ids[i]; }, lv.T,
                rooms + wave * kRoom, list);
  }
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
  write_vector(lv, v, given, m, S, U, list);
}

template <bool BF16, int WAVES, int E>
void part_launch(const LogprobView &lv, hipStream_t st) {
  const int64_t items = lv.vectors * lv.parts;
  const dim3 grid((unsigned)(WAVES == 1 ? (items + 3) / 4 : items));
  if (lv.T > 1)
    hipLaunchKernelGGL((part_kernel<BF16, WAVES, E, kTop>), grid, dim3(256), 0, st, lv);
  else if (lv.T)
    hipLaunchKernelGGL((part_kernel<BF16, WAVES, E, kFirst>), grid, dim3(256), 0, st, lv);
  else
    hipLaunchKernelGGL((part_kernel<BF16, WAVES, E, kNoTop>), grid, dim3(256), 0, st, lv);
}

template <bool BF16>
void logprobs_launch(const LogprobView &lv, const LogprobPlan &p, hipStream_t st) {
  if (p.part == 1024) part_launch<BF16, 1, 16>(lv, st);
  else if (p.part == 4096) part_launch<BF16, 4, 16>(lv, st);
  else part_launch<BF16, 4, 32>(lv, st);
  if (p.parts == 1) return;
  const dim3 grid((unsigned)((lv.vectors + 3) / 4));
  const int entries = (lv.parts * lv.T + 63) / 64;   // (at most kMostTop: 64 parts)
  if (lv.T > 1 && entries <= 4)
    hipLaunchKernelGGL((join_kernel<BF16, kTop, 4>), grid, dim3(256), 0, st, lv);
  else if (lv.T > 1 && entries <= 16)
    hipLaunchKernelGGL((join_kernel<BF16, kTop, 16>), grid, dim3(256), 0, st, lv);
  else if (lv.T > 1)
    hipLaunchKernelGGL((join_kernel<BF16, kTop, kMostTop>), grid, dim3(256), 0, st, lv);
  else if (lv.T) hipLaunchKernelGGL((join_kernel<BF16, kFirst>), grid, dim3(256), 0, st, lv);
  else hipLaunchKernelGGL((join_kernel<BF16, kNoTop>), grid, dim3(256), 0, st, lv);
}

}  // namespace

LogprobPlan logprob_plan(int64_t vectors, int32_t V) {
  LogprobPlan p;
  p.part = V <= 1024 ? 1024 : 4096;
  if (V > 4096 && (vectors * ((V + 4095) / 4096) > 2048 || V > 64 * 4096)) p.part = 8192;
  p.parts = (V + p.part - 1) / p.part;
  return p;
}

int64_t logprob_groups(int64_t vectors, int32_t V) {
  const LogprobPlan p = logprob_plan(vectors, V);
  const int64_t items = vectors * p.parts;
  return p.part == 1024 ? (items + 3) / 4 : items;   // (as part_launch)
}

hipError_t launch_logprobs(const LogprobView &lv, const LogprobPlan &p, bool bf16,
                           hipStream_t st) {
  if (bf16) logprobs_launch<true>(lv, p, st);
  else logprobs_launch<false>(lv, p, st);
  return hipGetLastError();
}

}  // namespace mcd
