// Attention over the 4-bit key/value cache: a page of keys and values against tiles of
// query rows, the kernel of few query rows, and that of many for any rows that have
//   row_span(cv, rows, r)   a row's tokens and positions, and its first page to read
//   tile_row(rows, G, TQ, x, tile)  the row and tile of work item x
//   Rows::kParts            results as parts of every query row, for another kernel to join
#pragma once

#include "cache_common.h"

#include <algorithm>

namespace mcd {

// a * b, 0 when either is 0 whatever the other is (v_mul_legacy_f32)
__device__ float mul_zero(float a, float b) __asm("llvm.amdgcn.fmul.legacy");

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// 8 e2m1 codes to bfloat16, times 2^(exponent of scale): exact.
__device__ __forceinline__ bf16x8 dequant(uint32_t w, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ floatx4 mfma(bf16x8 a, bf16x8 b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// x in SPL bfloat16 terms whose sum is x to 8 SPL bits
template <int SPL>
__device__ __forceinline__ void split8(const float x[8], bf16x8 (&out)[SPL]) {
  typedef float float2v __attribute__((ext_vector_type(2)));
  float rest[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
  for (int n = 0; n < SPL; ++n) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bf16x2 two = __builtin_convertvector(float2v{rest[2 * i], rest[2 * i + 1]}, bf16x2);
      w[i] = __builtin_bit_cast(uint32_t, two);
      if (n + 1 < SPL) {
        rest[2 * i] -= __uint_as_float(w[i] << 16);
        rest[2 * i + 1] -= __uint_as_float(w[i] & 0xFFFF0000u);
      }
    }
    out[n] = __builtin_bit_cast(bf16x8, w);
  }
}

// Lane moves on the vector units: x of lane i + n / i - n of the row of 16 lanes
// (CTRL row_shl / row_shr / row_ror n), into the lanes of the banks of four of
// BANKS; the other lanes keep old.
template <int CTRL, int BANKS = 0xF>
__device__ __forceinline__ uint32_t lane_move(uint32_t old, uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)x, CTRL, 0xF, BANKS, false);
}
template <int CTRL, int BANKS = 0xF>
__device__ __forceinline__ float lane_move(float old, float x) {
  return __uint_as_float(lane_move<CTRL, BANKS>(__float_as_uint(old), __float_as_uint(x)));
}
constexpr int kSame = 0xE4;                      // quad_perm 0 1 2 3
constexpr int shl(int n) { return n == 0 ? kSame : n > 0 ? 0x100 + n : 0x110 - n; }
constexpr int ror(int n) { return 0x120 + n; }

// Over the four lanes 16 g + m of a column m.
__device__ __forceinline__ float across_groups_max(float x) {
  const uint32_t u = __float_as_uint(x);
  auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t v = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
  auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float across_groups_sum(float x) {
  const uint32_t u = __float_as_uint(x);
  auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t v = __float_as_uint(__uint_as_float(a[0]) + __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// A page's codes and scales as a wave's lanes hold them.  Lane 16 g + m has
// keys of tokens 16 t + m, channels g D / 4 onwards, and value words of channel
// slot m and tokens 16 t + 4 g + i.
template <int D>
struct PageRegs {
  uint32_t k[4][D / 32];
  uint32_t ks[D == 256 ? 2 : 1];       // byte t: exponent of token 16 t + m
  uint32_t v[2][D / 16];
  uint32_t vs[8];                      // bfloat16 4 t + i
};

// A load at a wave-uniform address plus a 32-bit lane offset: the address stays
// in scalar registers.
// ONCE: read by no other workgroup, so not kept in the caches.
template <class T, bool ONCE = false>
__device__ __forceinline__ T load_at(const uint8_t *base, uint32_t lane_at, uint32_t at) {
  const T *p = reinterpret_cast<const T *>(base + at + lane_at);
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  else return *p;
}

template <int D, bool ONCE = false>
__device__ __forceinline__ void load_keys(const uint8_t *page, uint32_t g, uint32_t m,
                                          PageRegs<D> &x) {
  const uint32_t lane_at = m * (D / 2) + g * (D / 8);
#pragma unroll
  for (uint32_t t = 0; t < 4; ++t) {
    if constexpr (D == 64) {
      const uint2 w = load_at<uint2>(page, lane_at, 16 * t * (D / 2));
      x.k[t][0] = w.x;
      x.k[t][1] = w.y;
    } else {
#pragma unroll
      for (uint32_t i = 0; i < D / 128; ++i) {
        const u32x4 w = load_at<u32x4, ONCE>(page, lane_at, 16 * t * (D / 2) + 16 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) x.k[t][4 * i + e] = w[e];
      }
    }
  }
  if constexpr (D == 64) x.ks[0] = load_at<uint32_t>(page, m * 8 + (g >> 1) * 4, 64 * D);
  else if constexpr (D == 128) x.ks[0] = load_at<uint32_t>(page, m * 16 + g * 4, 64 * D);
  else {
    const uint2 w = load_at<uint2>(page, m * 32 + g * 8, 64 * D);
    x.ks[0] = w.x;
    x.ks[1] = w.y;
  }
}

template <int D, bool SCALES = true, bool ONCE = false>
__device__ __forceinline__ void load_values(const uint8_t *page, uint32_t lane, PageRegs<D> &x) {
#pragma unroll
  for (uint32_t h = 0; h < 2; ++h)
#pragma unroll
    for (uint32_t q = 0; q < D / 64; ++q) {
      const u32x4 w =
          load_at<u32x4, ONCE>(page, lane * 16, 32 * D + (h * (D / 64) + q) * 1024);
#pragma unroll
      for (int e = 0; e < 4; ++e) x.v[h][4 * q + e] = w[e];
    }
#pragma unroll
  for (uint32_t i = 0; i < (SCALES ? 2 : 0); ++i) {
    const u32x4 w = load_at<u32x4>(page, (lane >> 4) * 32, 66 * D + 16 * i);
#pragma unroll
    for (int e = 0; e < 4; ++e) x.vs[4 * i + e] = w[e];
  }
}

// float whose exponent is key scale byte t of word w; 255, infinity: dequant
// then gives NaN for every code
__device__ __forceinline__ float key_exp(uint32_t w, int t) {
  return __uint_as_float(t == 3 ? (w >> 24) << 23 : ((w >> (8 * t)) & 0xFFu) << 23);
}

// A page's operands from its registers.
template <int D>
__device__ __forceinline__ auto keys_of(const PageRegs<D> &x) {
  return [&x](int t, int e) __attribute__((always_inline)) {
    return dequant(x.k[t][e], key_exp(x.ks[e / 4], t));
  };
}
template <int D>
__device__ __forceinline__ auto values_of(const PageRegs<D> &x) {
  return [&x](int h, int ct) __attribute__((always_inline)) { return dequant(x.v[h][ct], 1.0f); };
}

// Scores of the page's tokens 16 t + 4 g + i (i: component) against query
// column m of each of NT tiles.  k(t, e): the keys' operand of tile t for
// channels' step e; q(n, p, e): term p of the queries'.  The four tiles of tokens
// are four independent chains of matrix instructions.
template <int D, int SPL, int NT, class K, class Q>
__device__ __forceinline__ void scores(K &&k, Q &&q, floatx4 (&s)[NT][4]) {
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int t = 0; t < 4; ++t) s[n][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int e = 0; e < D / 32; ++e) {
    // (one step's operands in registers, where registers make waves)
    if constexpr (NT == 1) __builtin_amdgcn_sched_barrier(0);
    bf16x8 b[NT][SPL];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int p = 0; p < SPL; ++p) b[n][p] = q(n, p, e);
    bf16x8 a[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) a[t] = k(t, e);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int p = SPL - 1; p >= 0; --p)
#pragma unroll
        for (int t = 0; t < 4; ++t) s[n][t] = mfma(a[t], b[n][p], s[n][t]);
  }
}

// Query rows of a row's tile: (token, query head of the K/V head), token-major.
struct Query {
  int tok, head;               // of the row's tokens; of all query heads
  int limit;                   // last visible position, -1: none
  bool valid;
};

__device__ __forceinline__ Query query_of(const Span &sp, const AttendView &av, int h, int rho) {
  Query q;
  q.tok = rho / av.G;
  q.head = h * av.G + (rho - q.tok * av.G);
  q.valid = q.tok < sp.n;
  const int64_t lim = min((int64_t)sp.ctx + q.tok, (int64_t)sp.len - 1);
  q.limit = q.valid ? (int)max(lim, (int64_t)-1) : -1;
  return q;
}

// A row whose query rows of a K/V head fit one narrow tile.
__device__ __forceinline__ bool is_narrow(const Span &sp, const AttendView &av) {
  return sp.n > 0 && (int64_t)sp.n * av.G <= av.narrow;
}

// Pages seen by the query rows below end.
__device__ __forceinline__ int tile_pages(const Span &sp, int G, int end) {
  const int last = min(sp.len - 1, sp.ctx + (end - 1) / G);
  return last < 0 ? 0 : last / kPage + 1;
}

// Splits of the pages from the first on that hold any, of a tile that sees `pages`.
__device__ __forceinline__ int splits_used(const Span &sp, const AttendView &av, int pages) {
  return (max(pages - sp.page0, 0) + av.split_pages - 1) / av.split_pages;
}

// First part of a query row (Rows::kParts).
__device__ __forceinline__ int64_t part_of(const AttendView &av, int tok, int head) {
  return ((int64_t)tok * av.Hq + head) * av.parts + av.part0;
}

// (rows of which a lane's column has none: zeros)
template <int D, int SPL, int NT>
__device__ __forceinline__ void load_queries(const AttendView &av, const Span &sp,
                                             const Query (&qr)[NT], int g,
                                             bf16x8 (&q)[NT][SPL][D / 32], bool has = true) {
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int64_t at = (int64_t)(sp.t0 + qr[n].tok) * av.q_stride + qr[n].head * D + g * (D / 4);
#pragma unroll
    for (int e = 0; e < D / 32; ++e) {
      if constexpr (SPL == 1) {
        u32x4 w = {0u, 0u, 0u, 0u};
        if (qr[n].valid && has)
          w = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(av.q) + at + 8 * e);
        q[n][0][e] = __builtin_bit_cast(bf16x8, w);
      } else {
        float x[8] = {};
        if (qr[n].valid && has) {
          const float4 *p =
              reinterpret_cast<const float4 *>(static_cast<const float *>(av.q) + at + 8 * e);
          const float4 a = p[0], b = p[1];
          x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
          x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        }
        bf16x8 t[SPL];
        split8<SPL>(x, t);
#pragma unroll
        for (int p = 0; p < SPL; ++p) q[n][p][e] = t[p];
      }
    }
  }
}

// Items of a K/V head: tiles of TQ query rows, at most tokens G / TQ + 1 of a
// row, so row r's begin at start[r] G / TQ + r.  each: rows of at most a token, and
// as many tokens: every row's tiles side by side, with no search for the row.
__host__ __device__ inline bool token_each(const RowsView &rv) {
  return rv.max_tokens == 1 && rv.N == rv.R;
}
__host__ __device__ inline int64_t tile_items(int32_t R, int32_t N, int32_t G, int TQ, bool each) {
  return each ? (int64_t)R * ((G + TQ - 1) / TQ) : (int64_t)N * G / TQ + R;
}

__device__ __forceinline__ int tile_row(const RowsView &rv, int G, int TQ, int64_t x, int &tile) {
  if (token_each(rv)) {
    const int per = (G + TQ - 1) / TQ;
    tile = (int)(x % per);
    return (int)(x / per);
  }
  auto base = [&](int r) __attribute__((always_inline)) {
    return (int64_t)row_start(rv, r) * G / TQ + r;
  };
  const int r = find_row(rv.R, x, base);
  tile = (int)(x - base(r));
  return r;
}

template <bool BF16>
__device__ __forceinline__ void store4(void *p, int64_t at, const float x[4]) {
  if constexpr (BF16) {
    uint2 w;
    w.x = bf16_bits(x[0]) | bf16_bits(x[1]) << 16;
    w.y = bf16_bits(x[2]) | bf16_bits(x[3]) << 16;
    *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p) + at) = w;
  } else {
    *reinterpret_cast<float4 *>(static_cast<float *>(p) + at) =
        make_float4(x[0], x[1], x[2], x[3]);
  }
}

// The reference of a query row's softmax weights is a score, about its largest so
// far; -infinity: none seen.  The weight of score s is 2^((s - reference) c), and
// every sum is a multiple of the reference's: partial sums, the row's statistics and
// the received weight all carry the reference itself.  Below 2^20 (in powers of
// two) the product of reference and c is rounded once and stands for the
// reference everywhere, so one fused multiply-add gives an exponent; beyond,
// that rounding would be a part of the exponent that counts, or overflow it, and
// differences are taken before they are scaled.
constexpr float kLargeLogit = 0x1p20f;

// (the product as fp32 rounds it, in no fused operation)
__device__ __forceinline__ float scaled(float score, float c) {
#pragma clang fp contract(off)
  return score * c;
}

struct Origin {
  float shift, top;            // exponent of score s: fma(s - shift, c, -top)
};
__device__ __forceinline__ Origin origin_of(float ref, float c) {
  const float x = scaled(ref, c);
  const bool none = ref == -INFINITY, large = fabsf(x) >= kLargeLogit;
  return Origin{large && !none ? ref : 0.0f, large ? 0.0f : x};
}

// Exponent of what sums of reference a are multiplied with to become b's (a may
// be -infinity).  LARGE: one of the two may be large.
__device__ __forceinline__ bool is_large(float ref, float c) {
  return fabsf(scaled(ref, c)) >= kLargeLogit && ref != -INFINITY;
}
template <bool LARGE>
__device__ __forceinline__ float origin_gap_of(float a, float b, float c) {
#pragma clang fp contract(off)
  const float x = a * c, y = b * c;
  if constexpr (!LARGE) return x - y;
  const bool ax = is_large(a, c), by = is_large(b, c);
  // beside a reference below 2^20: what the large one's product was rounded by
  // (nothing that counts from 2^30 on)
  const float ra = ax && fabsf(x) < 0x1p30f ? fmaf(a, c, -x) : 0.0f;
  const float rb = by && fabsf(y) < 0x1p30f ? fmaf(b, c, -y) : 0.0f;
  return ax && by ? (a - b) * c : (x - y) + (ra - rb);
}
__device__ __forceinline__ float origin_gap(float a, float b, float c) {
  if (__any(is_large(a, c) || is_large(b, c))) return origin_gap_of<true>(a, b, c);
  return origin_gap_of<false>(a, b, c);
}

// A finished query row's reference and sum: its lse, and what weight_kernel needs
// of them.
__device__ __forceinline__ void finish_row(const AttendView &av, int64_t row, float ref, float l) {
  if (av.lse)
    av.lse[row] = l == 0.0f ? -INFINITY
                            : (scaled(ref, av.c) + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
  if (av.stats) av.stats[row] = make_float2(ref, l == 0.0f ? 0.0f : 1.0f / l);
}

// A wave's running state: for each of NT tiles of 16 query rows (column m of the
// lane) the reference of its softmax weights, the sum of its softmax weights at
// the lane's positions, and the sums of weight x value code for the lane's channels.
template <int D, int NT>
struct Running {
  float ref[NT], top[NT], sum[NT];             // top: the reference times c
  floatx4 o[NT][D / 16];
};

typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
// Value scales from 2^64 on are looked at: sums of weights of up to 2^8 might
// overflow with them though the result does not, so the reference goes kLift
// (powers of two) above the largest score where a row sees one: weights are then
// below 2^-56 and sums of 2^30 of them below 2^105.  (A reference of 2^30 and more
// does not hold the difference.)
constexpr uint32_t kLargeScale = 0x5F80u, kNanScale = 0x7F80u;   // bfloat16
constexpr float kLift = 64.0f;

// Whether one of a page's value scales (bfloat16, two to a word, no negative one
// that is visible) is at least kLargeScale.  Uniform.
template <int N, int M>
__device__ __forceinline__ bool special_scales(const uint32_t (&vs)[M]) {
  ushort2v top = __builtin_bit_cast(ushort2v, vs[0]);
#pragma unroll
  for (int i = 1; i < N; ++i)
    top = __builtin_elementwise_max(top, __builtin_bit_cast(ushort2v, vs[i]));
  constexpr unsigned short below = kLargeScale - 1;
  return __any(__builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(
                   top, ushort2v{below, below})) != 0u);
}
__device__ __forceinline__ uint32_t scale_bits(uint32_t two, int i) {
  return (i & 1 ? two >> 16 : two) & 0x7FFFu;
}

// Takes tile n's reference up to its largest score once that is 2^8 above it: sums
// stay far below fp32's range, and most pages scale nothing.
template <int D, int NT>
__device__ __forceinline__ void move_reference(Running<D, NT> &st, int n, float top, float c) {
  if (__any((top - st.ref[n]) * c > 8.0f)) {
    const float next = fmaxf(st.ref[n], top);
    const float f = __builtin_amdgcn_exp2f(origin_gap(st.ref[n], next, c));
    // (nothing seen so far: -infinity less itself)
    const float keep = st.ref[n] == -INFINITY ? 0.0f : f;
    st.ref[n] = next;
    st.top[n] = scaled(next, c);
    st.sum[n] *= keep;
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct) st.o[n][ct] *= keep;
  }
}

// A page's scales of kLargeScale and more that the lane's query row of tile n sees
// (seen: the largest, as bits) where its softmax weight is a number of fp32 a value
// that is not finite gives NaN by itself; where it is not, the product is 0, and the
// sums become NaN here.  Returns what to add to the largest score for the
// reference: uniform.
template <int D, int NT>
__device__ __forceinline__ float special_row(Running<D, NT> &st, int n, uint32_t seen, float c) {
  const bool nan = seen >= kNanScale;
  if (__any(nan)) {
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct) st.o[n][ct] += nan ? __builtin_nanf("") : 0.0f;
  }
  return __any(seen >= kLargeScale && !nan) ? fminf(kLift / c, 0x1p126f) : 0.0f;
}
__device__ __forceinline__ uint32_t across_groups_max(uint32_t bits) {
  auto a = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
  const uint32_t v = max(a[0], a[1]);
  auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return max(b[0], b[1]);
}

// The same for a page's scales vs (PageRegs::vs) and all tiles; limit as in add_page.
template <int D, int NT>
__device__ __forceinline__ float special_page(const uint32_t (&vs)[8], int g,
                                              const int (&limit)[NT], float c,
                                              Running<D, NT> &st) {
  float lift = 0.0f;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    uint32_t seen = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (16 * (i >> 2) + 4 * g + (i & 3) <= limit[n]) seen = max(seen, scale_bits(vs[i >> 1], i));
    lift = fmaxf(lift, special_row(st, n, across_groups_max(seen), c));
  }
  return lift;
}

// One page into the running state.  edge (uniform): some of its positions may be
// hidden from some rows (limit: each row's last visible position less the page's
// first).  lift: special_page's; CHECK: looked for here.
// scored(): called when the keys are done with.
struct Nothing {
  __device__ __forceinline__ void operator()() const {}
};
template <int D, int SPL, int NT, bool CHECK, class K, class V, class Q, class F = Nothing>
__device__ __forceinline__ void add_page(K &&k, V &&v, const uint32_t (&vs)[8], Q &&q, int g,
                                         bool edge, const int (&limit)[NT], float c, float lift,
                                         Running<D, NT> &st, F &&scored = F()) {
  // terms of a softmax weight: 16 bits, so that a bf16 output is off by its own
  // rounding alone; 24 for fp32
  constexpr int PTERMS = SPL == 1 ? 2 : 3;
  floatx4 s[NT][4];
  scores<D, SPL, NT>(k, q, s);
  scored();
  if (edge) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        asm volatile("" : "+v"(s[n][t]));        // (kept a branch: few pages take it)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (16 * t + 4 * g + i > limit[n]) s[n][t][i] = -INFINITY;
      }
  }
  if constexpr (CHECK)
    if (special_scales<8>(vs)) lift = special_page<D, NT>(vs, g, limit, c, st);
  float ref[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, s[n][t][i]);
    move_reference(st, n, across_groups_max(top) + lift, c);
    ref[n] = st.top[n] == -INFINITY ? 0.0f : st.top[n];
    if (__any(fabsf(ref[n]) >= kLargeLogit)) {
      const Origin at = origin_of(st.ref[n], c);
      ref[n] = at.top;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        asm volatile("" : "+v"(s[n][t]));        // (kept a branch)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][t][i] -= at.shift;
      }
    }
  }
  // tokens 32 h onwards: weights, then their values
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    bf16x8 w[NT][PTERMS];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int t = 2 * h + (i >> 2);
        const uint32_t two = vs[4 * h + (i >> 1)];
        e[i] = __builtin_amdgcn_exp2f(fmaf(s[n][t][i & 3], c, -ref[n]));
        st.sum[n] += e[i];
        // (0 times anything is 0: a hidden position may hold a scale that is not finite)
        e[i] = mul_zero(
            e[i], __uint_as_float(i & 1 ? two & 0xFFFF0000u : two << 16));
      }
      split8<PTERMS>(e, w[n]);
    }
#pragma unroll
    for (int c0 = 0; c0 < D / 16; c0 += 4) {
      if constexpr (NT == 1) __builtin_amdgcn_sched_barrier(0);
      bf16x8 a[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = v(h, c0 + i);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = PTERMS - 1; e >= 0; --e)
#pragma unroll
          for (int i = 0; i < 4; ++i) st.o[n][c0 + i] = mfma(a[i], w[n][e], st.o[n][c0 + i]);
    }
  }
}

// ---- few query rows: PACK tiles of tokens side by side ---------------------------
//
// With at most 16 / PACK query rows, most of a score tile's 16 columns are
// empty.  The columns of PACK tiles of tokens are moved side by side (lane moves
// within a row of 16 lanes), so that the softmax works on full registers, and
// the terms of the weights go back to columns of their own: the first to the
// query rows' columns, the second 16 / PACK columns further, so that one matrix
// instruction multiplies the values with both; unpack_rows adds the sums up at
// the end.  (Where the third term of fp32 finds no column it takes an
// instruction of its own.)  32 matrix instructions for a page of 64 tokens and 128
// channels, where full tiles take 48, and fewer vector ones.  512 rows of 100 to
// 1100 positions, 32 query and 8 K/V heads of 128: 66 us for four tiles side by
// side, 68 for two, 78 for one; 256 rows of 8 query heads a K/V head: 38.5 for
// two, 44 for one.

// Value scales of tokens 16 t + 4 g + i as bfloat16 i, t the lane's tile of each
// of the 4 / PACK registers' worth.
template <int D, int PACK>
__device__ __forceinline__ void load_packed_scales(const uint8_t *page, uint32_t g, uint32_t m,
                                                   PageRegs<D> &x) {
#pragma unroll
  for (uint32_t u = 0; u < 4 / PACK; ++u) {
    const uint32_t lane_at = g * 32 + m / (16 / PACK) * 8;
    const uint2 w = load_at<uint2>(page, lane_at, 66 * D + u * PACK * 8);
    x.vs[2 * u] = w.x;
    x.vs[2 * u + 1] = w.y;
  }
}

template <int D, int SPL, int PACK, class Q, class F = Nothing>
__device__ __forceinline__ void add_page_packed(const PageRegs<D> &x, Q &&q, int g, int m, bool edge,
                                                int limit, float c, floatx4 *keep_scores,
                                                Running<D, 1> &st, F &&scored = F()) {
  constexpr int PTERMS = SPL == 1 ? 2 : 3;
  constexpr int W = 16 / PACK, U = 4 / PACK;     // columns of a tile; registers of scores x 4
  floatx4 s[1][4];
  scores<D, SPL, 1>(keys_of(x), q, s);
  scored();
  // p[u][i]: lane 16 g + m has token 16 (PACK u + m / W) + 4 g + i, query row m % W
  float p[U][4];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (PACK == 4) {
        float v = s[0][0][i];
        v = lane_move<shl(-4), 0x2>(v, s[0][1][i]);
        v = lane_move<shl(-8), 0x4>(v, s[0][2][i]);
        p[u][i] = lane_move<shl(-12), 0x8>(v, s[0][3][i]);
      } else {
        p[u][i] = lane_move<shl(-8), 0xC>(s[0][2 * u][i], s[0][2 * u + 1][i]);
      }
    }
  if (keep_scores) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      keep_scores[u * 64 + 16 * g + m] = floatx4{p[u][0], p[u][1], p[u][2], p[u][3]};
  }
  if (edge) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        asm volatile("" : "+v"(p[u][i]));        // (kept a branch: few pages take it)
        if (16 * (PACK * u + m / W) + 4 * g + i > limit) p[u][i] = -INFINITY;
      }
  }
  float lift = 0.0f;
  if (special_scales<2 * U>(x.vs)) {
    uint32_t seen = 0;
#pragma unroll
    for (int i = 0; i < 4 * U; ++i)
      if (16 * (PACK * (i >> 2) + m / W) + 4 * g + (i & 3) <= limit)
        seen = max(seen, scale_bits(x.vs[i >> 1], i));
    if constexpr (PACK == 4) seen = max(seen, lane_move<ror(4)>(seen, seen));
    seen = max(seen, lane_move<ror(8)>(seen, seen));
    lift = special_row(st, 0, across_groups_max(seen), c);
  }
  float top = -INFINITY;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(top, p[u][i]);
  if constexpr (PACK == 4) top = fmaxf(top, lane_move<ror(4)>(top, top));
  top = fmaxf(top, lane_move<ror(8)>(top, top));
  move_reference(st, 0, across_groups_max(top) + lift, c);
  float ref = st.top[0] == -INFINITY ? 0.0f : st.top[0];
  if (__any(fabsf(ref) >= kLargeLogit)) {
    const Origin at = origin_of(st.ref[0], c);
    ref = at.top;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        asm volatile("" : "+v"(p[u][i]));        // (kept a branch)
        p[u][i] -= at.shift;
      }
  }
  // terms of the weights, two to a word
  uint32_t w[U][PTERMS][2];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t two = x.vs[2 * u + (i >> 1)];
      e[i] = __builtin_amdgcn_exp2f(fmaf(p[u][i], c, -ref));
      st.sum[0] += e[i];
      e[i] = mul_zero(e[i], __uint_as_float(i & 1 ? two & 0xFFFF0000u : two << 16));
    }
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      typedef float float2v __attribute__((ext_vector_type(2)));
      float a = e[2 * d], b = e[2 * d + 1];
#pragma unroll
      for (int n = 0; n < PTERMS; ++n) {
        w[u][n][d] = __builtin_bit_cast(uint32_t, __builtin_convertvector(float2v{a, b}, bf16x2));
        a -= __uint_as_float(w[u][n][d] << 16);
        b -= __uint_as_float(w[u][n][d] & 0xFFFF0000u);
      }
    }
  }
  // the operand of tokens 32 h onwards: tile t's first term from lanes W t' on to
  // lanes 0 .., its second to lanes W .., its third to lanes 2 W ..
  auto tile_words = [&](auto tc, int d) __attribute__((always_inline)) {
    constexpr int t = decltype(tc)::value;
    if constexpr (PACK == 4) {
      uint32_t v = lane_move<shl(4 * t)>(0u, w[0][0][d]);
      v = lane_move<shl(4 * t - 4), 0x2>(v, w[0][1][d]);
      if constexpr (PTERMS == 3) v = lane_move<shl(4 * t - 8), 0x4>(v, w[0][2][d]);
      return v;
    } else if constexpr (t % 2 == 0) {
      return lane_move<shl(-8), 0xC>(w[t / 2][0][d], w[t / 2][1][d]);
    } else {
      return lane_move<shl(8), 0x3>(w[t / 2][1][d], w[t / 2][0][d]);
    }
  };
  static_for<0, 2>([&](auto hc) __attribute__((always_inline)) {
    constexpr int h = decltype(hc)::value;
    const std::integral_constant<int, 2 * h> t0{};
    const std::integral_constant<int, 2 * h + 1> t1{};
    const bf16x8 b = __builtin_bit_cast(
        bf16x8, u32x4{tile_words(t0, 0), tile_words(t0, 1), tile_words(t1, 0), tile_words(t1, 1)});
    bf16x8 third = b;
    if constexpr (PACK == 2 && PTERMS == 3)
      // (nothing in the second term's columns)
      third = __builtin_bit_cast(
          bf16x8, u32x4{lane_move<kSame, 0x3>(0u, w[h][2][0]), lane_move<kSame, 0x3>(0u, w[h][2][1]),
                        lane_move<shl(8)>(0u, w[h][2][0]), lane_move<shl(8)>(0u, w[h][2][1])});
#pragma unroll
    for (int c0 = 0; c0 < D / 16; c0 += 4) {
      __builtin_amdgcn_sched_barrier(0);
      bf16x8 a[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = dequant(x.v[h][c0 + i], 1.0f);
      if constexpr (PACK == 2 && PTERMS == 3) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          st.o[0][c0 + i] = mfma(a[i], third, st.o[0][c0 + i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) st.o[0][c0 + i] = mfma(a[i], b, st.o[0][c0 + i]);
    }
  });
}

// Sums of the terms' columns to the query rows' columns, and the softmax sum of
// all lanes of a query row to each of them.
template <int D, int SPL, int PACK>
__device__ __forceinline__ void unpack_rows(Running<D, 1> &st) {
  if constexpr (PACK > 1) {
    constexpr int W = 16 / PACK;
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = st.o[0][c][i];
        float y = x + lane_move<shl(W)>(0.0f, x);
        if constexpr (PACK == 4 && SPL == 3) y += lane_move<shl(2 * W)>(0.0f, x);
        st.o[0][c][i] = y;
      }
    if constexpr (PACK == 4) st.sum[0] += lane_move<ror(4)>(st.sum[0], st.sum[0]);
    st.sum[0] += lane_move<ror(8)>(st.sum[0], st.sum[0]);
  }
  st.sum[0] = across_groups_sum(st.sum[0]);
}

// A query row's result, or its part of it where the row's pages are split over
// workgroups: the lanes of a column hold its channels' sums o (from channel g D / 4).
template <int D, bool BF16>
__device__ __forceinline__ void write_row(const AttendView &av, const Span &sp, const Query &q,
                                          int64_t part, bool partial, int g, float ref, float sum,
                                          const floatx4 (&o)[D / 16]) {
  if (partial) {
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
      *reinterpret_cast<floatx4 *>(av.part_o + part * D + g * (D / 4) + 4 * c) = o[c];
    if (g == 0) av.part_ml[part] = make_float2(ref, sum);
    return;
  }
  const bool none = sum == 0.0f;                 // nothing seen
  const float inv = none ? 0.0f : 1.0f / sum;
  const int64_t tok = sp.t0 + q.tok;
#pragma unroll
  for (int c = 0; c < D / 16; ++c) {
    const float y[4] = {none ? 0.0f : o[c][0] * inv, none ? 0.0f : o[c][1] * inv,
                        none ? 0.0f : o[c][2] * inv, none ? 0.0f : o[c][3] * inv};
    store4<BF16>(av.out, tok * av.out_stride + q.head * D + g * (D / 4) + 4 * c, y);
  }
  if (g == 0) finish_row(av, tok * av.Hq + q.head, ref, sum);
}

// Narrow rows: a workgroup of four waves for each (row, K/V head) and split, the
// pages dealt out to the waves, whose sums meet in LDS.  HBM bounds it; four
// waves on a SIMD, each waiting for a page of its own or working on one, keep
// the loads going (three or two waves that load a page ahead were slower).  512
// rows of 100 to 1100 positions (8 K/V heads of 128, 341 MB): 62 us, 5.5 TB/s,
// where a plain read reaches 6.4.
template <int D, int SPL, int PACK>
struct NarrowLds {
  static constexpr int W = 16 / PACK, WAVES = 4, PITCH = D + 4;
  float ml[2][WAVES][W];
  alignas(16) float o[WAVES * W * PITCH];
  // the queries' operands: in LDS they leave registers for the fourth wave
  bf16x8 q[SPL * (D / 32) * 64];
};

template <int D, int SPL, int PACK, int OCC>
__global__ __launch_bounds__(256, OCC) void narrow_kernel(CacheView cv, RowsView rv, AttendView av) {
  constexpr int W = 16 / PACK, WAVES = 4;
  constexpr bool BF16 = SPL == 1;
  constexpr int PITCH = D + 4;
  __shared__ NarrowLds<D, SPL, PACK> sh;
  auto &sh_ml = sh.ml;
  auto &sh_o = sh.o;
  auto &sh_q = sh.q;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, m = lane & 15;
  // (heads fastest: a page's heads lie side by side)
  const int h = blockIdx.x % cv.Hkv;
  const int r = blockIdx.x / cv.Hkv / av.splits;
  const int split = blockIdx.x / cv.Hkv - r * av.splits;
  const Span sp = row_span(cv, rv, r);
  if (sp.bad && h == 0 && threadIdx.x == 0) set_bad(av.status);
  if (!is_narrow(sp, av)) return;
  const int rows = sp.n * av.G;
  const int pages = tile_pages(sp, av.G, rows);
  const int used = splits_used(sp, av, pages);
  if (split > 0 && split >= used) return;
  const int p0 = split * av.split_pages, p1 = min(pages, p0 + av.split_pages);

  const Query qr = query_of(sp, av, h, m % W);
  const int all = min(sp.len - 1, sp.ctx);       // positions that every row sees
  Running<D, 1> st;
  st.ref[0] = st.top[0] = -INFINITY;
  st.sum[0] = 0.0f;
#pragma unroll
  for (int c = 0; c < D / 16; ++c) st.o[0][c] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};

  PageRegs<D> x;
  const int32_t *table = cv.table + (int64_t)sp.slot * cv.max_pages;
  // a page id out of range is replaced by page 0 with every position hidden
  auto fetch = [&](int id) __attribute__((always_inline)) {
    const bool ok = id >= 0 && id < cv.n_pages;
    const uint8_t *page = cv.pages + ((int64_t)(ok ? id : 0) * cv.Hkv + h) * cache_page_bytes(D);
    load_keys<D, true>(page, g, m, x);
    load_values<D, PACK == 1, true>(page, lane, x);
    if constexpr (PACK > 1) load_packed_scales<D, PACK>(page, g, m, x);
  };
  auto q = [&](int, int p, int e) __attribute__((always_inline)) {
    return sh_q[(p * (D / 32) + e) * 64 + lane];
  };
  int p = p0 + wave;
  int id = p < p1 ? ld_const(table, p) : 0, id_next = 0;
  if (p < p1) {
    fetch(id);
    if (p + WAVES < p1) id_next = ld_const(table, p + WAVES);
  }
  if (wave == 0) {
    const Query one[1] = {qr};
    bf16x8 w[1][SPL][D / 32];
    load_queries<D, SPL, 1>(av, sp, one, g, w, m < W);
#pragma unroll
    for (int i = 0; i < SPL; ++i)
#pragma unroll
      for (int e = 0; e < D / 32; ++e) sh_q[(i * (D / 32) + e) * 64 + lane] = w[0][i][e];
  }
  __syncthreads();
  while (p < p1) {
    const bool ok = id >= 0 && id < cv.n_pages;
    if (!ok && lane == 0) set_bad(av.status);
    const int limit[1] = {ok ? qr.limit - p * kPage : -1};
    const bool edge = !ok || p * kPage + kPage - 1 > all;
    if constexpr (PACK == 1)
      add_page<D, SPL, 1, true>(keys_of(x), values_of(x), x.vs, q, g, edge, limit, av.c, 0.0f, st);
    else
      add_page_packed<D, SPL, PACK>(
          x, q, g, m, edge, limit[0], av.c,
          av.scores ? av.scores + (((int64_t)r * cv.Hkv + h) * av.score_pages + p) * (256 / PACK)
                    : nullptr,
          st);
    p += WAVES;
    id = id_next;
    if (p < p1) fetch(id);
    id_next = p + WAVES < p1 ? ld_const(table, p + WAVES) : 0;
  }
  unpack_rows<D, SPL, PACK>(st);

  // the waves' sums, to their largest reference
  if (g == 0 && m < W) sh_ml[0][wave][m] = st.ref[0];
  __syncthreads();
  if (m < W) {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) top = fmaxf(top, sh_ml[0][i][m]);
    const float f = st.ref[0] == -INFINITY
                        ? 0.0f
                        : __builtin_amdgcn_exp2f(origin_gap(st.ref[0], top, av.c));
    if (g == 0) sh_ml[1][wave][m] = st.sum[0] * f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
      *reinterpret_cast<floatx4 *>(sh_o + (wave * W + m) * PITCH + g * (D / 4) + 4 * c) =
          st.o[0][c] * f;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < W * (D / 4); i += 256) {
    const int row = i / (D / 4), c4 = i % (D / 4) * 4;
    const Query qy = query_of(sp, av, h, row);
    if (!qy.valid) continue;
    float top = -INFINITY, l = 0.0f;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) top = fmaxf(top, sh_ml[0][k][row]);
    floatx4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < WAVES; ++k) {
      l += sh_ml[1][k][row];
      acc += *reinterpret_cast<const floatx4 *>(sh_o + (k * W + row) * PITCH + c4);
    }
    if (used > 1) {
      const int64_t part = (((int64_t)r * cv.Hkv + h) * av.splits + split) * W + row;
      *reinterpret_cast<floatx4 *>(av.part_o + part * D + c4) = acc;
      if (c4 == 0) av.part_ml[part] = make_float2(top, l);
      continue;
    }
    const bool none = l == 0.0f;                 // nothing seen
    const float inv = none ? 0.0f : 1.0f / l;
    const float y[4] = {none ? 0.0f : acc[0] * inv, none ? 0.0f : acc[1] * inv,
                        none ? 0.0f : acc[2] * inv, none ? 0.0f : acc[3] * inv};
    const int64_t tok = sp.t0 + qy.tok;
    store4<BF16>(av.out, tok * av.out_stride + qy.head * D + c4, y);
    if (c4 == 0) finish_row(av, tok * av.Hq + qy.head, top, l);
  }
}

// Wide rows: a workgroup of four waves for 64 NT query rows of a K/V head and a
// split of their pages.  The waves convert a quarter of the next page each, once
// for all, into operands in LDS (two pages: the one at work and the next; one,
// with another barrier, where two do not fit twice into a compute unit).  Matrix
// instructions and the softmax's vector work take about as long as each other;
// two workgroups on a compute unit overlap them (one of eight waves was slower,
// 785 against 753 us).  Four rows of 2048 new tokens over up to 4096 positions (32
// query and 8 K/V heads of 128): 723 us, 0.77 PFLOP/s (849 in the first passes
// after a pause; the clock settles in 40), the matrix units busy half of the time;
// the values' second term is a third of their work.  The look at the scales stands
// before the barrier: within the page's pass it cost 10 to 20 us more.
template <int D, int SPL, int NT, int OCC, class Rows>
__global__ __launch_bounds__(256, OCC) void wide_kernel(CacheView cv, Rows rv, AttendView av) {
  constexpr int TQ = 64 * NT, KF = D / 32, VF = D / 16;    // key operands of a tile, value of a half
  constexpr int BUFS = D == 256 ? 1 : 2;
  constexpr bool BF16 = SPL == 1;
  __shared__ bf16x8 sh_k[BUFS][4 * KF * 64], sh_v[BUFS][2 * VF * 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, m = lane & 15;
  // (heads fastest: tiles that read the same pages are a multiple of Hkv apart)
  const int h = blockIdx.x % cv.Hkv;
  const int item = blockIdx.x / cv.Hkv / av.splits;
  const int split = blockIdx.x / cv.Hkv - item * av.splits;
  int tile;
  const int r = tile_row(rv, av.G, TQ, item, tile);
  const Span sp = row_span(cv, rv, r);
  if (sp.bad && h == 0 && threadIdx.x == 0) set_bad(av.status);
  const int rows = sp.n * av.G, tiles = (rows + TQ - 1) / TQ;
  if (tile >= tiles || is_narrow(sp, av)) return;
  const int rho0 = (tiles - 1 - tile) * TQ;      // the longest first
  const int pages = tile_pages(sp, av.G, min(rho0 + TQ, rows));
  const int used = splits_used(sp, av, pages);
  if (split > 0 && split >= used) return;
  const int p0 = sp.page0 + split * av.split_pages, p1 = min(pages, p0 + av.split_pages);

  Query qr[NT];
  const int rhow = rho0 + wave * 16 * NT;
#pragma unroll
  for (int n = 0; n < NT; ++n) qr[n] = query_of(sp, av, h, rhow + 16 * n + m);
  // positions that every, and that any valid row of the wave sees
  const int all = min(sp.len - 1, sp.ctx + rhow / av.G);
  const int any = rhow < rows ? min(sp.len - 1, sp.ctx + (min(rhow + 16 * NT, rows) - 1) / av.G)
                              : -1;
  Running<D, NT> st;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    st.ref[n] = st.top[n] = -INFINITY;
    st.sum[n] = 0.0f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) st.o[n][c] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  // the wave's quarter of a page: tokens 16 wave onwards of the keys, VF / 2
  // operands of the values (one of two halves' worth of 64 channels each)
  constexpr int VQ = D / 64 >= 2 ? D / 128 : 1;  // 16-byte chunks of a lane
  constexpr bool VALL = D >= 128;                // (64 channels: two waves' work)
  struct Quarter {
    uint32_t k[KF], ks[D == 256 ? 2 : 1], vs[8];
    u32x4 v[VQ];
  } x;
  const int32_t *table = cv.table + (int64_t)sp.slot * cv.max_pages;
  auto fetch = [&](int id) __attribute__((always_inline)) {
    const bool ok = id >= 0 && id < cv.n_pages;
    const uint8_t *page = cv.pages + ((int64_t)(ok ? id : 0) * cv.Hkv + h) * cache_page_bytes(D);
    const uint32_t at = m * (D / 2) + g * (D / 8), tile_at = wave * 8 * D;
    if constexpr (D == 64) {
      const uint2 w = load_at<uint2>(page, at, tile_at);
      x.k[0] = w.x;
      x.k[1] = w.y;
    } else {
#pragma unroll
      for (uint32_t i = 0; i < D / 128; ++i) {
        const u32x4 w = load_at<u32x4>(page, at, tile_at + 16 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) x.k[4 * i + e] = w[e];
      }
    }
    if constexpr (D == 64) x.ks[0] = load_at<uint32_t>(page, m * 8 + (g >> 1) * 4, 64 * D);
    else if constexpr (D == 128) x.ks[0] = load_at<uint32_t>(page, m * 16 + g * 4, 64 * D);
    else {
      const uint2 w = load_at<uint2>(page, m * 32 + g * 8, 64 * D);
      x.ks[0] = w.x;
      x.ks[1] = w.y;
    }
    if (VALL || wave < 2) {
#pragma unroll
      for (uint32_t i = 0; i < VQ; ++i)
        x.v[i] = load_at<u32x4>(page, lane * 16, 32 * D + (wave * VQ + i) * 1024);
    }
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) {
      const u32x4 w = load_at<u32x4>(page, g * 32, 66 * D + 16 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) x.vs[4 * i + e] = w[e];
    }
  };
  auto convert = [&](int b) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < KF; ++e) {
      const float scale = __uint_as_float(((x.ks[e / 4] >> (8 * wave)) & 0xFFu) << 23);
      sh_k[b][(wave * KF + e) * 64 + lane] = dequant(x.k[e], scale);
    }
    if (VALL || wave < 2) {
#pragma unroll
      for (int i = 0; i < VQ; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sh_v[b][((wave * VQ + i) * 4 + e) * 64 + lane] = dequant(x.v[i][e], 1.0f);
    }
  };
  int id = p0 < p1 ? ld_const(table, p0) : 0;
  if (p0 < p1) fetch(id);
  bf16x8 qreg[NT][SPL][D / 32];
  load_queries<D, SPL, NT>(av, sp, qr, g, qreg);
  auto q = [&](int n, int p, int e) __attribute__((always_inline)) { return qreg[n][p][e]; };
  int b = 0;
  uint32_t vs[8];
  for (int p = p0; p < p1; ++p) {
    convert(b);
#pragma unroll
    for (int i = 0; i < 8; ++i) vs[i] = x.vs[i];
    const bool ok = id >= 0 && id < cv.n_pages;
    if (!ok && lane == 0) set_bad(av.status);
    id = p + 1 < p1 ? ld_const(table, p + 1) : 0;
    if (p + 1 < p1) fetch(id);
    int limit[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) limit[n] = ok ? qr[n].limit - p * kPage : -1;
    float lift = 0.0f;
    if (special_scales<8>(vs)) lift = special_page<D, NT>(vs, g, limit, av.c, st);
    __syncthreads();
    if (p * kPage <= any) {
      auto k = [&](int t, int e) __attribute__((always_inline)) {
        return sh_k[b][(t * KF + e) * 64 + lane];
      };
      auto v = [&](int hh, int ct) __attribute__((always_inline)) {
        return sh_v[b][(hh * VF + ct) * 64 + lane];
      };
      add_page<D, SPL, NT, false>(k, v, vs, q, g, !ok || p * kPage + kPage - 1 > all, limit, av.c,
                                  lift, st);
    }
    if constexpr (BUFS == 1) __syncthreads();
    else b ^= 1;
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const float sum = across_groups_sum(st.sum[n]);
    const int64_t part = Rows::kParts
                             ? part_of(av, sp.t0 + qr[n].tok, qr[n].head) + split
                             : (((int64_t)item * cv.Hkv + h) * av.splits + split) * TQ +
                                   (rhow + 16 * n + m - rho0);
    if (qr[n].valid)
      write_row<D, BF16>(av, sp, qr[n], part, Rows::kParts || used > 1, g, st.ref[n], sum, st.o[n]);
  }
}

template <int D, int SPL, int PACK>
void narrow_launch(const CacheView &cv, const RowsView &rv, const AttendView &av, const TilePlan &t,
                   hipStream_t st) {
  // registers for four waves on a SIMD; a single tile of 128 channels spilled there
  // (256 rows, 16 query heads a K/V head: 53 us, with three 47.5).  256 channels, 128
  // rows of 100 to 1100 positions, 4 query heads a K/V head: bf16 with two 27 us,
  // with one 37, with three (spills) 40; fp32 with one 46.5, with two 31.
  constexpr int OCC = D * SPL > 384 ? 1 : D * SPL > 128 ? 2 : PACK == 1 ? 3 : 4;
  hipLaunchKernelGGL((narrow_kernel<D, SPL, PACK, OCC>),
                     dim3((unsigned)(t.tiles * t.splits * cv.Hkv)), dim3(256), 0, st, cv, rv, av);
}

template <int D, int SPL, class Rows>
void wide_launch(const CacheView &cv, const Rows &rv, const AttendView &av, const TilePlan &t,
                 hipStream_t st) {
  const dim3 grid((unsigned)(t.tiles * t.splits * cv.Hkv));
  // (workgroups on a compute unit of 256 channels, 4 chunks of 400 to 512 tokens: bf16
  // two 127 us, one 195; fp32 one 239, two, with 12 registers spilled, 171.  Of 128
  // channels in fp32: one 146, two 150.)
  if (t.tile == 64) {
    hipLaunchKernelGGL((wide_kernel<D, SPL, 1, (D * SPL > 384 ? 1 : 2), Rows>), grid, dim3(256), 0,
                       st, cv, rv, av);
  } else {
    if constexpr (D < 256)
      hipLaunchKernelGGL((wide_kernel<D, SPL, 2, (D * SPL > 256 ? 1 : 2), Rows>), grid, dim3(256),
                         0, st, cv, rv, av);
  }
}

}  // namespace

// Tiles of `tile` query rows whose pages are split over workgroups until there
// are kWantGroups of them, in splits of at least `least` pages.  512 workgroups, two
// on a compute unit, against 256 and 1024: narrow rows, 8 of up to 16 k positions
// 28.6 us, 36.7 and 31.6, 64 of up to 3000 32.7, 32.4 and 37.6; wide ones, 2 of 512
// tokens over 4 k 129, 181 and 147, 9 of 150 to 357 over up to 3 k 79, 99 and 79.
// Least splits of narrow rows 8 pages: one row of 4000 positions 11.8 us, 16 pages
// 14.0, 4 pages 10.8.  Rows of up to kWholeNarrow pages are not split, for the
// join's launch costs more: in us, whole and in splits of 8 pages,
//   pages              11            16            24            32
//   1 row          8.3  11.3    10.1  11.9    12.9  12.1    15.2  11.6
//   8 rows         9.2  12.2    10.4  12.4    13.1  12.6    16.0  12.1
//   37 rows       11.6  15.8    14.0  16.0    17.9  19.4    21.6  23.4
// (64 rows alike).  Least splits of wide rows 4 pages: one of 500 tokens over 3.4 k
// positions 26.3, 8 pages 30.3; but 49 of 2 to 5 tokens over 270 positions, which
// that makes two splits of, 29 and 15.6.
constexpr int64_t kWantGroups = 512, kLeastNarrow = 8, kWholeNarrow = 16, kLeastWide = 4;

TilePlan tile_plan(int32_t tile, int64_t tiles, int64_t pages, int Hkv, int D, int64_t least,
                   int64_t want = kWantGroups);

}  // namespace mcd
