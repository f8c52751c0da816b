// Attention over the 4-bit key/value cache (mcd.h, mcd_cache_attend).
//
//   s[t] = scale q . k[t];  p = softmax(s) over the visible t;  out = sum p[t] v[t]
//
// in one pass over the pages with a running maximum and sum (base 2, fp32).
#include "cache_common.h"

namespace mcd {
namespace {

// a * b, 0 when either is 0 whatever the other is (v_mul_legacy_f32)
__device__ float mul_zero(float a, float b) __asm("llvm.amdgcn.fmul.legacy");

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
  float rest[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
  for (int n = 0; n < SPL; ++n) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      out[n][i] = (__bf16)rest[i];
      if (n + 1 < SPL) rest[i] -= (float)out[n][i];
    }
  }
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
template <class T>
__device__ __forceinline__ T load_at(const uint8_t *base, uint32_t lane_at, uint32_t at) {
  return *reinterpret_cast<const T *>(base + at + lane_at);
}

template <int D>
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
        const u32x4 w = load_at<u32x4>(page, lane_at, 16 * t * (D / 2) + 16 * i);
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

template <int D>
__device__ __forceinline__ void load_values(const uint8_t *page, uint32_t lane, PageRegs<D> &x) {
#pragma unroll
  for (uint32_t h = 0; h < 2; ++h)
#pragma unroll
    for (uint32_t q = 0; q < D / 64; ++q) {
      const u32x4 w = load_at<u32x4>(page, lane * 16, 32 * D + (h * (D / 64) + q) * 1024);
#pragma unroll
      for (int e = 0; e < 4; ++e) x.v[h][4 * q + e] = w[e];
    }
#pragma unroll
  for (uint32_t i = 0; i < 2; ++i) {
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

// Scores of the page's tokens 16 t + 4 g + i (i: component) against query
// column m of each of NT tiles.
template <int D, int SPL, int NT>
__device__ __forceinline__ void scores(const PageRegs<D> &x, const bf16x8 (&q)[NT][SPL][D / 32],
                                       floatx4 (&s)[NT][4]) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {
#pragma unroll
    for (int n = 0; n < NT; ++n) s[n][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < D / 32; ++e) {
      // (converted codes of two steps at a time, to keep the registers of three waves)
      if (e % 2 == 0) __builtin_amdgcn_sched_barrier(0);
      const bf16x8 a = dequant(x.k[t][e], key_exp(x.ks[e / 4], t));
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int p = SPL - 1; p >= 0; --p) s[n][t] = mfma(a, q[n][p][e], s[n][t]);
    }
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

// Pages seen by the query rows below end.
__device__ __forceinline__ int tile_pages(const Span &sp, int G, int end) {
  const int last = min(sp.len - 1, sp.ctx + (end - 1) / G);
  return last < 0 ? 0 : last / kPage + 1;
}

template <int D, int SPL, int NT>
__device__ __forceinline__ void load_queries(const AttendView &av, const Span &sp,
                                             const Query (&qr)[NT], int g,
                                             bf16x8 (&q)[NT][SPL][D / 32]) {
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int64_t at = (int64_t)(sp.t0 + qr[n].tok) * av.q_stride + qr[n].head * D + g * (D / 4);
#pragma unroll
    for (int e = 0; e < D / 32; ++e) {
      if constexpr (SPL == 1) {
        u32x4 w = {0u, 0u, 0u, 0u};
        if (qr[n].valid)
          w = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(av.q) + at + 8 * e);
        q[n][0][e] = __builtin_bit_cast(bf16x8, w);
      } else {
        float x[8] = {};
        if (qr[n].valid) {
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
// row, so row r's begin at start[r] G / TQ + r.
__host__ __device__ inline int64_t tile_items(int32_t R, int32_t N, int32_t G, int TQ, bool each) {
  return each ? (int64_t)R * ((G + TQ - 1) / TQ) : (int64_t)N * G / TQ + R;
}

__device__ __forceinline__ int tile_row(const RowsView &rv, int G, int TQ, int64_t x, int &tile) {
  if (!rv.start) {
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

__device__ __forceinline__ float across_groups_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float across_groups_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
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

// A finished query row's largest q . k and sum: its lse, and what weight_kernel
// needs of it.  Logits are compared before they are scaled, and the scale and
// log2(e) applied to differences: no size of logits overflows a difference.
__device__ __forceinline__ void finish_row(const AttendView &av, int64_t row, float top, float l) {
  if (av.lse)
    av.lse[row] = l == 0.0f ? -INFINITY
                            : (top * av.c + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
  if (av.stats) av.stats[row] = make_float2(top, l == 0.0f ? 0.0f : 1.0f / l);
}

// A wave's running state: for each of NT tiles of 16 query rows (column m of the
// lane) the largest q . k so far, the sum of its softmax weights at the lane's
// positions, and the sums of weight x value code for the lane's channels.
template <int D, int NT>
struct Running {
  float mx[NT], sum[NT];
  floatx4 o[NT][D / 16];
};

// One page into the running state.  edge (uniform): some of its positions may be
// hidden from some rows (limit: each row's last visible position less the page's
// first).
template <int D, int SPL, int NT>
__device__ __forceinline__ void add_page(const PageRegs<D> &x,
                                         const bf16x8 (&q)[NT][SPL][D / 32], int g, bool edge,
                                         const int (&limit)[NT], float c, Running<D, NT> &st) {
  // terms of a softmax weight: 16 bits, so that a bf16 output is off by its own
  // rounding alone; 24 for fp32
  constexpr int PTERMS = SPL == 1 ? 2 : 3;
  floatx4 s[NT][4];
  scores<D, SPL, NT>(x, q, s);
  if (edge) {
    __builtin_amdgcn_sched_barrier(0);           // (kept a branch: few pages take it)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (16 * t + 4 * g + i > limit[n]) s[n][t][i] = -INFINITY;
  }
  float ref[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, s[n][t][i]);
    top = across_groups_max(top);
    if (__any(top > st.mx[n])) {
      const float next = fmaxf(st.mx[n], top);
      const float from = next == -INFINITY ? 0.0f : next;
      const float f = __builtin_amdgcn_exp2f((st.mx[n] - from) * c);
      st.mx[n] = next;
      st.sum[n] *= f;
#pragma unroll
      for (int ct = 0; ct < D / 16; ++ct) st.o[n][ct] *= f;
    }
    ref[n] = st.mx[n] == -INFINITY ? 0.0f : st.mx[n];
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
        const uint32_t two = x.vs[4 * h + (i >> 1)];
        e[i] = __builtin_amdgcn_exp2f((s[n][t][i & 3] - ref[n]) * c);
        st.sum[n] += e[i];
        // (0 times anything is 0: a hidden position may hold a scale that is not finite)
        e[i] = mul_zero(
            e[i], __uint_as_float(i & 1 ? two & 0xFFFF0000u : two << 16));
      }
      split8<PTERMS>(e, w[n]);
    }
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct) {
      if (ct % 2 == 0) __builtin_amdgcn_sched_barrier(0);
      const bf16x8 a = dequant(x.v[h][ct], 1.0f);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = PTERMS - 1; e >= 0; --e) st.o[n][ct] = mfma(a, w[n][e], st.o[n][ct]);
    }
  }
}

// A workgroup of WQ x WK waves: WQ groups of 16 NT query rows, whose pages WK
// waves share out.
template <int D, int SPL, int NT, int WQ, int WK, int OCC>
__global__ __launch_bounds__(64 * WQ * WK, OCC) void attend_kernel(CacheView cv, RowsView rv,
                                                                  AttendView av) {
  constexpr int TQ = 16 * NT * WQ, NCT = D / 16;
  constexpr bool BF16 = SPL == 1;
  constexpr int PITCH = D + 4;
  __shared__ float sh_ml[WK > 1 ? 2 * WK * TQ : 1];
  __shared__ __align__(16) float sh_o[WK > 1 ? WK * TQ * PITCH : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, m = lane & 15, wq = wave / WK, wk = wave % WK;
  const int h = blockIdx.y;
  const int item = blockIdx.x / av.splits;
  const int split = blockIdx.x - item * av.splits;
  int tile;
  const int r = tile_row(rv, av.G, TQ, item, tile);
  const Span sp = row_span(cv, rv, r);
  if (sp.bad && h == 0 && threadIdx.x == 0) set_bad(av.status);
  const int rows = sp.n * av.G, rho0 = tile * TQ;
  if (tile < 0 || rho0 >= rows) return;
  // pages that any row of the tile sees
  const int pages = tile_pages(sp, av.G, min(rho0 + TQ, rows));
  const int used = (pages + av.split_pages - 1) / av.split_pages;
  if (split > 0 && split >= used) return;
  const int p0 = split * av.split_pages, p1 = min(pages, p0 + av.split_pages);

  Query qr[NT];
  const int rhow = rho0 + wq * 16 * NT;
#pragma unroll
  for (int n = 0; n < NT; ++n) qr[n] = query_of(sp, av, h, rhow + 16 * n + m);
  // positions that every valid row of the wave sees
  const int all = min(sp.len - 1, sp.ctx + rhow / av.G);

  Running<D, NT> st;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    st.mx[n] = -INFINITY;
    st.sum[n] = 0.0f;
#pragma unroll
    for (int c = 0; c < NCT; ++c) st.o[n][c] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  PageRegs<D> xa;
  const int32_t *table = cv.table + (int64_t)sp.slot * cv.max_pages;
  // the wave's pages p, p + WK, ...; a page id out of range is replaced by page
  // 0 with every position hidden
  int p = p0 + wk;
  int id = p < p1 ? ld_const(table, p) : 0, id_next = 0;
  auto fetch = [&](int page_id, PageRegs<D> &x) __attribute__((always_inline)) {
    const bool ok = page_id >= 0 && page_id < cv.n_pages;
    const uint8_t *page =
        cv.pages + ((int64_t)(ok ? page_id : 0) * cv.Hkv + h) * cache_page_bytes(D);
    load_keys<D>(page, g, m, x);
    load_values<D>(page, lane, x);
  };
  bf16x8 q[NT][SPL][D / 32];
  auto work = [&](int at, int page_id, const PageRegs<D> &x) __attribute__((always_inline)) {
    const bool ok = page_id >= 0 && page_id < cv.n_pages;
    if (!ok && lane == 0) set_bad(av.status);
    int limit[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) limit[n] = ok ? qr[n].limit - at * kPage : -1;
    add_page<D, SPL, NT>(x, q, g, !ok || at * kPage + kPage - 1 > all, limit, av.c, st);
  };
  if (p < p1) {
    fetch(id, xa);
    if (p + WK < p1) id_next = ld_const(table, p + WK);
  }
  load_queries<D, SPL, NT>(av, sp, qr, g, q);
  while (p < p1) {
    work(p, id, xa);
    p += WK;
    id = id_next;
    if (p < p1) fetch(id, xa);
    id_next = p + WK < p1 ? ld_const(table, p + WK) : 0;
  }
  float (&mx)[NT] = st.mx;
  float (&sum)[NT] = st.sum;
  floatx4 (&o)[NT][NCT] = st.o;
#pragma unroll
  for (int n = 0; n < NT; ++n) sum[n] = across_groups_sum(sum[n]);

  if constexpr (WK > 1) {
    // join the waves of a query group: scale each to the common maximum
#pragma unroll
    for (int n = 0; n < NT; ++n)
      if (g == 0) {
        sh_ml[wk * TQ + wq * 16 * NT + 16 * n + m] = mx[n];
        sh_ml[(WK + wk) * TQ + wq * 16 * NT + 16 * n + m] = sum[n];
      }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int row = wq * 16 * NT + 16 * n + m;
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < WK; ++i) top = fmaxf(top, sh_ml[i * TQ + row]);
      const float f = mx[n] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((mx[n] - top) * av.c);
#pragma unroll
      for (int c = 0; c < NCT; ++c)
        *reinterpret_cast<floatx4 *>(sh_o + (wk * TQ + row) * PITCH + g * (D / 4) + 4 * c) =
            o[n][c] * f;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < TQ * (D / 4); i += 64 * WQ * WK) {
      const int row = i / (D / 4), c4 = i % (D / 4) * 4;
      const Query qy = query_of(sp, av, h, rho0 + row);
      if (!qy.valid) continue;
      float top = -INFINITY, l = 0.0f;
#pragma unroll
      for (int k = 0; k < WK; ++k) top = fmaxf(top, sh_ml[k * TQ + row]);
      floatx4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < WK; ++k) {
        const float mk = sh_ml[k * TQ + row];
        l += sh_ml[(WK + k) * TQ + row] * (mk == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((mk - top) * av.c));
        acc += *reinterpret_cast<const floatx4 *>(sh_o + (k * TQ + row) * PITCH + c4);
      }
      if (used > 1) {
        const int64_t part = ((item * cv.Hkv + h) * av.splits + split) * TQ + row;
        *reinterpret_cast<floatx4 *>(av.part_o + part * D + c4) = acc;
        if (c4 == 0) av.part_ml[part] = make_float2(top, l);
        continue;
      }
      const bool none = l == 0.0f;                // nothing seen
      const float inv = none ? 0.0f : 1.0f / l;
      const float y[4] = {none ? 0.0f : acc[0] * inv, none ? 0.0f : acc[1] * inv,
                          none ? 0.0f : acc[2] * inv, none ? 0.0f : acc[3] * inv};
      const int64_t tok = sp.t0 + qy.tok;
      store4<BF16>(av.out, tok * av.out_stride + qy.head * D + c4, y);
      if (c4 == 0) {
        finish_row(av, tok * av.Hq + qy.head, top, l);
      }
    }
  } else {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (!qr[n].valid) continue;
      if (used > 1) {
        const int64_t part =
            ((item * cv.Hkv + h) * av.splits + split) * TQ + wq * 16 * NT + 16 * n + m;
#pragma unroll
        for (int c = 0; c < NCT; ++c)
          *reinterpret_cast<floatx4 *>(av.part_o + part * D + g * (D / 4) + 4 * c) = o[n][c];
        if (g == 0) av.part_ml[part] = make_float2(mx[n], sum[n]);
        continue;
      }
      const bool none = sum[n] == 0.0f;
      const float inv = none ? 0.0f : 1.0f / sum[n];
      const int64_t tok = sp.t0 + qr[n].tok;
#pragma unroll
      for (int c = 0; c < NCT; ++c) {
        const float y[4] = {none ? 0.0f : o[n][c][0] * inv, none ? 0.0f : o[n][c][1] * inv,
                            none ? 0.0f : o[n][c][2] * inv, none ? 0.0f : o[n][c][3] * inv};
        store4<BF16>(av.out, tok * av.out_stride + qr[n].head * D + g * (D / 4) + 4 * c, y);
      }
      if (g == 0) {
        finish_row(av, tok * av.Hq + qr[n].head, mx[n], sum[n]);
      }
    }
  }
}

// Joins the splits of a tile: a thread for four channels of a query row.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void join_kernel(CacheView cv, RowsView rv, AttendView av,
                                                   int TQ) {
  const int h = blockIdx.y;
  const int64_t item = blockIdx.x;
  int tile;
  const int r = tile_row(rv, av.G, TQ, item, tile);
  const Span sp = row_span(cv, rv, r);
  const int rows = sp.n * av.G, rho0 = tile * TQ;
  if (tile < 0 || rho0 >= rows) return;
  const int pages = tile_pages(sp, av.G, min(rho0 + TQ, rows));
  const int used = (pages + av.split_pages - 1) / av.split_pages;
  if (used <= 1) return;
  for (int i = threadIdx.x; i < TQ * (D / 4); i += 256) {
    const int row = i / (D / 4), c4 = i % (D / 4) * 4;
    const Query qy = query_of(sp, av, h, rho0 + row);
    if (!qy.valid) continue;
    const int64_t part = (item * cv.Hkv + h) * av.splits * TQ + row;
    float top = -INFINITY, l = 0.0f;
    for (int k = 0; k < used; ++k) top = fmaxf(top, av.part_ml[part + (int64_t)k * TQ].x);
    floatx4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = 0; k < used; ++k) {
      const float2 ml = av.part_ml[part + (int64_t)k * TQ];
      const float f = ml.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((ml.x - top) * av.c);
      l += ml.y * f;
      acc += *reinterpret_cast<const floatx4 *>(av.part_o + (part + (int64_t)k * TQ) * D + c4) * f;
    }
    const bool none = l == 0.0f;
    const float inv = none ? 0.0f : 1.0f / l;
    const float y[4] = {none ? 0.0f : acc[0] * inv, none ? 0.0f : acc[1] * inv,
                        none ? 0.0f : acc[2] * inv, none ? 0.0f : acc[3] * inv};
    const int64_t tok = sp.t0 + qy.tok;
    store4<BF16>(av.out, tok * av.out_stride + qy.head * D + c4, y);
    if (c4 == 0) {
      finish_row(av, tok * av.Hq + qy.head, top, l);
    }
  }
}

// Weight that every position received: the scores again, against the finished
// sums.  A wave for each page; its query tiles in order, so the sum's order is
// fixed.
template <int D, int SPL>
__global__ __launch_bounds__(256) void weight_kernel(CacheView cv, RowsView rv, AttendView av) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int g = lane >> 4, m = lane & 15, h = blockIdx.y, r = blockIdx.z;
  const int p = blockIdx.x * 4 + wave;
  const Span sp = row_span(cv, rv, r);
  if (sp.n == 0 || p * kPage >= sp.len) return;
  const uint8_t *page = page_of<D>(cv, sp.slot, p, h);
  if (!page) return;                           // reported by attend_kernel
  PageRegs<D> x;
  load_keys<D>(page, g, m, x);
  float total[16] = {};
  const int rows = sp.n * av.G;
  // the first token that sees the page
  const int first = max(0, p * kPage - sp.ctx) * av.G / 16 * 16;
  for (int rho = first; rho < rows; rho += 16) {
    Query qr[1] = {query_of(sp, av, h, rho + m)};
    bf16x8 q[1][SPL][D / 32];
    load_queries<D, SPL, 1>(av, sp, qr, g, q);
    const float2 st = qr[0].valid
                          ? av.stats[(int64_t)(sp.t0 + qr[0].tok) * av.Hq + qr[0].head]
                          : make_float2(0.0f, 0.0f);
    floatx4 s[1][4];
    scores<D, SPL, 1>(x, q, s);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (p * kPage + 16 * t + 4 * g + i <= qr[0].limit)
          total[4 * t + i] +=
              __builtin_amdgcn_exp2f((s[0][t][i] - st.x) * av.c) * st.y;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) total[i] += __shfl_xor(total[i], d);
  }
  // lane 16 g + m writes position 16 (m / 4) + 4 g + m % 4
  float mine = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (m == i) mine = total[i];
  const int pos = p * kPage + 16 * (m >> 2) + 4 * g + (m & 3);
  if (pos < sp.len) {
    const int64_t at = ((int64_t)sp.slot * cv.Hkv + h) * cv.max_pages * kPage + pos;
    av.weight_out[at] = (cv.weight ? cv.weight[at] : 0.0f) + mine;
  }
}

}  // namespace

AttendPlan cache_attend_plan(const CacheView &cv, const RowsView &rv, int D, int32_t Hq) {
  AttendPlan p;
  const int32_t G = Hq / cv.Hkv;
  const bool wide = (int64_t)rv.max_tokens * G > 16;
  p.tile = !wide ? 16 : D == 256 ? 64 : 128;
  p.tiles = tile_items(rv.R, rv.N, G, p.tile, rv.start == nullptr);
  const int64_t pages = ((int64_t)rv.max_context + kPage - 1) / kPage;
  const int64_t groups = p.tiles * cv.Hkv;
  const int64_t want = wide ? 512 : 1024;
  int64_t splits = groups > 0 ? (want + groups - 1) / groups : 1;
  splits = splits < 1 ? 1 : splits;
  const int64_t most = (pages + 3) / 4 < 1 ? 1 : (pages + 3) / 4;
  if (splits > most) splits = most;
  int64_t per = (pages + splits - 1) / splits;
  per = per < 4 ? 4 : (per + 3) / 4 * 4;
  splits = (pages + per - 1) / per;
  p.splits = (int32_t)(splits < 1 ? 1 : splits);
  p.split_pages = (int32_t)per;
  const size_t parts = p.splits > 1 ? (size_t)(groups * p.splits) * p.tile : 0;
  p.ml_bytes = parts * sizeof(float2);
  p.o_bytes = parts * D * sizeof(float);
  p.stat_bytes = (size_t)rv.N * Hq * sizeof(float2);
  return p;
}

namespace {

template <int D, int SPL>
void attend_launch(const CacheView &cv, const RowsView &rv, const AttendView &av,
                   const AttendPlan &plan, hipStream_t st) {
  const dim3 grid((unsigned)(plan.tiles * plan.splits), (unsigned)cv.Hkv);
  constexpr int OCC = D * SPL > 384 ? 1 : D * SPL > 128 ? 2 : 3;
  if (plan.tile == 16)
    hipLaunchKernelGGL((attend_kernel<D, SPL, 1, 1, 4, OCC>), grid, dim3(256), 0, st, cv, rv, av);
  else
    hipLaunchKernelGGL((attend_kernel<D, SPL, (D == 256 ? 1 : 2), 4, 1, 1>), grid, dim3(256), 0,
                       st, cv, rv, av);
  if (plan.splits > 1)
    hipLaunchKernelGGL((join_kernel<D, SPL == 1>), dim3((unsigned)plan.tiles, (unsigned)cv.Hkv),
                       dim3(256), 0, st, cv, rv, av, plan.tile);
  if (av.weight_out) {
    const unsigned pages = (unsigned)((rv.max_context + kPage - 1) / kPage);
    hipLaunchKernelGGL((weight_kernel<D, SPL>),
                       dim3((pages + 3) / 4, (unsigned)cv.Hkv, (unsigned)rv.R), dim3(256), 0, st,
                       cv, rv, av);
  }
}

}  // namespace

hipError_t launch_cache_attend(const CacheView &cv, const RowsView &rv, const AttendView &av,
                               const AttendPlan &plan, int D, bool bf16, hipStream_t st) {
  auto go = [&](auto d) {
    constexpr int W = decltype(d)::value;
    if (bf16) attend_launch<W, 1>(cv, rv, av, plan, st);
    else attend_launch<W, 3>(cv, rv, av, plan, st);
  };
  if (D == 64) go(std::integral_constant<int, 64>{});
  else if (D == 128) go(std::integral_constant<int, 128>{});
  else go(std::integral_constant<int, 256>{});
  return hipGetLastError();
}

}  // namespace mcd
