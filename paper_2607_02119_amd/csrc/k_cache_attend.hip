// Attention over the 4-bit key/value cache (mcd.h, mcd_cache_attend).
//
//   s[t] = scale q . k[t];  p = softmax(s) over the visible t;  out = sum p[t] v[t]
//
// in one pass over the pages with a running maximum and sum (base 2, fp32).
#include "cache_attend_tile.h"

namespace mcd {
namespace {

// Joins the splits of a tile: a thread for four channels of a query row, a
// workgroup for 256 of them.  A chain of loads over the splits, so four splits'
// loads go out together, and spread over the chip: one workgroup for a tile of 128
// rows of 14 splits took 100 us.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void join_kernel(CacheView cv, RowsView rv, AttendView av,
                                                   int TQ, bool narrow) {
  const int h = blockIdx.y;
  const int64_t item = blockIdx.x;
  int tile = 0;
  const int r = narrow ? (int)item : tile_row(rv, av.G, TQ, item, tile);
  const Span sp = row_span(cv, rv, r);
  const int rows = sp.n * av.G, tiles = (rows + TQ - 1) / TQ;
  if (tile >= tiles || is_narrow(sp, av) != narrow) return;
  const int rho0 = (tiles - 1 - tile) * TQ;
  const int pages = tile_pages(sp, av.G, min(rho0 + TQ, rows));
  const int used = splits_used(sp, av, pages);
  if (used <= 1) return;
  const int i = blockIdx.z * 256 + threadIdx.x, row = i / (D / 4), c4 = i % (D / 4) * 4;
  if (row >= TQ) return;
  const Query qy = query_of(sp, av, h, rho0 + row);
  if (!qy.valid) return;
  const int64_t part = (item * cv.Hkv + h) * av.splits * TQ + row;
  float top = -INFINITY, l = 0.0f;
  bool large = false;
#pragma unroll 4
  for (int k = 0; k < used; ++k) {
    const float ref = av.part_ml[part + (int64_t)k * TQ].x;
    top = fmaxf(top, ref);
    large |= is_large(ref, av.c);
  }
  floatx4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  auto add = [&](auto any_large) __attribute__((always_inline)) {
#pragma unroll 4
    for (int k = 0; k < used; ++k) {
      const float2 ml = av.part_ml[part + (int64_t)k * TQ];
      const float gap = origin_gap_of<decltype(any_large)::value>(ml.x, top, av.c);
      const float f = ml.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(gap);
      l += ml.y * f;
      acc += *reinterpret_cast<const floatx4 *>(av.part_o + (part + (int64_t)k * TQ) * D + c4) * f;
    }
  };
  if (__any(large)) add(std::integral_constant<bool, true>{});
  else add(std::integral_constant<bool, false>{});
  const bool none = l == 0.0f;
  const float inv = none ? 0.0f : 1.0f / l;
  const float y[4] = {none ? 0.0f : acc[0] * inv, none ? 0.0f : acc[1] * inv,
                      none ? 0.0f : acc[2] * inv, none ? 0.0f : acc[3] * inv};
  const int64_t tok = sp.t0 + qy.tok;
  store4<BF16>(av.out, tok * av.out_stride + qy.head * D + c4, y);
  if (c4 == 0) finish_row(av, tok * av.Hq + qy.head, top, l);
}

// ---- received weight ------------------------------------------------------------

// The same lane moves within four lanes.
template <int PERM>
__device__ __forceinline__ float quad_move(float x) {
  return __uint_as_float(
      (uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), PERM, 0xF, 0xF, false));
}

// A row without a token receives nothing: where weight_out is another array, what
// its positions [pos0, pos0 + n) had received before, by the lanes of a wave.
__device__ __forceinline__ void keep_weight(const CacheView &cv, const AttendView &av,
                                            const Span &sp, int h, int pos0, int n) {
  if (av.weight_out == cv.weight) return;
  const int64_t row = ((int64_t)sp.slot * cv.Hkv + h) * cv.max_pages * kPage;
  const int end = min(sp.len, pos0 + n);
  for (int pos = pos0 + (threadIdx.x & 63); pos < end; pos += 64)
    av.weight_out[row + pos] = cv.weight ? cv.weight[row + pos] : 0.0f;
}

// Four of the caller's weights, which may begin at any float (one access all the same).
typedef float weight4 __attribute__((ext_vector_type(4), aligned(4)));

// Narrow rows, from the scores that narrow_kernel left: 1 KiB of a page of 64
// tokens and 4 query rows (a quarter of its key codes, or a half for 8 rows).  A
// wave for four pages, their loads in flight together; bound by HBM: 15 us for 128
// rows of 900 to 4500 positions.
template <int PACK>
__global__ __launch_bounds__(256) void weight_scores_kernel(CacheView cv, RowsView rv,
                                                           AttendView av) {
  constexpr int W = 16 / PACK, U = 4 / PACK, PAGES = 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int g = lane >> 4, m = lane & 15, h = blockIdx.y, r = blockIdx.z;
  const int first = (blockIdx.x * 4 + wave) * PAGES;
  const Span sp = row_span(cv, rv, r);
  if (first * kPage >= sp.len) return;
  if (sp.n == 0) keep_weight(cv, av, sp, h, first * kPage, PAGES * kPage);
  if (!is_narrow(sp, av)) return;
  const Query qr = query_of(sp, av, h, m % W);
  const int last = min(first + PAGES - 1, (sp.len - 1) / kPage);
  const floatx4 *from =
      av.scores + (((int64_t)r * cv.Hkv + h) * av.score_pages) * (256 / PACK) + lane;
  const int64_t row = ((int64_t)sp.slot * cv.Hkv + h) * cv.max_pages * kPage;
  floatx4 s[PAGES][U], w[PAGES][U];
#pragma unroll
  for (int k = 0; k < PAGES; ++k)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int p = min(first + k, last);
      s[k][u] = from[(int64_t)p * (256 / PACK) + u * 64];
      const int64_t at = row + p * kPage + 16 * (PACK * u + m / W) + 4 * g;
      w[k][u] = cv.weight ? *reinterpret_cast<const weight4 *>(cv.weight + at)
                          : floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    }
  const float2 st = qr.valid ? av.stats[(int64_t)(sp.t0 + qr.tok) * av.Hq + qr.head]
                             : make_float2(0.0f, 0.0f);
  const Origin at = origin_of(st.x, av.c);
#pragma unroll
  for (int k = 0; k < PAGES; ++k) {
    const int p = first + k;
    if (p > last) break;
    const int id = ld_const(cv.table + (int64_t)sp.slot * cv.max_pages, p);
    if (id < 0 || id >= cv.n_pages) continue;  // reported by narrow_kernel
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int pos = p * kPage + 16 * (PACK * u + m / W) + 4 * g;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float e = __builtin_amdgcn_exp2f(fmaf(s[k][u][i] - at.shift, av.c, -at.top)) * st.y;
        e = pos + i <= qr.limit ? e : 0.0f;
        e += quad_move<0xB1>(e);               // lanes 1 0 3 2
        e += quad_move<0x4E>(e);               // lanes 2 3 0 1
        if constexpr (W == 8) e += lane_move<shl(4)>(0.0f, e);   // (for the lane that writes)
        w[k][u][i] += e;
      }
      if (m % W != 0) continue;
      if (pos + 4 <= sp.len) {
        *reinterpret_cast<weight4 *>(av.weight_out + row + pos) = w[k][u];
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (pos + i < sp.len) av.weight_out[row + pos + i] = w[k][u][i];
      }
    }
  }
}

// The other rows: the scores again, against the finished sums.  SHARED (where
// there are wide rows): the waves of a workgroup take a page's query tiles in
// turn and their sums meet in LDS, in the same order always; otherwise a wave for
// each page.  Bound by the chain of its query loads: 21 rows of up to 820
// positions and 5 prompts with 8 query heads on one K/V head of 64 channels took
// 145 us (the whole call) with a wave for each page, 52 with eight.  (Of 256
// channels' fp32 operands eight waves spill: 394 us for 4 chunks of 400 to 512
// tokens, 424 with eight.)
constexpr int weight_waves(int D, int SPL) { return D * SPL > 384 ? 4 : 8; }

template <int D, int SPL, bool SHARED>
__global__ __launch_bounds__(SHARED ? 64 * weight_waves(D, SPL) : 256)
void weight_kernel(CacheView cv, RowsView rv, AttendView av) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int g = lane >> 4, m = lane & 15, h = blockIdx.y, r = blockIdx.z;
  constexpr int W = SHARED ? weight_waves(D, SPL) : 1;
  const int p = SHARED ? blockIdx.x : blockIdx.x * 4 + wave;
  const Span sp = row_span(cv, rv, r);
  if (p * kPage >= sp.len) return;
  if (av.scores && (sp.n == 0 || is_narrow(sp, av))) return;   // (weight_scores_kernel's)
  if (sp.n == 0) {
    if (!SHARED || wave == 0) keep_weight(cv, av, sp, h, p * kPage, kPage);
    return;
  }
  const uint8_t *page = page_of<D>(cv, sp.slot, p, h);
  if (!page) return;                           // reported by the kernels above
  PageRegs<D> x;
  load_keys<D>(page, g, m, x);
  float total[16] = {};
  const int rows = sp.n * av.G;
  // the first token that sees the page
  const int first = max(0, p * kPage - sp.ctx) * av.G / 16 * 16;
  for (int rho = first + (SHARED ? 16 * wave : 0); rho < rows; rho += 16 * W) {
    Query qr[1] = {query_of(sp, av, h, rho + m)};
    bf16x8 q[1][SPL][D / 32];
    load_queries<D, SPL, 1>(av, sp, qr, g, q);
    const float2 st = qr[0].valid
                          ? av.stats[(int64_t)(sp.t0 + qr[0].tok) * av.Hq + qr[0].head]
                          : make_float2(0.0f, 0.0f);
    floatx4 s[1][4];
    scores<D, SPL, 1>(
        keys_of(x), [&](int n, int p, int e) __attribute__((always_inline)) { return q[n][p][e]; }, s);
    const Origin at = origin_of(st.x, av.c);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (p * kPage + 16 * t + 4 * g + i <= qr[0].limit)
          total[4 * t + i] +=
              __builtin_amdgcn_exp2f(fmaf(s[0][t][i] - at.shift, av.c, -at.top)) * st.y;
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
  if constexpr (SHARED) {
    __shared__ float part[W][64];
    part[wave][lane] = mine;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 1; w < W; ++w) mine += part[w][lane];
  }
  const int pos = p * kPage + 16 * (m >> 2) + 4 * g + (m & 3);
  if (pos < sp.len) {
    const int64_t at = ((int64_t)sp.slot * cv.Hkv + h) * cv.max_pages * kPage + pos;
    av.weight_out[at] = (cv.weight ? cv.weight[at] : 0.0f) + mine;
  }
}

// Kept scores at most; larger steps compute them again (128 rows of 900 to 4500
// positions: 105 us with the scores kept, 152 without).
constexpr size_t kMostScores = (size_t)1 << 30;

size_t score_bytes(int64_t R, int64_t Hkv, int64_t pages, int pack) {
  // (below 2^56: R, Hkv < 2^16, pages <= 2^24; the bytes may pass 64 bits)
  const size_t tiles = (size_t)(R * Hkv * pages);
  return std::min(tiles, kMostScores) * (64 * 16 / pack) * sizeof(float);
}

}  // namespace

TilePlan tile_plan(int32_t tile, int64_t tiles, int64_t pages, int Hkv, int D, int64_t least,
                   int64_t want) {
  TilePlan p = {};
  if (tiles == 0) return p;
  p.tile = tile;
  p.tiles = tiles;
  const int64_t groups = tiles * Hkv;
  const int64_t most = std::max<int64_t>((pages + least - 1) / least, 1);
  int64_t splits = std::min(std::max<int64_t>((want + groups - 1) / groups, 1), most);
  const int64_t per = std::max<int64_t>(((pages + splits - 1) / splits + 3) / 4 * 4, least);
  splits = std::max<int64_t>((pages + per - 1) / per, 1);
  p.splits = (int32_t)splits;
  p.split_pages = (int32_t)per;
  const size_t parts = splits > 1 ? (size_t)(groups * splits) * tile : 0;
  p.ml_bytes = parts * sizeof(float2);
  p.o_bytes = parts * D * sizeof(float);
  return p;
}

AttendPlan cache_attend_plan(const CacheView &cv, const RowsView &rv, int D, int32_t Hq) {
  AttendPlan p = {};
  const int32_t G = Hq / cv.Hkv;
  const int64_t pages =
      std::min<int64_t>(((int64_t)rv.max_context + kPage - 1) / kPage, cv.max_pages);
  // rows of more than a tile of 16 query rows, and rows that may be of fewer: of
  // one token where there are both
  const bool wide = (int64_t)rv.max_tokens * G > 16;
  const bool narrow = !wide || (G <= 16 && rv.start && rv.N < (int64_t)rv.R * rv.max_tokens);
  const int64_t rows = wide ? G : (int64_t)rv.max_tokens * G;
  p.pack = rows <= 4 ? 4 : rows <= 8 ? 2 : 1;
  p.narrow_rows = narrow ? 16 / p.pack : 0;
  if (narrow)
    p.narrow = tile_plan(16 / p.pack, rv.R, pages, cv.Hkv, D,
                         pages <= kWholeNarrow ? kWholeNarrow : kLeastNarrow);
  if (wide) {
    // steps of short chunks in tiles of 64 rows: 52 rows of 2 to 12 tokens of four
    // heads (fp32, up to 2221 positions) 34 us, in tiles of 128 43; 49 of 2 to 5
    // (bf16, 270) 29 and 37
    const int tile = D == 256 || (int64_t)rv.max_tokens * G <= 64 ? 64 : 128;
    p.wide = tile_plan(tile, tile_items(rv.R, rv.N, G, tile, token_each(rv)), pages, cv.Hkv, D,
                       kLeastWide);
  }
  p.stat_bytes = (size_t)rv.N * Hq * sizeof(float2);
  // kept scores, of a cache that has weights: worth it where they are fewer bytes
  // than the key codes
  p.score_pages = (int32_t)pages;
  if (narrow && p.pack > 1 && cv.weight) {
    const size_t bytes = score_bytes(rv.R, cv.Hkv, pages, p.pack);
    p.score_bytes = bytes <= kMostScores ? bytes : 0;
  }
  return p;
}

// The most that the plan of any rows within these bounds asks for: fewer rows
// are split into more parts, and keep scores where more rows do not.
AttendPlan cache_attend_room(const CacheView &cv, const RowsView &rv, int D, int32_t Hq) {
  AttendPlan p = {};
  const int32_t G = Hq / cv.Hkv;
  const int64_t pages =
      std::min<int64_t>(((int64_t)rv.max_context + kPage - 1) / kPage, cv.max_pages);
  auto part_rows = [&](int64_t tiles, int64_t tile, int64_t least) {
    const int64_t most = (pages + least - 1) / least;
    // (from kWantGroups workgroups on nothing is split)
    const int64_t groups = std::min(tiles * cv.Hkv, kWantGroups - 1);
    return most <= 1 ? 0 : std::min(kWantGroups + groups - 1, groups * most) * tile;
  };
  const int64_t narrow = std::min<int64_t>(rv.max_tokens, 16 / G) * G;   // query rows, 0: none
  int64_t rows = 0;
  if (narrow > 0 && pages > kWholeNarrow)
    rows += part_rows(rv.R, narrow <= 4 ? 4 : narrow <= 8 ? 8 : 16, kLeastNarrow);
  if ((int64_t)rv.max_tokens * G > 16) {
    auto wide = [&](int64_t tile) {
      return part_rows(tile_items(rv.R, rv.N, G, (int)tile, false), tile, kLeastWide);
    };
    rows += D < 256 && (int64_t)rv.max_tokens * G > 64 ? std::max(wide(64), wide(128)) : wide(64);
  }
  p.wide.ml_bytes = (size_t)rows * sizeof(float2);
  p.wide.o_bytes = (size_t)rows * D * sizeof(float);
  p.stat_bytes = (size_t)rv.N * Hq * sizeof(float2);
  const int64_t kept = std::min<int64_t>(rv.max_tokens, 8 / G) * G;
  if (kept > 0 && cv.weight)
    p.score_bytes = std::min(score_bytes(rv.R, cv.Hkv, pages, kept <= 4 ? 4 : 2), kMostScores);
  return p;
}

namespace {

template <int D, int SPL>
void attend_launch(const CacheView &cv, const RowsView &rv, AttendView av, const AttendPlan &plan,
                   hipStream_t st) {
  for (const bool narrow : {true, false}) {
    const TilePlan &t = narrow ? plan.narrow : plan.wide;
    if (t.tiles == 0) continue;
    av.splits = t.splits;
    av.split_pages = t.split_pages;
    if (!narrow) wide_launch<D, SPL>(cv, rv, av, t, st);
    else if (plan.pack == 4) narrow_launch<D, SPL, 4>(cv, rv, av, t, st);
    else if (plan.pack == 2) narrow_launch<D, SPL, 2>(cv, rv, av, t, st);
    else narrow_launch<D, SPL, 1>(cv, rv, av, t, st);
    if (t.splits > 1)
      hipLaunchKernelGGL((join_kernel<D, SPL == 1>),
                         dim3((unsigned)t.tiles, (unsigned)cv.Hkv,
                              (unsigned)((t.tile * (D / 4) + 255) / 256)),
                         dim3(256), 0, st, cv, rv, av, t.tile, narrow);
    av.part_ml += t.ml_bytes / sizeof(float2);
    av.part_o += t.o_bytes / sizeof(float);
  }
  const unsigned pages = (unsigned)plan.score_pages;
  if (av.weight_out && pages > 0) {              // (0: no row sees a position)
    if (av.scores) {
      const dim3 grid((pages + 15) / 16, (unsigned)cv.Hkv, (unsigned)rv.R);
      if (plan.pack == 4)
        hipLaunchKernelGGL(weight_scores_kernel<4>, grid, dim3(256), 0, st, cv, rv, av);
      else
        hipLaunchKernelGGL(weight_scores_kernel<2>, grid, dim3(256), 0, st, cv, rv, av);
      if (plan.wide.tiles == 0) return;
    }
    if (plan.wide.tiles)
      hipLaunchKernelGGL((weight_kernel<D, SPL, true>),
                         dim3(pages, (unsigned)cv.Hkv, (unsigned)rv.R),
                         dim3(64 * weight_waves(D, SPL)), 0, st, cv, rv, av);
    else
      hipLaunchKernelGGL((weight_kernel<D, SPL, false>),
                         dim3((pages + 3) / 4, (unsigned)cv.Hkv, (unsigned)rv.R), dim3(256), 0, st,
                         cv, rv, av);
  }
}

}  // namespace

hipError_t launch_cache_keep_weight(const CacheView &cv, const RowsView &rv, float *weight_out,
                                    hipStream_t st) {
  AttendView av = {};
  av.weight_out = weight_out;
  const int64_t pages =
      std::min<int64_t>(((int64_t)rv.max_context + kPage - 1) / kPage, cv.max_pages);
  if (pages == 0) return hipSuccess;
  // (no row has a token, so channels and type do not matter)
  hipLaunchKernelGGL((weight_kernel<64, 1, false>),
                     dim3((unsigned)((pages + 3) / 4), (unsigned)cv.Hkv, (unsigned)rv.R), dim3(256),
                     0, st, cv, rv, av);
  return hipGetLastError();
}

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
