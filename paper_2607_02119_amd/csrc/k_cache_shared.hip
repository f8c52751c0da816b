// Attention of rows that begin with the same pages (mcd.h, mcd_cache_attend_shared).
//
// The rows of a group see the whole pages of its prefix all alike, so their tokens
// are one tile's query rows there: a page of a prefix is read, and its codes turned
// into operands, once for the group instead of once for each row.  What a row has
// past the prefix it reads by itself.  Both leave parts of every query row's softmax,
// {reference a, sum l, sums o}, which join_parts_kernel adds up:
//
//   A = max a;  l = sum l_i 2^((a_i - A) c);  out = sum o_i 2^((a_i - A) c) / l
#include "cache_attend_tile.h"

namespace mcd {
namespace {

// Group g's rows [a, b) and the whole pages that they share.
struct Group {
  int a, b, pages;
  bool bad;
};

__device__ __forceinline__ int group_start(const RowsView &rv, const GroupsView &gv, int g) {
  return min(max(gv.start[g], 0), rv.R);
}

__device__ __forceinline__ Group group_at(const CacheView &cv, const RowsView &rv,
                                          const GroupsView &gv, int g) {
  Group x;
  const int a = ld_const(gv.start, g), b = ld_const(gv.start, g + 1), n = ld_const(gv.prefix, g);
  x.a = min(max(a, 0), rv.R);
  x.b = min(max(b, x.a), rv.R);
  x.pages = min(min(max(n, 0), gv.max_prefix) / kPage, cv.max_pages);
  x.bad = x.a != a || x.b != b || x.b - x.a > gv.max_rows || n < 0 || n > gv.max_prefix ||
          n / kPage > cv.max_pages;
  x.b = min(x.b, x.a + min(gv.max_rows, rv.R));  // (rows past max_rows are in no group)
  return x;
}

// The group's tokens as those of one row whose positions are the prefix: token i of
// the span is token start[first row] + i, and sees all of it.
__device__ __forceinline__ Span group_span(const CacheView &cv, const RowsView &rv,
                                           const GroupsView &gv, const Group &x) {
  Span s;
  s.page0 = 0;
  s.bad = x.bad;
  s.len = x.pages * kPage;
  s.ctx = s.len - 1;
  s.t0 = x.a < x.b ? row_start(rv, x.a) : 0;
  const int t1 = x.a < x.b ? (rv.start ? min(max(rv.start[x.b], s.t0), rv.N) : x.b) : 0;
  const int64_t most = (int64_t)gv.max_rows * rv.max_tokens;
  s.bad |= t1 - s.t0 > most;
  s.n = (int)min((int64_t)(t1 - s.t0), most);
  s.slot = x.a < x.b ? (rv.slot ? ld_const(rv.slot, x.a) : x.a) : 0;
  if (s.slot < 0 || s.slot >= cv.n_slots) {
    s.bad = true;
    s.slot = 0;
    s.len = 0;
    s.ctx = -1;
  }
  return s;
}

// The group of a row (the wave together), or none: -1.
__device__ __forceinline__ int group_of(const CacheView &cv, const RowsView &rv,
                                        const GroupsView &gv, int r, Group &x) {
  const int g = find_row(gv.n, r, [&](int i) __attribute__((always_inline)) {
    return group_start(rv, gv, i);
  });
  x = group_at(cv, rv, gv, g);
  return r >= x.a && r < x.b ? g : -1;
}

// A row's own pages; page0 < 0: it is in no group, or does not reach past its group's
// prefix, and sees nothing.
__device__ __forceinline__ Span own_span(const CacheView &cv, const RowsView &rv,
                                         const GroupsView &gv, int r, Group &x) {
  Span s = row_span(cv, rv, r);
  const int g = group_of(cv, rv, gv, r, x);
  s.page0 = x.pages;
  if (g < 0 || (s.n > 0 && s.ctx < x.pages * kPage)) {
    s.bad = true;
    s.page0 = -1;
    s.len = 0;
    return s;
  }
  const int64_t cap = (int64_t)x.pages * kPage + gv.max_own;
  s.bad |= s.len > cap;
  s.len = (int)min((int64_t)s.len, cap);
  return s;
}

// The two kinds of rows for the tiles' kernels.
struct PrefixRows {
  RowsView rv;
  GroupsView gv;
};
__device__ __forceinline__ Span row_span(const CacheView &cv, const PrefixRows &p, int g) {
  return group_span(cv, p.rv, p.gv, group_at(cv, p.rv, p.gv, g));
}
__device__ __forceinline__ int tile_row(const PrefixRows &p, int G, int TQ, int64_t x, int &tile) {
  auto base = [&](int g) __attribute__((always_inline)) {
    const int a = group_start(p.rv, p.gv, g);
    const int t = a >= p.rv.R ? p.rv.N : row_start(p.rv, a);
    return (int64_t)t * G / TQ + g;
  };
  const int g = find_row(p.gv.n, x, base);
  tile = (int)min(max(x - base(g), (int64_t)0), (int64_t)1 << 30);
  return g;
}

struct OwnRows {
  static constexpr bool kParts = true;
  RowsView rv;
  GroupsView gv;
};
__device__ __forceinline__ Span row_span(const CacheView &cv, const OwnRows &p, int r) {
  Group x;
  Span s = own_span(cv, p.rv, p.gv, r, x);
  s.page0 = max(s.page0, 0);
  return s;
}
__device__ __forceinline__ int tile_row(const OwnRows &p, int G, int TQ, int64_t x, int &tile) {
  return tile_row(p.rv, G, TQ, x, tile);
}

// ---- prefixes of few query rows -------------------------------------------------
//
// A workgroup of four waves for 16 NT query rows of a group and K/V head and a split of the
// prefix, the pages dealt out to the waves: each turns the codes of its page into
// operands in registers, for all of its NT tiles, with no barrier until the end, and has
// the next page's codes in flight.  Issuing vector instructions bounds it (560 a page of 128
// channels for two tiles, 128 of them conversions), at two waves on a SIMD, which hardly
// overlap them with the matrix units.  The prefix of 64 rows on 16000 positions (32 query
// and 8 K/V heads of 128): two tiles 36 us, one 41 (the conversions for half the
// rows), four 60 (one wave on a SIMD), the tiles of 128 rows of wide_kernel, whose
// waves share the conversions but wait for each other, 49.
template <int D, int SPL, int NT>
struct PrefixLds {
  float ml[2][4][16 * NT];
  alignas(16) float o[4 * 16 * (D + 4)];
  bf16x8 q[NT * SPL * (D / 32) * 64];
};

template <int D, int SPL, int NT>
__device__ __forceinline__ void prefix_rows(const CacheView &cv, const PrefixRows &rv,
                                            const AttendView &av, uint32_t block,
                                            PrefixLds<D, SPL, NT> &sh) {
  constexpr int TQ = 16 * NT, WAVES = 4, PITCH = D + 4;
  auto &sh_ml = sh.ml;
  auto &sh_o = sh.o;
  auto &sh_q = sh.q;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, m = lane & 15;
  const int h = block % cv.Hkv;
  const int item = block / cv.Hkv / av.splits;
  const int split = block / cv.Hkv - item * av.splits;
  int tile;
  const int r = tile_row(rv, av.G, TQ, item, tile);
  const Span sp = row_span(cv, rv, r);
  if (sp.bad && h == 0 && threadIdx.x == 0) set_bad(av.status);
  const int rows = sp.n * av.G, rho0 = tile * TQ;
  const int pages = sp.len / kPage;
  const int p0 = split * av.split_pages, p1 = min(pages, p0 + av.split_pages);
  if (rho0 >= rows || p0 >= p1) return;

  Query qr[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) qr[n] = query_of(sp, av, h, rho0 + 16 * n + m);
  Running<D, NT> st;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    st.ref[n] = st.top[n] = -INFINITY;
    st.sum[n] = 0.0f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) st.o[n][c] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  PageRegs<D> x;
  const int32_t *table = cv.table + (int64_t)sp.slot * cv.max_pages;
  // a page id out of range is replaced by page 0 with every position hidden
  auto page_at = [&](int id) __attribute__((always_inline)) {
    const bool ok = id >= 0 && id < cv.n_pages;
    return cv.pages + ((int64_t)(ok ? id : 0) * cv.Hkv + h) * cache_page_bytes(D);
  };
  int p = p0 + wave;
  int id = p < p1 ? ld_const(table, p) : 0, id_next = 0;
  if (p < p1) {
    load_keys<D>(page_at(id), g, m, x);
    load_values<D>(page_at(id), lane, x);
    id_next = ld_const(table, min(p + WAVES, p1 - 1));
  }
  for (int n = wave; n < NT; n += WAVES) {
    const Query one[1] = {query_of(sp, av, h, rho0 + 16 * n + m)};
    bf16x8 w[1][SPL][D / 32];
    load_queries<D, SPL, 1>(av, sp, one, g, w);
#pragma unroll
    for (int i = 0; i < SPL; ++i)
#pragma unroll
      for (int e = 0; e < D / 32; ++e) sh_q[((n * SPL + i) * (D / 32) + e) * 64 + lane] = w[0][i][e];
  }
  __syncthreads();
  auto q = [&](int n, int i, int e) __attribute__((always_inline)) {
    return sh_q[((n * SPL + i) * (D / 32) + e) * 64 + lane];
  };
  while (p < p1) {
    const bool ok = id >= 0 && id < cv.n_pages;
    if (!ok && lane == 0) set_bad(av.status);
    int limit[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) limit[n] = ok ? kPage - 1 : -1;
    // the next keys into the registers of these once the scores are there, the next values
    // once these are added; after the last page that page again, for loads on a condition
    // would have the values waited for together with the keys behind them
    auto scored = [&]() __attribute__((always_inline)) {
      load_keys<D>(page_at(id_next), g, m, x);
    };
    add_page<D, SPL, NT, true>(keys_of(x), values_of(x), x.vs, q, g, !ok, limit, av.c, 0.0f, st,
                               scored);
    p += WAVES;
    id = id_next;
    load_values<D>(page_at(id), lane, x);
    id_next = ld_const(table, min(p + WAVES, p1 - 1));
  }

  // the waves' sums, to their largest reference, a tile at a time
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    st.sum[n] = across_groups_sum(st.sum[n]);
    if (g == 0) sh_ml[0][wave][16 * n + m] = st.ref[n];
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) top = fmaxf(top, sh_ml[0][i][16 * n + m]);
    const float f = st.ref[n] == -INFINITY
                        ? 0.0f
                        : __builtin_amdgcn_exp2f(origin_gap(st.ref[n], top, av.c));
    if (g == 0) sh_ml[1][wave][16 * n + m] = st.sum[n] * f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
      *reinterpret_cast<floatx4 *>(sh_o + (wave * 16 + m) * PITCH + g * (D / 4) + 4 * c) =
          st.o[n][c] * f;
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * (D / 4); i += 256) {
      const int row = i / (D / 4), c4 = i % (D / 4) * 4;
      const Query qy = query_of(sp, av, h, rho0 + 16 * n + row);
      if (!qy.valid) continue;
      floatx4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
      float best = -INFINITY, l = 0.0f;
#pragma unroll
      for (int k = 0; k < WAVES; ++k) {
        best = fmaxf(best, sh_ml[0][k][16 * n + row]);
        l += sh_ml[1][k][16 * n + row];
        acc += *reinterpret_cast<const floatx4 *>(sh_o + (k * 16 + row) * PITCH + c4);
      }
      const int64_t part = part_of(av, sp.t0 + qy.tok, qy.head) + split;
      *reinterpret_cast<floatx4 *>(av.part_o + part * D + c4) = acc;
      if (c4 == 0) av.part_ml[part] = make_float2(best, l);
    }
    if (n + 1 < NT) __syncthreads();
  }
}

// ---- the rows' own pages ---------------------------------------------------------
//
// A wave for each narrow row, K/V head and split of the row's own pages: few pages mostly,
// whose cost is a chain of loads.  Beside the prefixes there is room for two workgroups on a
// compute unit, where waves that work alone are sooner through many rows than four that
// share a row's pages and meet in LDS (256 rows of 5 pages, whole call: 46 and 55 us).
template <int D, int SPL, int PACK>
__device__ __forceinline__ void own_rows(const CacheView &cv, const OwnRows &rv,
                                         const AttendView &av, uint32_t unit) {
  constexpr int W = 16 / PACK;
  const int lane = threadIdx.x & 63, g = lane >> 4, m = lane & 15;
  const int h = unit % cv.Hkv;
  const int r = unit / cv.Hkv / av.splits;
  const int split = unit / cv.Hkv - r * av.splits;
  if (r >= rv.rv.R) return;
  const Span sp = row_span(cv, rv, r);
  if (sp.bad && h == 0 && lane == 0) set_bad(av.status);
  if (!is_narrow(sp, av)) return;
  const int rows = sp.n * av.G;
  const int pages = tile_pages(sp, av.G, rows), used = splits_used(sp, av, pages);
  if (split > 0 && split >= used) return;
  const int p0 = sp.page0 + split * av.split_pages, p1 = min(pages, p0 + av.split_pages);
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
  auto page_at = [&](int id) __attribute__((always_inline)) {
    const bool ok = id >= 0 && id < cv.n_pages;
    return cv.pages + ((int64_t)(ok ? id : 0) * cv.Hkv + h) * cache_page_bytes(D);
  };
  auto get_values = [&](int id) __attribute__((always_inline)) {
    load_values<D, PACK == 1, true>(page_at(id), lane, x);
    if constexpr (PACK > 1) load_packed_scales<D, PACK>(page_at(id), g, m, x);
  };
  int p = p0, id = p < p1 ? ld_const(table, p) : 0, id_next = 0;
  if (p < p1) {
    load_keys<D, true>(page_at(id), g, m, x);
    get_values(id);
    id_next = ld_const(table, min(p + 1, p1 - 1));
  }
  const Query one[1] = {qr};
  bf16x8 w[1][SPL][D / 32];
  load_queries<D, SPL, 1>(av, sp, one, g, w, m < W);
  auto q = [&](int, int i, int e) __attribute__((always_inline)) { return w[0][i][e]; };
  while (p < p1) {
    const bool ok = id >= 0 && id < cv.n_pages;
    if (!ok && lane == 0) set_bad(av.status);
    const int limit[1] = {ok ? qr.limit - p * kPage : -1};
    const bool edge = !ok || p * kPage + kPage - 1 > all;
    auto scored = [&]() __attribute__((always_inline)) {
      load_keys<D, true>(page_at(id_next), g, m, x);
    };
    if constexpr (PACK == 1)
      add_page<D, SPL, 1, true>(keys_of(x), values_of(x), x.vs, q, g, edge, limit, av.c, 0.0f, st,
                                scored);
    else
      add_page_packed<D, SPL, PACK>(x, q, g, m, edge, limit[0], av.c, nullptr, st, scored);
    ++p;
    id = id_next;
    get_values(id);
    id_next = ld_const(table, min(p + 1, p1 - 1));
  }
  unpack_rows<D, SPL, PACK>(st);
  if (m < W && qr.valid)
    write_row<D, SPL == 1>(av, sp, qr, part_of(av, sp.t0 + qr.tok, qr.head) + split, true, g,
                           st.ref[0], st.sum[0], st.o[0]);
}

// Prefixes and narrow rows' own pages in one launch, so that the long chains of loads
// of the rows, which leave the compute units mostly idle, run beside the prefixes' matrix
// products.  prefix: the workgroups of the prefixes, in front.  64 rows on 16000 positions:
// 41 us, in launches of their own 36 and 10; 256 rows in 8 groups on 2000: 38, 24 and 21.
template <int D, int SPL, int NT, int PACK, int OCC>
__global__ __launch_bounds__(256, OCC) void together_kernel(CacheView cv, RowsView rv,
                                                           GroupsView gv, AttendView av,
                                                           AttendView own, uint32_t prefix) {
  __shared__ PrefixLds<D, SPL, NT> sh;
  if (blockIdx.x < prefix)
    prefix_rows<D, SPL, NT>(cv, PrefixRows{rv, gv}, av, blockIdx.x, sh);
  else
    own_rows<D, SPL, PACK>(cv, OwnRows{rv, gv}, own,
                           __builtin_amdgcn_readfirstlane((blockIdx.x - prefix) * 4 +
                                                          (threadIdx.x >> 6)));
}

// A workgroup for 1024 / D query heads of a token, a thread for four channels of one: a
// search for the token's row and group, then its parts, 5.5 us for 183 tokens (6.4 with the
// parts' sums loaded after their references).
template <int D, bool BF16>
__global__ __launch_bounds__(256) void join_parts_kernel(CacheView cv, RowsView rv, GroupsView gv,
                                                         AttendView av, int prefix_pages,
                                                         int narrow_pages, int wide_pages) {
  const int tok = blockIdx.x;
  // (a step of a token for every row may have idle rows, whose tokens the others' follow)
  const bool same = token_each(rv) && row_start(rv, tok) == tok &&
                    (tok + 1 == rv.R || row_start(rv, tok + 1) > tok);
  const int r = same ? tok : find_row(rv.R, tok, [&](int i) __attribute__((always_inline)) {
    return row_start(rv, i);
  });
  Group x;
  const Span sp = own_span(cv, rv, gv, r, x);
  if (tok < sp.t0 || tok >= sp.t0 + sp.n) return;
  const int i = blockIdx.y * 256 + threadIdx.x, head = i / (D / 4), c4 = i % (D / 4) * 4;
  if (head >= av.Hq) return;
  const Span all = group_span(cv, rv, gv, x);
  const bool none_seen = sp.page0 < 0 || tok < all.t0 || tok >= all.t0 + all.n;
  if (none_seen && !sp.bad && threadIdx.x == 0) set_bad(av.status);
  const bool narrow = is_narrow(sp, av);
  const int per = narrow ? narrow_pages : wide_pages;
  // parts of the prefix, then those of the row's own pages: the ones that the row's
  // tile has written (a narrow row's tile ends with its last token, a wide one's with
  // the last token of its tile).  Nothing waits for none_seen's loads.
  const int n0 = (x.pages + prefix_pages - 1) / prefix_pages;
  const int rows = sp.n * av.G;
  int end = rows;
  if (!narrow) {
    const int TQ = max(av.wide_tile, 1);
    end = min(((tok - sp.t0) * av.G + head % av.G) / TQ * TQ + TQ, rows);
  }
  AttendView own = av;
  own.split_pages = per;
  const int n1 = sp.page0 < 0 ? 0 : max(splits_used(sp, own, tile_pages(sp, av.G, end)), 1);
  const int64_t part = ((int64_t)tok * av.Hq + head) * av.parts;
  const int used = n0 + n1, skip = av.part0 - n0;      // own parts begin at part0
  float top = -INFINITY, l = 0.0f;
  floatx4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  // eight parts at a time, references and sums in flight together
  constexpr int STEP = 8;
  for (int k0 = 0; k0 < used; k0 += STEP) {
    float2 ml[STEP];
    floatx4 o[STEP];
#pragma unroll
    for (int j = 0; j < STEP; ++j) {
      const int k = min(k0 + j, used - 1);
      const int64_t at = part + (k < n0 ? k : k + skip);
      ml[j] = av.part_ml[at];
      o[j] = *reinterpret_cast<const floatx4 *>(av.part_o + at * D + c4);
    }
    float next = top;
    bool large = is_large(top, av.c);
#pragma unroll
    for (int j = 0; j < STEP; ++j) {
      if (k0 + j >= used) ml[j].x = -INFINITY;
      next = fmaxf(next, ml[j].x);
      large |= is_large(ml[j].x, av.c);
    }
    auto add = [&](auto any_large) __attribute__((always_inline)) {
      auto factor = [&](float ref) __attribute__((always_inline)) {
        const float gap = origin_gap_of<decltype(any_large)::value>(ref, next, av.c);
        return ref == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(gap);
      };
      const float f = factor(top);
      l *= f;
      acc *= f;
#pragma unroll
      for (int j = 0; j < STEP; ++j) {
        const float e = factor(ml[j].x);
        if (k0 + j < used) {
          l += ml[j].y * e;
          acc += o[j] * e;
        }
      }
    };
    if (__any(large)) add(std::integral_constant<bool, true>{});
    else add(std::integral_constant<bool, false>{});
    top = next;
  }
  if (none_seen) l = 0.0f;                             // (whatever lies in its parts)
  const bool none = l == 0.0f;
  const float inv = none ? 0.0f : 1.0f / l;
  const float y[4] = {none ? 0.0f : acc[0] * inv, none ? 0.0f : acc[1] * inv,
                      none ? 0.0f : acc[2] * inv, none ? 0.0f : acc[3] * inv};
  store4<BF16>(av.out, tok * av.out_stride + head * D + c4, y);
  if (c4 == 0) finish_row(av, (int64_t)tok * av.Hq + head, top, l);
}

// Waves that are to work on the rows' own pages.
constexpr int64_t kWantWaves = 4096;
static_assert(16 * kWantWaves <= 128 * kWantGroups, "the room for parts");

// Splits at most: of four pages and more.
int64_t most_splits(int64_t pages) { return std::max<int64_t>((pages + 3) / 4, 1); }

}  // namespace

// Alone each row reads its prefix through the caches, at about 8 (units of 0.1 ns over the
// chip, 128 channels) for a page and K/V head of a row of up to 4 query rows, 10 of up to 16,
// and 46 in a tile of 64; together a page costs 23 for each tile of 32 query rows of its group,
// and some 8 us for the join and the rows' longer chain.  Rows of 64 query rows
// fill tiles by themselves.  In us, alone and together (32 query and 8 K/V heads of 128,
// bf16, one token a row if not said):
//   groups x rows, prefix        1 x 8, 1000     10  12      1 x 64, 16000          110  47
//                                1 x 8, 16000    23  26      1 x 256, 4000          100  59
//                                1 x 16, 16000   33  27      8 x 32, 2000            61  46
//                                32 x 8, 1000    41  44      16 x 4 to 16, 500-4000   75  55
//                                64 x 2, 1000    25  27      4 x 16, 3000, 4 tokens  35  45
//   1 to 6 tokens a row: 1 x 64, 16000 790 and 133, 8 x 32, 2000 246 and 108
//   8 query heads a K/V head: 4 x 32, 4000 60 and 52; fp32: 81 and 47; 256 channels 66 and 51
// From the call's bounds: groups of shorter prefixes than max_prefix gain less (prefixes of 29
// to 380, 4 x 30 to 53 rows of 1 to 4 tokens: 63 us alone, 81 as taken), and bounds far above
// what is there cost splits too (64 rows on 16000 positions with up to 380 of their own 46 us;
// with max_own 16768 60).  Of 90 shapes drawn
// over all of these 83 take the quicker way or one within 12 %; the worst take rows alone with
// two K/V heads on long prefixes, where they do not fill the chip and wait for loads instead
// (4 x 7 to 48 rows, 482-8901, 8 query heads of 64: 35.7 us, 18.4 together).
bool cache_shared_worth(const CacheView &cv, const RowsView &rv, const GroupsView &gv, int D,
                        int32_t Hq) {
  const int32_t G = Hq / cv.Hkv;
  const double rows = (double)rv.N * G, each = rows / std::max(rv.R, 1);
  if (gv.max_prefix < kPage || each >= 64.0) return false;
  // (rows of several tokens beside single ones go through tiles of 64)
  const bool wide = (int64_t)rv.max_tokens * G > 16 && (G > 16 || each > 1.5 * G);
  const double alone = (wide ? 46.0 : each > 4.0 ? 10.0 : 8.0) * rv.R;
  const double together = 23.0 * (rows / 32 + 0.5 * gv.n);
  return (alone - together) * cv.Hkv * (gv.max_prefix / kPage) * (D / 128.0) > 120e3;
}

SharedPlan cache_shared_plan(const CacheView &cv, const RowsView &rv, const GroupsView &gv, int D,
                             int32_t Hq) {
  SharedPlan p = {};
  const int32_t G = Hq / cv.Hkv;
  CacheView c = cv;
  c.weight = nullptr;
  RowsView own = rv;
  own.max_context = std::min(rv.max_context, gv.max_own);
  p.own = cache_attend_plan(c, own, D, Hq);
  const int64_t own_pages =
      std::min<int64_t>(((int64_t)own.max_context + kPage - 1) / kPage, cv.max_pages);
  if (p.own.narrow.tiles)
    // (up to 8 pages whole: 256 rows of 5 pages 46 us, in splits of 4 53; but 183 rows of up
    // to 11 in splits of 4 54, of 8 60)
    p.own.narrow = tile_plan(16 / p.own.pack, rv.R, own_pages, cv.Hkv, D, own_pages <= 8 ? 8 : 4,
                             kWantWaves);
  if (p.own.narrow.tiles && p.own.wide.tiles &&
      (int64_t)rv.N * Hq * (p.own.narrow.splits - 1) > 128 * kWantGroups) {
    // (as many parts for every token, those of the wide rows too: past the room for them)
    p.own.narrow.splits = p.own.wide.splits;
    p.own.narrow.split_pages = p.own.wide.split_pages;
  }
  const int64_t pages = std::min<int64_t>(gv.max_prefix / kPage, cv.max_pages);
  const int64_t most = std::min<int64_t>(rv.N, (int64_t)gv.max_rows * rv.max_tokens) * G;
  // (with 16 query rows of a group or fewer, in tiles of 16)
  const int tile = most <= 16 ? 16 : 32;
  p.prefix = tile_plan(tile, tile_items(gv.n, rv.N, G, tile, false), pages, cv.Hkv, D,
                       kLeastNarrow);
  p.parts = p.prefix.splits + std::max(p.own.narrow.splits, p.own.wide.splits);
  return p;
}

// Splits are made until there are kWantGroups workgroups (kWantWaves waves of rows that work
// alone), whose tiles hold at most 128 query rows (16), so N Hq s <= N Hq + 128
// kWantGroups for s splits of N tokens.
int64_t cache_shared_room(const RowsView &rv, const GroupsView &gv, int32_t Hq) {
  const int64_t rows = (int64_t)rv.N * Hq, more = rows + 128 * kWantGroups;
  const int64_t own = std::min(rv.max_context, gv.max_own);
  auto parts = [&](int64_t positions) {
    return std::min(rows * most_splits((positions + kPage - 1) / kPage), more);
  };
  return parts(gv.max_prefix) + parts(own);
}

namespace {

template <int D, int SPL, int NT>
void together_launch(const CacheView &cv, const RowsView &rv, const GroupsView &gv,
                     const AttendView &av, const AttendView &own, int pack, unsigned prefix,
                     unsigned all, hipStream_t st) {
  constexpr int OCC = NT == 1 ? (D * SPL > 384 ? 1 : D * SPL > 128 ? 2 : 3) : D < 256 ? 2 : 1;
  auto go = [&](auto p) {
    hipLaunchKernelGGL((together_kernel<D, SPL, NT, decltype(p)::value, OCC>), dim3(all), dim3(256),
                       0, st, cv, rv, gv, av, own, prefix);
  };
  if (pack == 4) go(std::integral_constant<int, 4>{});
  else if (pack == 2) go(std::integral_constant<int, 2>{});
  else go(std::integral_constant<int, 1>{});
}

template <int D, int SPL>
void shared_launch(const CacheView &cv, const RowsView &rv, const GroupsView &gv, AttendView av,
                   const SharedPlan &plan, hipStream_t st) {
  av.parts = plan.parts;
  av.part0 = 0;
  av.narrow = 0;
  av.splits = plan.prefix.splits;
  av.split_pages = plan.prefix.split_pages;
  AttendView own = av;
  own.part0 = plan.prefix.splits;
  own.narrow = plan.own.narrow_rows;
  const TilePlan &n = plan.own.narrow, &w = plan.own.wide;
  own.splits = std::max(n.splits, 1);
  own.split_pages = std::max(n.split_pages, 1);
  const unsigned prefix = (unsigned)(plan.prefix.tiles * plan.prefix.splits * cv.Hkv);
  const unsigned all = prefix + (unsigned)((n.tiles * n.splits * cv.Hkv + 3) / 4);
  if (plan.prefix.tile == 16)
    together_launch<D, SPL, 1>(cv, rv, gv, av, own, plan.own.pack, prefix, all, st);
  else
    together_launch<D, SPL, 2>(cv, rv, gv, av, own, plan.own.pack, prefix, all, st);
  if (w.tiles) {
    AttendView wide = own;
    wide.splits = w.splits;
    wide.split_pages = w.split_pages;
    wide_launch<D, SPL>(cv, OwnRows{rv, gv}, wide, w, st);
  }
  own.wide_tile = w.tile;
  hipLaunchKernelGGL((join_parts_kernel<D, SPL == 1>),
                     dim3((unsigned)rv.N, (unsigned)(((int64_t)av.Hq * (D / 4) + 255) / 256)),
                     dim3(256), 0, st, cv, rv, gv, own, plan.prefix.split_pages,
                     std::max(n.split_pages, 1), std::max(w.split_pages, 1));
}

}  // namespace

hipError_t launch_cache_shared(const CacheView &cv, const RowsView &rv, const GroupsView &gv,
                               const AttendView &av, const SharedPlan &plan, int D, bool bf16,
                               hipStream_t st) {
  auto go = [&](auto d) {
    constexpr int W = decltype(d)::value;
    if (bf16) shared_launch<W, 1>(cv, rv, gv, av, plan, st);
    else shared_launch<W, 3>(cv, rv, gv, av, plan, st);
  };
  if (D == 64) go(std::integral_constant<int, 64>{});
  else if (D == 128) go(std::integral_constant<int, 128>{});
  else go(std::integral_constant<int, 256>{});
  return hipGetLastError();
}

}  // namespace mcd
