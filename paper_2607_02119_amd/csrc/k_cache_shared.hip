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
  static constexpr bool kParts = true;
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

// A workgroup for 1024 / D query heads of a token, a thread for four channels of one.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void join_parts_kernel(CacheView cv, RowsView rv, GroupsView gv,
                                                         AttendView av, int prefix_pages,
                                                         int narrow_pages, int wide_pages) {
  const int tok = blockIdx.x;
  const int r = token_each(rv) ? tok : find_row(rv.R, tok, [&](int i) __attribute__((always_inline)) {
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
  // the last token of its tile)
  const int n0 = none_seen ? 0 : (all.len / kPage + prefix_pages - 1) / prefix_pages;
  int n1 = 0;
  if (!none_seen) {
    const int rows = sp.n * av.G;
    int end = rows;
    if (!narrow) {
      const int TQ = max(av.wide_tile, 1);
      end = min(((tok - sp.t0) * av.G + head % av.G) / TQ * TQ + TQ, rows);
    }
    AttendView own = av;
    own.split_pages = per;
    n1 = max(splits_used(sp, own, tile_pages(sp, av.G, end)), 1);
  }
  const int64_t part = ((int64_t)tok * av.Hq + head) * av.parts;
  const int used = n0 + n1, skip = av.part0 - n0;      // own parts begin at part0
  float top = -INFINITY, l = 0.0f;
  bool large = false;
#pragma unroll 4
  for (int k = 0; k < used; ++k) {
    const float ref = av.part_ml[part + (k < n0 ? k : k + skip)].x;
    top = fmaxf(top, ref);
    large |= is_large(ref, av.c);
  }
  floatx4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  auto add = [&](auto any_large) __attribute__((always_inline)) {
#pragma unroll 4
    for (int k = 0; k < used; ++k) {
      const int64_t at = part + (k < n0 ? k : k + skip);
      const float2 ml = av.part_ml[at];
      const float gap = origin_gap_of<decltype(any_large)::value>(ml.x, top, av.c);
      const float f = ml.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(gap);
      l += ml.y * f;
      acc += *reinterpret_cast<const floatx4 *>(av.part_o + at * D + c4) * f;
    }
  };
  if (__any(large)) add(std::integral_constant<bool, true>{});
  else add(std::integral_constant<bool, false>{});
  const bool none = l == 0.0f;
  const float inv = none ? 0.0f : 1.0f / l;
  const float y[4] = {none ? 0.0f : acc[0] * inv, none ? 0.0f : acc[1] * inv,
                      none ? 0.0f : acc[2] * inv, none ? 0.0f : acc[3] * inv};
  store4<BF16>(av.out, tok * av.out_stride + head * D + c4, y);
  if (c4 == 0) finish_row(av, (int64_t)tok * av.Hq + head, top, l);
}

// Splits at most of pages that are read in splits of `per` and more.
int64_t most_splits(int64_t pages) { return std::max<int64_t>((pages + 3) / 4, 1); }

}  // namespace

SharedPlan cache_shared_plan(const CacheView &cv, const RowsView &rv, const GroupsView &gv, int D,
                             int32_t Hq) {
  SharedPlan p = {};
  const int32_t G = Hq / cv.Hkv;
  // rows that fill tiles by themselves gain nothing
  p.together = gv.max_prefix >= kPage && (int64_t)rv.N * G < (int64_t)64 * rv.R;
  if (!p.together) return p;
  CacheView c = cv;
  c.weight = nullptr;
  RowsView own = rv;
  own.max_context = std::min(rv.max_context, gv.max_own);
  p.own = cache_attend_plan(c, own, D, Hq);
  if (p.own.narrow.tiles && p.own.wide.tiles) {
    // (one number of parts for all rows: the wide rows', which is bounded by the tokens)
    p.own.narrow.splits = p.own.wide.splits;
    p.own.narrow.split_pages = p.own.wide.split_pages;
  }
  const int64_t pages = std::min<int64_t>(gv.max_prefix / kPage, cv.max_pages);
  const int64_t most = std::min<int64_t>(rv.N, (int64_t)gv.max_rows * rv.max_tokens) * G;
  p.prefix_pack = most <= 4 ? 4 : most <= 8 ? 2 : most <= 16 ? 1 : 0;
  if (p.prefix_pack) {
    p.prefix = tile_plan(16 / p.prefix_pack, gv.n, pages, cv.Hkv, D, kLeastNarrow);
  } else {
    const int tile = D == 256 || most <= 64 ? 64 : 128;
    p.prefix = tile_plan(tile, tile_items(gv.n, rv.N, G, tile, false), pages, cv.Hkv, D,
                         kLeastWide);
  }
  p.parts = p.prefix.splits + std::max(p.own.narrow.splits, p.own.wide.splits);
  p.ml_bytes = (size_t)rv.N * Hq * p.parts * sizeof(float2);
  p.o_bytes = (size_t)rv.N * Hq * p.parts * D * sizeof(float);
  return p;
}

// Splits are made until there are kWantGroups workgroups, whose tiles hold at most 128 query
// rows, so N Hq s <= N Hq + 128 kWantGroups for s splits of N tokens.
int64_t cache_shared_room(const RowsView &rv, const GroupsView &gv, int32_t Hq) {
  const int64_t rows = (int64_t)rv.N * Hq, more = rows + 128 * kWantGroups;
  const int64_t own = std::min(rv.max_context, gv.max_own);
  auto parts = [&](int64_t positions) {
    return std::min(rows * most_splits((positions + kPage - 1) / kPage), more);
  };
  return parts(gv.max_prefix) + parts(own);
}

namespace {

template <int D, int SPL>
void shared_launch(const CacheView &cv, const RowsView &rv, const GroupsView &gv, AttendView av,
                   const SharedPlan &plan, hipStream_t st) {
  av.parts = plan.parts;
  av.part0 = 0;
  av.narrow = plan.prefix_pack ? 16 / plan.prefix_pack : 0;
  av.splits = plan.prefix.splits;
  av.split_pages = plan.prefix.split_pages;
  tiles_launch<D, SPL>(cv, PrefixRows{rv, gv}, av, plan.prefix_pack, plan.prefix,
                       plan.prefix_pack != 0, st);
  av.part0 = plan.prefix.splits;
  av.narrow = plan.own.narrow_rows;
  for (const bool narrow : {true, false}) {
    const TilePlan &t = narrow ? plan.own.narrow : plan.own.wide;
    if (t.tiles == 0) continue;
    av.splits = t.splits;
    av.split_pages = t.split_pages;
    tiles_launch<D, SPL>(cv, OwnRows{rv, gv}, av, plan.own.pack, t, narrow, st);
  }
  av.wide_tile = plan.own.wide.tile;
  hipLaunchKernelGGL((join_parts_kernel<D, SPL == 1>),
                     dim3((unsigned)rv.N, (unsigned)(((int64_t)av.Hq * (D / 4) + 255) / 256)),
                     dim3(256), 0, st, cv, rv, gv, av, plan.prefix.split_pages,
                     std::max(plan.own.narrow.split_pages, 1), std::max(plan.own.wide.split_pages, 1));
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
