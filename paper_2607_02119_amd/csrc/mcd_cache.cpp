// Host side of the 4-bit key/value cache: argument checks and launches.
// Nothing here allocates device memory, synchronises or throws.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <initializer_list>

#include "cache_common.h"

namespace {

mcd_status bad(const char *fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return mcd::record_error(MCD_E_INVALID, buf);
}

mcd_status launched(hipError_t e, const char *what) {
  if (e == hipSuccess) return MCD_OK;
  char buf[256];
  snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(e));
  return mcd::record_error(MCD_E_HIP, buf);
}

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
size_t round_up(size_t x) { return (x + 255) / 256 * 256; }

constexpr int64_t kMost = (int64_t)1 << 30;   // positions, items: sums stay in 32 bits

mcd_status check_cache(const mcd_cache *c) {
  if (!c) return bad("null cache");
  if (mcd_cache_page_bytes(c->D) == 0)
    return mcd::record_error(MCD_E_UNSUPPORTED, "heads of 64, 128 or 256 channels only");
  if (c->Hkv < 1 || c->Hkv > 65535 || c->n_slots < 1 || c->max_pages < 1 || c->n_pages < 1)
    return bad("bad cache sizes (Hkv=%d n_slots=%d max_pages=%d n_pages=%d)", c->Hkv, c->n_slots,
               c->max_pages, c->n_pages);
  if ((int64_t)c->max_pages * MCD_CACHE_PAGE > kMost) return bad("page table too wide");
  if ((int64_t)c->n_pages * c->Hkv > ((int64_t)1 << 40) / (int64_t)mcd_cache_page_bytes(c->D))
    return bad("cache too large");
  if (!c->pages || !c->table) return bad("null pages or table");
  if (!aligned(c->pages, 16)) return bad("pages must be 16-byte aligned");
  if (!aligned(c->table, 4) || !aligned(c->weight, 4) || !aligned(c->refs, 4))
    return bad("table, weight or refs not aligned");
  return MCD_OK;
}

mcd_status check_rows(const mcd_cache_rows *r) {
  if (!r) return bad("null rows");
  if (r->R < 0 || r->R > 65535 || r->n_tokens < 0 || r->max_tokens < 0 || r->max_context < 0 ||
      r->n_tokens > kMost || r->max_tokens > r->n_tokens || r->max_context > kMost)
    return bad("bad row sizes (R=%d n_tokens=%d max_tokens=%d max_context=%d)", r->R, r->n_tokens,
               r->max_tokens, r->max_context);
  if (r->n_tokens > 0 && (r->R == 0 || r->max_tokens == 0))
    return bad("%d tokens but R=%d, max_tokens=%d", r->n_tokens, r->R, r->max_tokens);
  if (r->R > 0 && !r->context) return bad("null context");
  if (!r->start && (r->n_tokens != r->R || (r->R > 0 && r->max_tokens != 1)))
    return bad("without start every row has one token (R=%d n_tokens=%d max_tokens=%d)", r->R,
               r->n_tokens, r->max_tokens);
  return MCD_OK;
}

mcd_status check_dtype(mcd_dtype d) {
  return d == MCD_F32 || d == MCD_BF16 ? MCD_OK : bad("bad dtype");
}

// An array of n_tokens rows of `width` elements, `stride` apart.
mcd_status check_tokens(const char *name, const void *p, int64_t stride, int64_t width,
                        mcd_dtype d) {
  const int64_t eb = d == MCD_BF16 ? 2 : 4;
  if (!p) return bad("null %s", name);
  if (stride < width || stride > kMost) return bad("%s: bad row stride", name);
  if (!aligned(p, 16) || stride * eb % 16)
    return bad("%s and its row stride must be multiples of 16 bytes", name);
  return MCD_OK;
}

// Whether n pieces of `bytes` each, a_step apart from a and b_step from b, meet.  (Each
// array's own pieces lie apart.)
bool meet(const void *a, int64_t a_step, const void *b, int64_t b_step, int64_t bytes, int64_t n) {
  uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  if (x + (n - 1) * a_step + bytes <= y || y + (n - 1) * b_step + bytes <= x) return false;
  for (int64_t i = 0, j = 0; i < n && j < n;) {
    if (x + bytes <= y) x += a_step, ++i;
    else if (y + bytes <= x) y += b_step, ++j;
    else return true;
  }
  return false;
}

mcd_status check_workspace(const void *w, size_t have, size_t need) {
  if (!w || !aligned(w, 256)) return bad("workspace must be 256-byte aligned");
  if (have < need) {
    char buf[128];
    snprintf(buf, sizeof buf, "workspace of %zu bytes, %zu needed", have, need);
    return mcd::record_error(MCD_E_WORKSPACE, buf);
  }
  return MCD_OK;
}

mcd::CacheView view(const mcd_cache *c) {
  return mcd::CacheView{c->Hkv, c->n_slots, c->max_pages, c->n_pages,
                        static_cast<uint8_t *>(c->pages), c->table, c->weight, c->refs};
}

mcd::RowsView view(const mcd_cache_rows *r) {
  return mcd::RowsView{r->R, r->n_tokens, r->max_tokens, r->max_context, r->slot, r->context,
                       r->start};
}

bool heads_ok(int32_t Hq, int32_t Hkv) { return Hq >= 1 && Hq % Hkv == 0; }

// Workspace: status, {reference, sum} of partial results, their sums, row statistics,
// kept scores.
size_t ml_bytes(const mcd::AttendPlan &p) { return round_up(p.narrow.ml_bytes + p.wide.ml_bytes); }
size_t o_bytes(const mcd::AttendPlan &p) { return round_up(p.narrow.o_bytes + p.wide.o_bytes); }
size_t attend_bytes(const mcd::AttendPlan &p) {
  return mcd::kStatusBytes + ml_bytes(p) + o_bytes(p) + round_up(p.stat_bytes) +
         round_up(p.score_bytes);
}

// What a call asks for: enough for every step within the rows' bounds.
size_t workspace_need(const mcd::AttendPlan &p, const mcd::CacheView &cv, const mcd::RowsView &rv,
                      int D, int32_t Hq) {
  return std::max(attend_bytes(p), attend_bytes(mcd::cache_attend_room(cv, rv, D, Hq)));
}

mcd_status check_pages(const mcd_cache_pages *p) {
  if (!p) return bad("null pages");
  if (p->n_slots < 1 || p->max_pages < 1 || p->n_pages < 1)
    return bad("bad page sizes (n_slots=%d max_pages=%d n_pages=%d)", p->n_slots, p->max_pages,
               p->n_pages);
  if ((int64_t)p->max_pages * MCD_CACHE_PAGE > kMost) return bad("page table too wide");
  if ((int64_t)p->n_slots * p->max_pages > ((int64_t)1 << 36)) return bad("page table too large");
  if (!p->table || !p->refs) return bad("null table or refs");
  if (!aligned(p->table, 4) || !aligned(p->refs, 4)) return bad("table or refs not aligned");
  return MCD_OK;
}

mcd::PagesView view(const mcd_cache_pages *p) {
  return mcd::PagesView{p->n_slots, p->max_pages, p->n_pages, p->table, p->refs};
}

size_t reserve_bytes(const mcd::ReserveRoom &p) {
  return mcd::kStatusBytes + p.row_bytes + p.block_bytes + p.chunk_bytes + p.bit_bytes;
}

// Arrays that a call reads and writes; nothing where there is no array.
struct Bytes {
  const void *p;
  int64_t n;
};
bool overlap(const Bytes &a, const Bytes &b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return x && y && a.n > 0 && b.n > 0 && x < y + b.n && y < x + a.n;
}
Bytes table_of(const mcd_cache_pages *p) {
  return Bytes{p->table, (int64_t)p->n_slots * p->max_pages * 4};
}
Bytes refs_of(const mcd_cache_pages *p) { return Bytes{p->refs, (int64_t)p->n_pages * 4}; }

// Rows' arrays of whole numbers that a call on page tables reads.
mcd_status check_page_rows(const mcd_cache_pages *p, int32_t R,
                           std::initializer_list<const int32_t *> rows) {
  if (R < 0 || R > 65535) return bad("bad row sizes (R=%d)", R);
  if (overlap(table_of(p), refs_of(p))) return bad("table and refs overlap");
  for (const int32_t *x : rows) {
    if (!aligned(x, 4)) return bad("array not aligned");
    if (overlap(table_of(p), Bytes{x, (int64_t)R * 4}) ||
        overlap(refs_of(p), Bytes{x, (int64_t)R * 4}))
      return bad("table and refs must not overlap the rows' arrays");
  }
  return MCD_OK;
}

mcd_status check_groups(const mcd_cache_groups *g, const mcd_cache_rows *r) {
  if (!g) return bad("null groups");
  if (g->n < 0 || g->n > 65535 || g->max_rows < 0 || g->max_prefix < 0 || g->max_own < 0 ||
      g->max_prefix > kMost || g->max_own > kMost)
    return bad("bad group sizes (n=%d max_rows=%d max_prefix=%d max_own=%d)", g->n, g->max_rows,
               g->max_prefix, g->max_own);
  if (r->n_tokens == 0) return MCD_OK;
  if ((int64_t)std::min(g->max_rows, r->R) * r->max_tokens * g->n < r->n_tokens ||
      (int64_t)r->R * r->max_tokens < r->n_tokens)
    return bad("%d groups of %d rows, %d in all, of %d tokens do not hold %d", g->n, g->max_rows,
               r->R, r->max_tokens, r->n_tokens);
  if (!g->start || !g->prefix) return bad("null array");
  if (!aligned(g->start, 4) || !aligned(g->prefix, 4)) return bad("array not aligned");
  return MCD_OK;
}

mcd::GroupsView view(const mcd_cache_groups *g) {
  return mcd::GroupsView{g->n, g->max_rows, g->max_prefix, g->max_own, g->start, g->prefix};
}

size_t shared_bytes(int64_t parts, int D) {
  return mcd::kStatusBytes + round_up((size_t)parts * sizeof(float2)) +
         round_up((size_t)parts * D * sizeof(float));
}

// Enough for every step within the bounds, together or each row on its own.
size_t shared_need(const mcd::CacheView &cv, const mcd::RowsView &rv, const mcd::GroupsView &gv,
                   int D, int32_t Hq) {
  return std::max(workspace_need(mcd::cache_attend_plan(cv, rv, D, Hq), cv, rv, D, Hq),
                  shared_bytes(mcd::cache_shared_room(rv, gv, Hq), D));
}

#define CHECK(x)                        \
  do {                                  \
    const mcd_status s_ = (x);          \
    if (s_ != MCD_OK) return s_;        \
  } while (0)

mcd_status check_attend(const mcd_cache *c, const mcd_cache_attend_args *a) {
  CHECK(check_dtype(a->dtype));
  if (!heads_ok(a->Hq, c->Hkv)) return bad("Hq=%d is no multiple of Hkv=%d", a->Hq, c->Hkv);
  if (!(a->scale > 0.0f) || !std::isfinite(a->scale)) return bad("scale must be > 0 and finite");
  if (!aligned(a->weight_out, 4) || !aligned(a->lse, 4)) return bad("weight_out or lse not aligned");
  return MCD_OK;
}

mcd_status check_query(const mcd_cache *c, const mcd_cache_rows *r, const mcd_cache_attend_args *a) {
  const int64_t width = (int64_t)a->Hq * c->D;
  if (r->n_tokens * (int64_t)a->Hq > kMost || width > kMost) return bad("too many query rows");
  CHECK(check_tokens("q", a->q, a->q_stride, width, a->dtype));
  CHECK(check_tokens("out", a->out, a->out_stride, width, a->dtype));
  // a query row is read before its own output is written, and again after it for
  // the received weight
  const int64_t eb = a->dtype == MCD_BF16 ? 2 : 4;
  const bool in_place = a->q == a->out && a->q_stride == a->out_stride && !a->weight_out;
  if (!in_place && meet(a->q, a->q_stride * eb, a->out, a->out_stride * eb, width * eb,
                        r->n_tokens))
    return bad("out must not overlap q%s", a->weight_out ? " with weight_out" : "");
  return MCD_OK;
}

// The queries, without the workspace and what each launch sets.
mcd::AttendView query_view(const mcd_cache *c, const mcd_cache_attend_args *a) {
  mcd::AttendView av = {};
  av.Hq = a->Hq;
  av.G = a->Hq / c->Hkv;
  av.q = a->q;
  av.out = a->out;
  av.q_stride = a->q_stride;
  av.out_stride = a->out_stride;
  av.c = a->scale * 1.4426950408889634f;
  av.lse = a->lse;
  return av;
}

mcd_status move_tokens(const mcd_cache *c, const mcd_cache_rows *r, mcd_dtype d, const void *k,
                       int64_t ks, const void *v, int64_t vs, void *ws, size_t wb) {
  CHECK(check_cache(c));
  CHECK(check_rows(r));
  CHECK(check_dtype(d));
  if (r->n_tokens == 0) return MCD_OK;
  const int64_t width = (int64_t)c->Hkv * c->D;
  CHECK(check_tokens("k", k, ks, width, d));
  CHECK(check_tokens("v", v, vs, width, d));
  return check_workspace(ws, wb, mcd::kStatusBytes);
}

}  // namespace

extern "C" {

size_t mcd_cache_page_bytes(int32_t D) {
  return D == 64 || D == 128 || D == 256 ? (size_t)mcd::cache_page_bytes(D) : 0;
}

size_t mcd_cache_workspace_bytes(const mcd_cache *c, const mcd_cache_rows *r, int32_t Hq) {
  if (check_cache(c) != MCD_OK || check_rows(r) != MCD_OK) return 0;
  if (!heads_ok(Hq, c->Hkv)) {
    bad("Hq=%d is no multiple of Hkv=%d", Hq, c->Hkv);
    return 0;
  }
  const mcd::CacheView cv = view(c);
  const mcd::RowsView rv = view(r);
  return workspace_need(mcd::cache_attend_plan(cv, rv, c->D, Hq), cv, rv, c->D, Hq);
}

mcd_status mcd_cache_append(const mcd_cache *c, const mcd_cache_rows *r, mcd_dtype d,
                            const void *k, int64_t ks, const void *v, int64_t vs, void *ws,
                            size_t wb, hipStream_t stream) {
  CHECK(move_tokens(c, r, d, k, ks, v, vs, ws, wb));
  if (r->n_tokens == 0) return MCD_OK;
  return launched(mcd::launch_cache_append(view(c), view(r), c->D, d == MCD_BF16, k, ks, v, vs,
                                           static_cast<uint32_t *>(ws), stream),
                  "cache append launch");
}

mcd_status mcd_cache_read(const mcd_cache *c, const mcd_cache_rows *r, mcd_dtype d, void *k,
                          int64_t ks, void *v, int64_t vs, void *ws, size_t wb,
                          hipStream_t stream) {
  CHECK(move_tokens(c, r, d, k, ks, v, vs, ws, wb));
  if (r->n_tokens == 0) return MCD_OK;
  return launched(mcd::launch_cache_read(view(c), view(r), c->D, d == MCD_BF16, k, ks, v, vs,
                                         static_cast<uint32_t *>(ws), stream),
                  "cache read launch");
}

mcd_status mcd_cache_attend(const mcd_cache *c, const mcd_cache_rows *r,
                            const mcd_cache_attend_args *a, hipStream_t stream) {
  CHECK(check_cache(c));
  CHECK(check_rows(r));
  if (!a) return bad("null args");
  CHECK(check_attend(c, a));
  // (at most 2^31 slots x 2^16 heads x 2^30 positions: counted in double)
  const double weights = 4.0 * c->n_slots * c->Hkv * c->max_pages * MCD_CACHE_PAGE;
  const double apart = std::fabs((double)reinterpret_cast<uintptr_t>(a->weight_out) -
                                 (double)reinterpret_cast<uintptr_t>(c->weight));
  if (a->weight_out && c->weight && apart > 0.0 && apart < weights)
    return bad("weight_out must be the cache's weight or apart from it");
  if (r->n_tokens == 0) {
    if (r->R == 0 || !a->weight_out || a->weight_out == c->weight) return MCD_OK;
    return launched(mcd::launch_cache_keep_weight(view(c), view(r), a->weight_out, stream),
                    "cache weight launch");
  }
  CHECK(check_query(c, r, a));
  const mcd::CacheView cv = view(c);
  const mcd::RowsView rv = view(r);
  const mcd::AttendPlan p = mcd::cache_attend_plan(cv, rv, c->D, a->Hq);
  if (std::max(p.narrow.tiles * p.narrow.splits, p.wide.tiles * p.wide.splits) * c->Hkv >
      mcd::kMostGroups)
    return bad("too many query rows");
  CHECK(check_workspace(a->workspace, a->workspace_bytes,
                        workspace_need(p, cv, rv, c->D, a->Hq)));
  char *w = static_cast<char *>(a->workspace);
  mcd::AttendView av = query_view(c, a);
  av.weight_out = a->weight_out;
  av.status = reinterpret_cast<uint32_t *>(w);
  w += mcd::kStatusBytes;
  av.part_ml = reinterpret_cast<float2 *>(w);
  w += ml_bytes(p);
  av.part_o = reinterpret_cast<float *>(w);
  w += o_bytes(p);
  av.stats = a->weight_out ? reinterpret_cast<float2 *>(w) : nullptr;
  w += round_up(p.stat_bytes);
  av.scores = a->weight_out && p.score_bytes ? reinterpret_cast<mcd::floatx4 *>(w) : nullptr;
  av.score_pages = p.score_pages;
  av.narrow = p.narrow_rows;
  return launched(mcd::launch_cache_attend(cv, rv, av, p, c->D, a->dtype == MCD_BF16, stream),
                  "cache attention launch");
}

mcd_status mcd_cache_evict(const mcd_cache *from, const mcd_cache *to,
                           const mcd_cache_evict_args *a, hipStream_t stream) {
  CHECK(check_cache(from));
  CHECK(check_cache(to));
  if (!a) return bad("null args");
  if (from->Hkv != to->Hkv || from->D != to->D)
    return bad("caches of different heads (%d x %d, %d x %d)", from->Hkv, from->D, to->Hkv, to->D);
  if (a->R < 0 || a->R > 65535 || a->max_length < 0 || a->max_length > kMost || a->keep < 1 ||
      a->recent < 0 || a->recent > a->keep)
    return bad("bad sizes (R=%d max_length=%d keep=%d recent=%d)", a->R, a->max_length, a->keep,
               a->recent);
  if (a->R == 0) return MCD_OK;
  if (a->R > to->n_slots) return bad("%d rows into %d slots", a->R, to->n_slots);
  if (!a->length || !a->kept || !a->length_out) return bad("null array");
  if (!from->weight && a->keep < a->max_length) return bad("eviction needs the cache's weights");
  CHECK(check_workspace(a->workspace, a->workspace_bytes, mcd::kStatusBytes));
  // every head's workgroup of a row reads its slot and length, one writes length_out
  const int64_t rows = (int64_t)a->R * 4, most = (int64_t)1 << 60;
  const int64_t kept = rows * from->Hkv > most / a->keep ? most : rows * from->Hkv * a->keep;
  const auto apart = [](const int32_t *x, int64_t nx, const int32_t *y, int64_t ny) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(x), q = reinterpret_cast<uintptr_t>(y);
    return !x || !y || p + nx <= q || q + ny <= p;
  };
  if (!apart(a->length_out, rows, a->length, rows) || !apart(a->length_out, rows, a->slot, rows) ||
      !apart(a->kept, kept, a->length, rows) || !apart(a->kept, kept, a->slot, rows) ||
      !apart(a->kept, kept, a->length_out, rows))
    return bad("kept and length_out must overlap neither each other nor length and slot");
  const mcd::EvictView ev{a->R, a->max_length, a->keep, a->recent, a->slot, a->length, a->kept,
                          a->length_out, static_cast<uint32_t *>(a->workspace)};
  return launched(mcd::launch_cache_evict(view(from), view(to), ev, from->D, stream),
                  "cache eviction launch");
}

size_t mcd_cache_shared_workspace_bytes(const mcd_cache *c, const mcd_cache_rows *r,
                                        const mcd_cache_groups *g, int32_t Hq) {
  if (check_cache(c) != MCD_OK || check_rows(r) != MCD_OK || check_groups(g, r) != MCD_OK) return 0;
  if (!heads_ok(Hq, c->Hkv)) {
    bad("Hq=%d is no multiple of Hkv=%d", Hq, c->Hkv);
    return 0;
  }
  if (r->n_tokens * (int64_t)Hq > kMost) {
    bad("too many query rows");
    return 0;
  }
  mcd::CacheView cv = view(c);
  cv.weight = nullptr;                           // (nothing is added up)
  const mcd::RowsView rv = view(r);
  const mcd::GroupsView gv = view(g);
  return shared_need(cv, rv, gv, c->D, Hq);
}

mcd_status mcd_cache_attend_shared(const mcd_cache *c, const mcd_cache_rows *r,
                                   const mcd_cache_groups *g, const mcd_cache_attend_args *a,
                                   hipStream_t stream) {
  return mcd_cache_attend_route(c, r, g, a, -1, stream);
}

mcd_status mcd_cache_attend_route(const mcd_cache *c, const mcd_cache_rows *r,
                                  const mcd_cache_groups *g, const mcd_cache_attend_args *a,
                                  int32_t way, hipStream_t stream) {
  CHECK(check_cache(c));
  CHECK(check_rows(r));
  CHECK(check_groups(g, r));
  if (!a) return bad("null args");
  if (a->weight_out)
    return mcd::record_error(MCD_E_UNSUPPORTED, "no weight_out for rows that share pages");
  mcd_cache alone = *c;
  alone.weight = nullptr;                        // (nothing is added up)
  CHECK(check_attend(c, a));
  if (r->n_tokens == 0) return MCD_OK;
  CHECK(check_query(c, r, a));
  const mcd::CacheView cv = view(&alone);
  const mcd::RowsView rv = view(r);
  const mcd::GroupsView gv = view(g);
  CHECK(check_workspace(a->workspace, a->workspace_bytes, shared_need(cv, rv, gv, c->D, a->Hq)));
  if (way < 0) way = mcd::cache_shared_worth(cv, rv, gv, c->D, a->Hq) ? 1 : 0;
  mcd::SharedPlan p = {};
  if (way) {
    p = mcd::cache_shared_plan(cv, rv, gv, c->D, a->Hq);
    const int64_t both = p.prefix.tiles * p.prefix.splits +
                         (p.own.narrow.tiles * p.own.narrow.splits + 3) / 4;
    // (the launches' grids, the join's with them)
    if (std::max(both, p.own.wide.tiles * p.own.wide.splits) * c->Hkv > mcd::kMostGroups ||
        rv.N > mcd::kMostGroups || (int64_t)a->Hq * c->D > (int64_t)65535 * 1024)
      way = 0;
  }
  if (!way) return mcd_cache_attend(&alone, r, a, stream);
  char *w = static_cast<char *>(a->workspace);
  mcd::AttendView av = query_view(c, a);
  av.status = reinterpret_cast<uint32_t *>(w);
  w += mcd::kStatusBytes;
  av.part_ml = reinterpret_cast<float2 *>(w);
  w += round_up((size_t)rv.N * a->Hq * p.parts * sizeof(float2));
  av.part_o = reinterpret_cast<float *>(w);
  return launched(mcd::launch_cache_shared(cv, rv, gv, av, p, c->D, a->dtype == MCD_BF16, stream),
                  "shared cache attention launch");
}

size_t mcd_cache_pages_workspace_bytes(const mcd_cache_pages *p, int32_t R) {
  if (check_pages(p) != MCD_OK || check_page_rows(p, R, {}) != MCD_OK) return 0;
  return reserve_bytes(mcd::reserve_room(R, p->n_pages));
}

mcd_status mcd_cache_count(const mcd_cache_pages *p, void *ws, size_t wb, hipStream_t stream) {
  CHECK(check_pages(p));
  CHECK(check_page_rows(p, 0, {}));
  CHECK(check_workspace(ws, wb, mcd::kStatusBytes));
  return launched(mcd::launch_cache_count(view(p), static_cast<uint32_t *>(ws), stream),
                  "page count launch");
}

mcd_status mcd_cache_release(const mcd_cache_pages *p, int32_t R, const int32_t *slot,
                             const int32_t *length, void *ws, size_t wb, hipStream_t stream) {
  CHECK(check_pages(p));
  CHECK(check_page_rows(p, R, {slot, length}));
  if (R == 0) return MCD_OK;
  CHECK(check_workspace(ws, wb, mcd::kStatusBytes));
  return launched(mcd::launch_cache_release(view(p), R, slot, length, static_cast<uint32_t *>(ws),
                                            stream),
                  "page release launch");
}

mcd_status mcd_cache_share(const mcd_cache_pages *p, int32_t R, const int32_t *slot,
                           const int32_t *source, const int32_t *length, void *ws, size_t wb,
                           hipStream_t stream) {
  CHECK(check_pages(p));
  CHECK(check_page_rows(p, R, {slot, source, length}));
  if (R == 0) return MCD_OK;
  if (!source || !length) return bad("null array");
  CHECK(check_workspace(ws, wb, mcd::kStatusBytes));
  return launched(mcd::launch_cache_share(view(p), R, slot, source, length,
                                          static_cast<uint32_t *>(ws), stream),
                  "page share launch");
}

mcd_status mcd_cache_reserve(const mcd_cache_pages *p, const mcd_cache_reserve_args *a,
                             hipStream_t stream) {
  CHECK(check_pages(p));
  if (!a) return bad("null args");
  CHECK(check_page_rows(p, a->R, {a->slot, a->context, a->tokens}));
  if (a->n_tokens < 0 || a->max_tokens < 0 || a->max_context < 0 || a->n_tokens > kMost ||
      a->max_tokens > a->n_tokens || a->max_context > kMost)
    return bad("bad row sizes (R=%d n_tokens=%d max_tokens=%d max_context=%d)", a->R, a->n_tokens,
               a->max_tokens, a->max_context);
  if (a->R == 0) return a->n_tokens ? bad("%d tokens but R=0", a->n_tokens) : MCD_OK;
  if (!a->context || !a->tokens || !a->start) return bad("null array");
  if (!aligned(a->start, 4) || !aligned(a->where, 8) || !aligned(a->row, 4) ||
      !aligned(a->position, 4))
    return bad("array not aligned");
  const mcd::ReserveRoom room = mcd::reserve_room(a->R, p->n_pages);
  CHECK(check_workspace(a->workspace, a->workspace_bytes, reserve_bytes(room)));
  const int64_t rows = (int64_t)a->R * 4, N = a->n_tokens;
  const Bytes out[] = {{a->start, rows + 4}, {a->where, 8 * N}, {a->row, 4 * N},
                       {a->position, 4 * N}};
  const Bytes in[] = {{a->slot, rows}, {a->context, rows}, {a->tokens, rows}, table_of(p),
                      refs_of(p)};
  for (int i = 0; i < 4; ++i) {
    for (const Bytes &x : in)
      if (overlap(out[i], x)) return bad("the arrays written must not overlap those read");
    for (int k = 0; k < i; ++k)
      if (overlap(out[i], out[k])) return bad("the arrays written must not overlap each other");
  }
  char *w = static_cast<char *>(a->workspace);
  mcd::ReserveView rv = {};
  rv.R = a->R;
  rv.N = a->n_tokens;
  rv.max_tokens = a->max_tokens;
  rv.max_context = a->max_context;
  rv.slot = a->slot;
  rv.context = a->context;
  rv.tokens = a->tokens;
  rv.start = a->start;
  rv.where = a->where;
  rv.row = a->row;
  rv.position = a->position;
  rv.status = reinterpret_cast<uint32_t *>(w);
  w += mcd::kStatusBytes;
  rv.row_sum = reinterpret_cast<mcd::RowSum *>(w);
  w += room.row_bytes;
  rv.block_sum = reinterpret_cast<mcd::RowSum *>(w);
  w += room.block_bytes;
  rv.chunk_free = reinterpret_cast<int32_t *>(w);
  w += room.chunk_bytes;
  rv.free_bits = reinterpret_cast<uint64_t *>(w);
  rv.row_blocks = room.row_blocks;
  rv.chunks = room.chunks;
  rv.chunk_words = room.chunk_words;
  return launched(mcd::launch_cache_reserve(view(p), rv, stream), "page reserve launch");
}

}  // extern "C"
