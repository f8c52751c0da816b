// The 4-bit key/value cache (mcd.h, mcd_cache): what its kernels share.  Views
// passed by value, a row's slot and span checked against the cache's and the
// call's bounds, page addresses, and where a page keeps which code and scale.
#pragma once

#include "gemm_common.h"

namespace mcd {

constexpr int kPage = MCD_CACHE_PAGE;

__host__ __device__ constexpr int cache_page_bytes(int D) { return 66 * D + 2 * kPage; }

struct CacheView {
  int32_t Hkv, n_slots, max_pages, n_pages;
  uint8_t *pages;
  const int32_t *table;
  float *weight;
  const int32_t *refs;
};

struct RowsView {
  static constexpr bool kParts = false;
  int32_t R, N, max_tokens, max_context;
  const int32_t *slot, *context, *start;
};

struct AttendView {
  int32_t Hq, G;               // query heads; of one K/V head
  const void *q;
  void *out;
  int64_t q_stride, out_stride;
  float c;                     // scale * log2(e): softmax in powers of two
  float *lse;                  // the caller's, or null
  float2 *stats;               // workspace [N][Hq] {reference, 1 / sum}, or null: no weights
  float *weight_out;
  // workspace [R][Hkv][score_pages][64 16 / pack], or null: narrow rows' q . k as
  // add_page_packed's lanes hold them, for the received weight
  floatx4 *scores;
  int32_t score_pages;
  // Partial results of rows whose pages are split over workgroups: for each
  // query row of a tile and split {reference, sum} and D sums.
  float2 *part_ml;
  float *part_o;
  int32_t splits, split_pages; // pages of a split: the workgroups of a tile
  // of rows whose results are parts (Rows::kParts): parts of a query row, and the first
  int32_t parts, part0;
  int32_t wide_tile;           // query rows of the wide rows' tiles
  int32_t narrow;              // query rows of a narrow row at most, 0: no narrow rows
  uint32_t *status;
};

hipError_t launch_cache_append(const CacheView &cv, const RowsView &rv, int D, bool bf16,
                               const void *k, int64_t ks, const void *v, int64_t vs,
                               uint32_t *status, hipStream_t st);
hipError_t launch_cache_read(const CacheView &cv, const RowsView &rv, int D, bool bf16, void *k,
                             int64_t ks, void *v, int64_t vs, uint32_t *status, hipStream_t st);
// How an attention call runs, and its workspace: the rows whose query rows of a
// K/V head fit a narrow tile (of 16 rows and fewer), and the others.
struct TilePlan {
  int32_t tile;                // query rows of a tile
  int64_t tiles;               // of one K/V head, 0: none
  int32_t splits, split_pages;
  size_t ml_bytes, o_bytes;    // partial results
};
struct AttendPlan {
  int32_t pack, narrow_rows;   // tiles of tokens side by side; AttendView::narrow
  TilePlan narrow, wide;
  size_t stat_bytes, score_bytes;
  int32_t score_pages;
};
AttendPlan cache_attend_plan(const CacheView &cv, const RowsView &rv, int D, int32_t Hq);
// Only the bytes: no plan of rows within rv's bounds has more of any of them.
AttendPlan cache_attend_room(const CacheView &cv, const RowsView &rv, int D, int32_t Hq);
hipError_t launch_cache_attend(const CacheView &cv, const RowsView &rv, const AttendView &av,
                               const AttendPlan &plan, int D, bool bf16, hipStream_t st);
// weight_out of a call without a token: what the rows' positions had received.
hipError_t launch_cache_keep_weight(const CacheView &cv, const RowsView &rv, float *weight_out,
                                    hipStream_t st);
// Rows that begin with the same pages (k_cache_shared.hip).
struct GroupsView {
  int32_t n, max_rows, max_prefix, max_own;
  const int32_t *start, *prefix;
};
// Rows together: own pages as cache_attend_plan has it, the groups' pages in tiles of all
// their rows' tokens, and parts of a query row in all.
struct SharedPlan {
  AttendPlan own;
  TilePlan prefix;
  int32_t parts;
};
// Whether rows that share pages run together.
bool cache_shared_worth(const CacheView &cv, const RowsView &rv, const GroupsView &gv, int D,
                        int32_t Hq);
SharedPlan cache_shared_plan(const CacheView &cv, const RowsView &rv, const GroupsView &gv, int D,
                             int32_t Hq);
// Parts of all query rows that no plan within the bounds of rv and gv passes.
int64_t cache_shared_room(const RowsView &rv, const GroupsView &gv, int32_t Hq);
hipError_t launch_cache_shared(const CacheView &cv, const RowsView &rv, const GroupsView &gv,
                               const AttendView &av, const SharedPlan &plan, int D, bool bf16,
                               hipStream_t st);
struct EvictView {
  int32_t R, max_length, keep, recent;
  const int32_t *slot, *length;
  int32_t *kept, *length_out;
  uint32_t *status;
};
hipError_t launch_cache_evict(const CacheView &from, const CacheView &to, const EvictView &ev,
                              int D, hipStream_t st);

// Page tables (k_cache_pages.hip).
struct PagesView {
  int32_t n_slots, max_pages, n_pages;
  int32_t *table, *refs;
};
constexpr int kMostChunks = 1024;
struct RowSum {
  long long need, tokens;      // columns without a page; tokens
};
struct ReserveView {
  int32_t R, N, max_tokens, max_context;
  const int32_t *slot, *context, *tokens;
  int32_t *start;
  int64_t *where;              // this and the next two: or null
  int32_t *row, *position;
  // workspace: [R] sums of the rows before within a block, [row_blocks], free pages
  // of a chunk, and a bit for every page
  RowSum *row_sum, *block_sum;
  int32_t *chunk_free;
  uint64_t *free_bits;
  int32_t row_blocks, chunks, chunk_words;
  uint32_t *status;
};
struct ReserveRoom {
  int32_t row_blocks, chunks, chunk_words;
  size_t row_bytes, block_bytes, chunk_bytes, bit_bytes;
};
ReserveRoom reserve_room(int32_t R, int32_t n_pages);
hipError_t launch_cache_count(const PagesView &pv, uint32_t *status, hipStream_t st);
hipError_t launch_cache_release(const PagesView &pv, int32_t R, const int32_t *slot,
                                const int32_t *length, uint32_t *status, hipStream_t st);
hipError_t launch_cache_share(const PagesView &pv, int32_t R, const int32_t *slot,
                              const int32_t *source, const int32_t *length, uint32_t *status,
                              hipStream_t st);
hipError_t launch_cache_reserve(const PagesView &pv, const ReserveView &rv, hipStream_t st);

namespace {

// A row's slot and its tokens; positions and tokens past a bound are cut off
// (bad is then set), so that everything a kernel derives from a span is in
// range.
struct Span {
  int slot, ctx, t0, n;        // positions before the tokens; first token; tokens
  int len;                     // positions up to and with the last token, clamped to >= 0
  int page0;                   // first page that attention reads
  bool bad;
};

__device__ __forceinline__ Span row_span(const CacheView &cv, const RowsView &rv, int r) {
  Span s;
  s.page0 = 0;
  s.slot = rv.slot ? ld_const(rv.slot, r) : r;
  // (far beyond every bound below, and sums with it stay in 32 bits)
  s.ctx = min(max(ld_const(rv.context, r), -(1 << 30)), 1 << 30);
  int t0 = r, t1 = r + 1;
  if (rv.start) {
    t0 = ld_const(rv.start, r);
    t1 = ld_const(rv.start, r + 1);
  }
  const int a = min(max(t0, 0), rv.N), b = min(max(t1, a), rv.N);
  s.bad = a != t0 || b != t1 || b - a > rv.max_tokens;
  s.t0 = a;
  s.n = min(b - a, rv.max_tokens);
  // max_context and the table's columns are below 2^30 (host), so len is too
  const int64_t len = (int64_t)s.ctx + s.n;
  const int64_t cap = min((int64_t)rv.max_context, (int64_t)cv.max_pages * kPage);
  s.bad |= len > cap;
  s.len = (int)max((int64_t)0, min(len, cap));
  if (s.slot < 0 || s.slot >= cv.n_slots) {
    s.bad = true;
    s.slot = 0;
    s.len = 0;
  }
  return s;
}

// First token of row r in [0, N], for find_row's bases.
__device__ __forceinline__ int row_start(const RowsView &rv, int r) {
  return rv.start ? min(max(rv.start[r], 0), rv.N) : r;
}

// The row that owns work item x, where row r's items begin at base(r), which
// ascends from base(0) = 0: the last r with base(r) <= x (0 if there is none, for
// arrays that do not begin at 0).  The 64 lanes of a wave probe at once: one round
// of loads for 64 rows, two for 4096.
template <class Base>
__device__ __forceinline__ int find_row(int R, int64_t x, Base &&base) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = R;
  while (n > 1) {
    const int step = (n + 63) >> 6;
    const int at = lane * step;
    const bool below = at < n && base(lo + at) <= x;
    // (the count is unsigned: less one it has to be an int before it meets 0)
    const int last = max((int)__popcll(__ballot(below)) - 1, 0);
    lo += last * step;
    n = min(step, n - last * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// First byte of page `at` of a slot for head h, or null for a page id out of
// range and (WRITE) for a page that other entries hold too.  at is below max_pages.
template <int D, bool WRITE = false>
__device__ __forceinline__ uint8_t *page_of(const CacheView &cv, int slot, int at, int h) {
  const int id = ld_const(cv.table + (int64_t)slot * cv.max_pages, at);
  if (id < 0 || id >= cv.n_pages) return nullptr;
  if (WRITE && cv.refs && ld_const(cv.refs, id) > 1) return nullptr;
  return cv.pages + ((int64_t)id * cv.Hkv + h) * cache_page_bytes(D);
}

__device__ inline void set_bad(uint32_t *status) {
  atomicOr(status, (uint32_t)MCD_DEV_BAD_PAGE);
}

// Where token t (of its page) and channel c lie.
template <int D>
__device__ __forceinline__ int key_scale_at(int t, int block) {
  return 64 * D + ((t & 15) * (D / 32) + block) * 4 + (t >> 4);
}
template <int D>
__device__ __forceinline__ int value_scale_at(int t) {
  return 66 * D + 2 * (((t >> 2) & 3) * 16 + (t >> 4) * 4 + (t & 3));
}
// the 32-bit word of channel c among those of token group g (of four) and half h
template <int D>
__device__ __forceinline__ int value_word(int h, int g, int c) {
  const int m = c / (D / 4) * 4 + (c & 3), ct = (c & (D / 4 - 1)) >> 2;
  return 32 * D + (((h * (D / 64) + (ct >> 2)) * 64 + 16 * g + m) * 4 + (ct & 3)) * 4;
}
// nibble of token t in its words
__device__ __forceinline__ int value_nibble(int t) { return ((t >> 4) & 1) * 4 + (t & 3); }

__device__ __forceinline__ float bf16_float(uint32_t bits) { return __uint_as_float(bits << 16); }
// round to nearest even; NaN stays NaN
__device__ __forceinline__ uint32_t bf16_bits(float x) {
  const uint32_t u = __float_as_uint(x);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0x7FC0u;
  return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

// e2m1 code of x in units of scale, ties to the even code.  The limits are
// products of at most 11 bits, exact in fp32: no rounding decides a code.
__device__ __forceinline__ uint32_t e2m1_code(float x, float scale) {
  const float a = fabsf(x);
  uint32_t c = (a > 0.25f * scale) + (a >= 0.75f * scale) + (a > 1.25f * scale) +
               (a >= 1.75f * scale) + (a > 2.5f * scale) + (a >= 3.5f * scale) +
               (a > 5.0f * scale);
  return (a > 0.0f ? c : 0u) | (__float_as_uint(x) >> 31) << 3;   // (all multiples of 0 are 0)
}
// Exponent byte of a key block whose largest magnitude is top (finite).
__device__ __forceinline__ uint32_t key_scale(float top) {
  const int e = (int)((__float_as_uint(top) + 0x1FFFFFu) >> 23) - 2;
  return (uint32_t)min(max(e, 1), 254);
}
}  // namespace
}  // namespace mcd
