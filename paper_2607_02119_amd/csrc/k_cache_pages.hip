// Page tables of the 4-bit key/value cache, kept on the GPU (mcd.h, mcd_cache_pages):
// counts of the table's entries that hold a page, pages given back, shared and
// taken, and where the new tokens of a step lie.
//
// Everything here is bound by the latency of a few dependent loads and of the
// launches themselves: a step of 512 rows moves some 40 KB (release 2.8 us, reserve 7.6),
// one of 2048 rows with 300 thousand tokens 5 MB (release 3.8 to 7, share 7.4, reserve
// 3.7 and 8.0).  Counts change by atomic additions of whole numbers, and
// which page a row gets follows from ranks alone, so the same table gives the same
// pages whatever order the workgroups run in.
#include "cache_common.h"

#include <algorithm>

namespace mcd {
namespace {

constexpr int kRowBlock = 64;            // rows whose sums a workgroup of count_kernel adds up

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  return x;
}
__device__ __forceinline__ int64_t wave_sum(int64_t x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor((long long)x, d);
  return x;
}
// sum of the lanes up to and with this one
template <class T>
__device__ __forceinline__ T wave_scan(T x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const T y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

__global__ __launch_bounds__(256) void clear_kernel(int32_t *refs, int32_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) refs[i] = 0;
}

// (in turns, where the table has more entries than a launch has threads)
__global__ __launch_bounds__(256) void refs_kernel(PagesView pv, uint32_t *status) {
  const int64_t entries = (int64_t)pv.n_slots * pv.max_pages;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < entries;
       i += (int64_t)gridDim.x * 256) {
    const int id = pv.table[i];
    if (id >= pv.n_pages) set_bad(status);
    else if (id >= 0) atomicAdd(pv.refs + id, 1);
  }
}

// A row's slot, or -1 (reported).
__device__ __forceinline__ int slot_of(const PagesView &pv, const int32_t *slot, int r,
                                       uint32_t *status) {
  const int s = slot ? ld_const(slot, r) : r;
  if (s >= 0 && s < pv.n_slots) return s;
  if ((threadIdx.x & 63) == 0) set_bad(status);
  return -1;
}

// A wave for each row.  An entry is exchanged, so a slot that a call names twice
// gives its pages back once.
__global__ __launch_bounds__(256) void release_kernel(PagesView pv, int R, const int32_t *slot,
                                                      const int32_t *length, uint32_t *status) {
  const int r = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (r >= R) return;
  const int s = slot_of(pv, slot, r, status);
  if (s < 0) return;
  const int keep = length ? ld_const(length, r) : 0;
  const int first = (int)(((int64_t)keep + kPage - 1) / kPage);
  if (keep < 0 || first > pv.max_pages) {
    if ((threadIdx.x & 63) == 0) set_bad(status);
    return;
  }
  int32_t *row = pv.table + (int64_t)s * pv.max_pages;
  for (int64_t c = (int64_t)first + (threadIdx.x & 63); c < pv.max_pages; c += 64) {
    if (row[c] < 0) continue;
    const int id = atomicExch(row + c, -1);
    if (id < 0) continue;
    if (id >= pv.n_pages) {
      set_bad(status);
    } else if (atomicSub(pv.refs + id, 1) <= 0) {  // (never counted: stays at none)
      atomicAdd(pv.refs + id, 1);
      set_bad(status);
    }
  }
}

// A wave for each row.  Only an entry without a page takes one.
__global__ __launch_bounds__(256) void share_kernel(PagesView pv, int R, const int32_t *slot,
                                                    const int32_t *source, const int32_t *length,
                                                    uint32_t *status) {
  const int r = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (r >= R) return;
  const int s = slot_of(pv, slot, r, status), from = slot_of(pv, source, r, status);
  if (s < 0 || from < 0) return;
  const int n = ld_const(length, r);
  const int pages = min(max(n, 0) / kPage, pv.max_pages);
  bool bad = n < 0 || max(n, 0) / kPage > pv.max_pages;
  int32_t *to = pv.table + (int64_t)s * pv.max_pages;
  const int32_t *row = pv.table + (int64_t)from * pv.max_pages;
  for (int c = threadIdx.x & 63; c < pages; c += 64) {
    const int id = row[c], old = to[c];
    if (id < 0 || id >= pv.n_pages || old >= 0 || atomicCAS(to + c, old, id) != old) bad = true;
    else atomicAdd(pv.refs + id, 1);
  }
  if (bad) set_bad(status);
}

// ---- new tokens -----------------------------------------------------------------

// A row's positions: its tokens as asked for, and of those positions the ones that
// the table and the call's bounds hold.
struct Want {
  int slot;                    // -1: none
  int64_t ctx, end;            // positions before and after the tokens
  int64_t cap;                 // positions are in [0, cap)
  int p0, p1;                  // columns of the positions in range
  bool bad;
};

__device__ __forceinline__ Want want_of(const PagesView &pv, const ReserveView &rv, int r) {
  Want w;
  w.slot = rv.slot ? rv.slot[r] : r;
  w.ctx = rv.context[r];
  const int t = rv.tokens[r], n = min(max(t, 0), rv.max_tokens);
  w.end = w.ctx + n;
  w.cap = min((int64_t)rv.max_context, (int64_t)pv.max_pages * kPage);
  w.bad = n != t || w.slot < 0 || w.slot >= pv.n_slots || w.ctx < 0 || w.end > w.cap;
  if (w.slot < 0 || w.slot >= pv.n_slots) w.slot = -1;
  const int64_t a = max(w.ctx, (int64_t)0), b = min(w.end, w.cap);
  const bool some = w.slot >= 0 && n > 0 && a < b;
  w.p0 = some ? (int)(a / kPage) : 0;
  w.p1 = some ? (int)((b + kPage - 1) / kPage) : 0;
  return w;
}

// First of two launches.  Workgroups below row_blocks: for kRowBlock rows the
// columns that need a page and the tokens, as sums of the rows before within the
// block, and the blocks' sums; LANES lanes to a row.  The others: a bit for every
// page of a chunk, set where no entry holds it, and the chunk's count.
template <int LANES>
__global__ __launch_bounds__(256) void count_kernel(PagesView pv, ReserveView rv) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if ((int)blockIdx.x < rv.row_blocks) {
    __shared__ int need[kRowBlock], tokens[kRowBlock];
    constexpr int AT_ONCE = 256 / LANES;
    const int l = threadIdx.x % LANES;
    for (int i = threadIdx.x / LANES; i < kRowBlock; i += AT_ONCE) {
      const int r = blockIdx.x * kRowBlock + i;
      int n = 0, t = 0;
      if (r < rv.R) {
        const Want w = want_of(pv, rv, r);
        const int32_t *row = pv.table + (int64_t)max(w.slot, 0) * pv.max_pages;
#pragma unroll 4
        for (int c = w.p0 + l; c < w.p1; c += LANES) n += row[c] < 0;
        t = (int)(w.end - w.ctx);
        if (w.bad && l == 0) set_bad(rv.status);
      }
#pragma unroll
      for (int d = LANES / 2; d > 0; d >>= 1) n += __shfl_xor(n, d);
      if (l == 0) {
        need[i] = n;
        tokens[i] = t;
      }
    }
    __syncthreads();
    if (wave) return;
    const long long n = need[lane], t = tokens[lane];
    const long long ns = wave_scan(n), ts = wave_scan(t);
    const int r = blockIdx.x * kRowBlock + lane;
    if (r < rv.R) rv.row_sum[r] = RowSum{ns - n, ts - t};
    if (lane == 63) rv.block_sum[blockIdx.x] = RowSum{ns, ts};
    return;
  }
  __shared__ int part[4];
  const int chunk = blockIdx.x - rv.row_blocks;
  int count = 0;
#pragma unroll 4
  for (int i = wave; i < rv.chunk_words; i += 4) {
    const int64_t word = (int64_t)chunk * rv.chunk_words + i, page = word * 64 + lane;
    const uint64_t bits = __ballot(page < pv.n_pages && pv.refs[min(page, (int64_t)pv.n_pages - 1)] <= 0);
    if (lane == 0) rv.free_bits[word] = bits;
    count += __popcll(bits);
  }
  if (lane == 0) part[wave] = count;
  __syncthreads();
  if (threadIdx.x == 0) rv.chunk_free[chunk] = part[0] + part[1] + part[2] + part[3];
}

// Position of the k-th set bit of x (k below its count).
__device__ __forceinline__ int select_bit(uint64_t x, int k) {
  int at = 0;
#pragma unroll
  for (int w = 32; w > 0; w >>= 1) {
    const int low = __popcll(x & ((1ull << w) - 1));
    if (k >= low) {
      k -= low;
      x >>= w;
      at += w;
    }
  }
  return at;
}

// The free pages of ranks first, first + 1, ..., one for every lane whose `rank` is
// among the `count` of them (a wave together; lanes without one: rank < 0); -1 from
// the rank of the last free page on.
// counts: the first 64 chunks'.
__device__ __forceinline__ int free_pages(const ReserveView &rv, int counts, int64_t first,
                                          int count, int64_t rank) {
  const int lane = threadIdx.x & 63;
  const int64_t end = first + count;
  int page = -1;
  int64_t before = 0;                            // free pages of the chunks so far
  for (int c0 = 0; c0 < rv.chunks && before < end; c0 += 64) {
    const int free = c0 == 0 ? counts : c0 + lane < rv.chunks ? rv.chunk_free[c0 + lane] : 0;
    const int upto = wave_scan(free), all = __shfl(upto, 63);
    // the chunks of these 64 that hold one of the ranks
    uint64_t holds = __ballot(free > 0 && before + upto > first && before + upto - free < end);
    while (holds) {
      const int k = __builtin_ctzll(holds);
      holds &= holds - 1;
      int64_t base = before + __shfl(upto - free, k);
      const int64_t chunk = c0 + k;
      for (int w0 = 0; w0 < rv.chunk_words; w0 += 64) {
        const int64_t word = chunk * rv.chunk_words + w0 + lane;
        const uint64_t bits = w0 + lane < rv.chunk_words ? rv.free_bits[word] : 0;
        const int n = __popcll(bits), so_far = wave_scan(n), total = __shfl(so_far, 63);
        const bool mine = rank >= base && rank < base + total;
        const int nth = mine ? (int)(rank - base) : 0;
        // the first lane with so_far > nth
        int from = 0;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1)
          if (__shfl(so_far, from + d - 1) <= nth) from += d;
        const uint64_t found = __shfl((unsigned long long)bits, from & 63);
        const int skipped = __shfl(so_far - n, from & 63);
        if (mine)
          page = (int)((chunk * rv.chunk_words + w0 + from) * 64 + select_bit(found, nth - skipped));
        base += total;
      }
    }
    before += all;
  }
  return page;
}

// Second launch: the rows' pages and their tokens' places.  A wave for each row, or
// (WIDE, rows of many tokens) a workgroup whose first wave sees to the pages.
template <bool WIDE>
__global__ __launch_bounds__(256) void reserve_kernel(PagesView pv, ReserveView rv) {
  __shared__ int column[WIDE ? 64 : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = WIDE ? blockIdx.x
                     : __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (int)(threadIdx.x >> 6));
  if (r >= rv.R) return;
  const Want w = want_of(pv, rv, r);
  int32_t *row = pv.table + (int64_t)max(w.slot, 0) * pv.max_pages;
  // loads that wait for no sum go out first: the first columns' entries, the chunks' counts
  const int64_t c0 = w.ctx >> 6;
  auto entry = [&](int64_t c) __attribute__((always_inline)) {
    return c >= w.p0 && c < w.p1 ? row[c] : 0;
  };
  int old = entry(c0 + lane);
  const int chunks = lane < rv.chunks ? rv.chunk_free[lane] : 0;
  int64_t need = 0, first = 0;                   // ranks and tokens before the row's
  for (int b = lane; b < r / kRowBlock; b += 64) {
    need += rv.block_sum[b].need;
    first += rv.block_sum[b].tokens;
  }
  need = wave_sum(need) + rv.row_sum[r].need;
  first = wave_sum(first) + rv.row_sum[r].tokens;
  if (lane == 0 && (!WIDE || wave == 0)) {
    rv.start[r] = (int)min(first, (int64_t)rv.N);
    const int64_t last = first + (w.end - w.ctx);
    if (r == rv.R - 1) rv.start[rv.R] = (int)min(last, (int64_t)rv.N);
    if (last > rv.N) set_bad(rv.status);
  }
  // 64 columns at a time
  for (int64_t c = c0; c * kPage < w.end; c += 64) {
    int id = -1;
    if (!WIDE || wave == 0) {
      const int64_t mine = c + lane;
      const bool in = mine >= w.p0 && mine < w.p1;
      if (c != c0) old = entry(mine);
      const bool lacks = in && old < 0;
      const uint64_t lacking = __ballot(lacks);
      id = in ? old : -1;
      if (lacking) {
        const int count = __popcll(lacking);
        const int64_t rank = need + __popcll(lacking & ((1ull << lane) - 1));
        const int page = free_pages(rv, chunks, need, count, lacks ? rank : -1);
        need += count;
        if (lacks) {
          id = page;
          if (page < 0) {
            atomicOr(rv.status, (uint32_t)MCD_DEV_NO_PAGE);
          } else {
            // (a slot named twice: the page stays free)
            const int seen = atomicCAS(row + mine, old, page);
            if (seen == old) pv.refs[page] = 1;
            else id = seen, set_bad(rv.status);
          }
        }
      }
      // a page that another entry holds too, or no page of the cache
      if (id >= pv.n_pages || (in && !lacks && pv.refs[id] > 1)) {
        id = -1;
        set_bad(rv.status);
      }
      if constexpr (WIDE) column[lane] = id;
    }
    if constexpr (WIDE) __syncthreads();
    const int64_t t0 = max(w.ctx, c * kPage), t1 = min(w.end, (c + 64) * kPage);
    constexpr int STEP = WIDE ? 256 : 64;
    for (int64_t p = t0; p < t1; p += STEP) {
      const int64_t pos = p + (WIDE ? threadIdx.x : lane);
      const int at = (int)((min(pos, t1 - 1) >> 6) - c) & 63;
      const int page = WIDE ? column[at] : __shfl(id, at);
      const int64_t tok = first + (pos - w.ctx);
      if (pos >= t1 || tok >= rv.N) continue;
      const bool ok = page >= 0 && pos >= 0 && pos < w.cap;
      if (rv.where) rv.where[tok] = ok ? (int64_t)page * kPage + (pos & (kPage - 1)) : -1;
      if (rv.row) rv.row[tok] = r;
      if (rv.position) rv.position[tok] = (int)pos;
    }
    if constexpr (WIDE) __syncthreads();
  }
}

// A decode step in one launch: rows of at most kFewTokens tokens, so of one column or two,
// a thread for each, and the free pages' bits in LDS.  512 rows of one token and 3200 pages:
// 7.6 us; the two launches below take 10.6.
constexpr int kSmallRows = 1024, kSmallPages = 32768, kFewTokens = 8;

__global__ __launch_bounds__(1024) void reserve_small_kernel(PagesView pv, ReserveView rv) {
  constexpr int WORDS = kSmallPages / 64;
  __shared__ uint64_t bits[WORDS];
  __shared__ int upto[WORDS];                    // free pages up to and with a word
  __shared__ int2 sums[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = threadIdx.x;
  Want w = {};
  int32_t *row = pv.table;
  int id[2] = {-1, -1}, need = 0, tokens = 0;
  if (r < rv.R) {
    w = want_of(pv, rv, r);
    row += (int64_t)max(w.slot, 0) * pv.max_pages + w.p0;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (w.p0 + i < w.p1) {
        id[i] = row[i];
        need += id[i] < 0;
      }
    tokens = (int)(w.end - w.ctx);
  }
  const int need_to = wave_scan(need), tokens_to = wave_scan(tokens);
  if (lane == 63) sums[wave] = make_int2(need_to, tokens_to);
  __syncthreads();
  int rank = need_to - need, first = tokens_to - tokens, wanted = 0, all = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int2 x = sums[i];
    if (i < wave) {
      rank += x.x;
      first += x.y;
    }
    wanted += x.x;
    all += x.y;
  }
  const int words = (pv.n_pages + 63) / 64;
  int free = 0;
  if (wanted) {                                  // (uniform)
#pragma unroll 8
    for (int i = wave; i < words; i += 16) {
      const int page = i * 64 + lane;
      const uint64_t b = __ballot(page < pv.n_pages && pv.refs[min(page, pv.n_pages - 1)] <= 0);
      if (lane == 0) bits[i] = b;
    }
    __syncthreads();
    if (wave == 0) {                             // words in order: WORDS / 64 a lane
      constexpr int PER = WORDS / 64;
      int n = 0;
      for (int i = 0; i < PER; ++i)
        if (lane * PER + i < words) n += __popcll(bits[lane * PER + i]);
      int so_far = wave_scan(n) - n;
      for (int i = 0; i < PER; ++i) {
        if (lane * PER + i < words) so_far += __popcll(bits[lane * PER + i]);
        upto[lane * PER + i] = so_far;
      }
    }
    __syncthreads();
    free = upto[WORDS - 1];
  }
  if (r < rv.R) {
    if (w.bad) set_bad(rv.status);
    rv.start[r] = min(first, rv.N);
    if (r == rv.R - 1) {
      rv.start[rv.R] = min(all, rv.N);
      if (all > rv.N) set_bad(rv.status);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (w.p0 + i >= w.p1) continue;
      if (id[i] < 0) {
        const int old = id[i], k = rank++;
        id[i] = -1;
        if (k >= free) {
          atomicOr(rv.status, (uint32_t)MCD_DEV_NO_PAGE);
          continue;
        }
        int at = 0;                              // the first word with upto > k
#pragma unroll
        for (int d = WORDS / 2; d > 0; d >>= 1)
          if (upto[at + d - 1] <= k) at += d;
        const uint64_t b = bits[at];
        const int page = at * 64 + select_bit(b, k - (upto[at] - (int)__popcll(b)));
        // (a slot named twice: the page stays free)
        const int seen = atomicCAS(row + i, old, page);
        id[i] = seen == old ? page : seen;
        if (seen == old) pv.refs[page] = 1;
        else set_bad(rv.status);
      } else if (id[i] >= pv.n_pages || pv.refs[id[i]] > 1) {
        id[i] = -1;
        set_bad(rv.status);
      }
      if (id[i] >= pv.n_pages) id[i] = -1;
    }
    for (int t = 0; t < tokens; ++t) {
      const int tok = first + t;
      const int64_t pos = w.ctx + t;
      if (tok >= rv.N) break;
      const int page = (pos >> 6) == w.p0 ? id[0] : id[1];
      const bool ok = page >= 0 && pos >= 0 && pos < w.cap && w.p1 > w.p0;
      if (rv.where) rv.where[tok] = ok ? (int64_t)page * kPage + (pos & (kPage - 1)) : -1;
      if (rv.row) rv.row[tok] = r;
      if (rv.position) rv.position[tok] = (int)pos;
    }
  }
}

size_t round_up(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

ReserveRoom reserve_room(int32_t R, int32_t n_pages) {
  ReserveRoom p;
  p.row_blocks = (R + kRowBlock - 1) / kRowBlock;
  // chunks of 1024 pages, more where that makes more than kMostChunks of them
  int64_t pages = 1024;
  while ((n_pages + pages - 1) / pages > kMostChunks) pages *= 2;
  p.chunks = (int32_t)((n_pages + pages - 1) / pages);
  p.chunk_words = (int32_t)(pages / 64);
  p.row_bytes = round_up((size_t)R * sizeof(RowSum));
  p.block_bytes = round_up((size_t)p.row_blocks * sizeof(RowSum));
  p.chunk_bytes = round_up((size_t)p.chunks * sizeof(int32_t));
  p.bit_bytes = (size_t)p.chunks * p.chunk_words * sizeof(uint64_t);
  return p;
}

hipError_t launch_cache_count(const PagesView &pv, uint32_t *status, hipStream_t st) {
  hipLaunchKernelGGL(clear_kernel, dim3((unsigned)(((int64_t)pv.n_pages + 255) / 256)), dim3(256),
                     0, st, pv.refs, pv.n_pages);
  const int64_t entries = (int64_t)pv.n_slots * pv.max_pages;
  const int64_t groups = std::min<int64_t>((entries + 255) / 256, kMostGroups);
  hipLaunchKernelGGL(refs_kernel, dim3((unsigned)groups), dim3(256), 0, st, pv, status);
  return hipGetLastError();
}

hipError_t launch_cache_release(const PagesView &pv, int32_t R, const int32_t *slot,
                                const int32_t *length, uint32_t *status, hipStream_t st) {
  hipLaunchKernelGGL(release_kernel, dim3((unsigned)((R + 3) / 4)), dim3(256), 0, st, pv, R, slot,
                     length, status);
  return hipGetLastError();
}

hipError_t launch_cache_share(const PagesView &pv, int32_t R, const int32_t *slot,
                              const int32_t *source, const int32_t *length, uint32_t *status,
                              hipStream_t st) {
  hipLaunchKernelGGL(share_kernel, dim3((unsigned)((R + 3) / 4)), dim3(256), 0, st, pv, R, slot,
                     source, length, status);
  return hipGetLastError();
}

hipError_t launch_cache_reserve(const PagesView &pv, const ReserveView &rv, hipStream_t st) {
  if (rv.R <= kSmallRows && rv.max_tokens <= kFewTokens && pv.n_pages <= kSmallPages) {
    hipLaunchKernelGGL(reserve_small_kernel, dim3(1), dim3(1024), 0, st, pv, rv);
    return hipGetLastError();
  }
  const dim3 grid((unsigned)(rv.row_blocks + rv.chunks));
  if (rv.max_tokens > 4096)
    hipLaunchKernelGGL(count_kernel<16>, grid, dim3(256), 0, st, pv, rv);
  else
    hipLaunchKernelGGL(count_kernel<4>, grid, dim3(256), 0, st, pv, rv);
  if (rv.max_tokens > 1024)
    hipLaunchKernelGGL(reserve_kernel<true>, dim3((unsigned)rv.R), dim3(256), 0, st, pv, rv);
  else
    hipLaunchKernelGGL(reserve_kernel<false>, dim3((unsigned)((rv.R + 3) / 4)), dim3(256), 0, st,
                       pv, rv);
  return hipGetLastError();
}

}  // namespace mcd
