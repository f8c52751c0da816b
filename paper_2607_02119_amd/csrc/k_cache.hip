// The 4-bit key/value cache's pages: quantising tokens into them, reading them
// back, and eviction by received weight (mcd.h, mcd_cache).
//
// All of it moves bytes: the codes are found by comparing with exact products
// of the scale, so every result is a function of the inputs alone, bit for bit.
#include "cache_common.h"

#include <algorithm>

namespace mcd {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float float2v __attribute__((ext_vector_type(2)));

constexpr int kHalf = 32;        // tokens whose value words lie together

template <bool BF16>
__device__ __forceinline__ void load8(const void *p, int64_t at, float x[8]) {
  if constexpr (BF16) {
    const u32x4 w = *reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(p) + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  } else {
    const float4 *q = reinterpret_cast<const float4 *>(static_cast<const float *>(p) + at);
    const float4 a = q[0], b = q[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
}

// Largest magnitude of x[8] and of the lanes whose index differs in the low
// bits below W, as bits: larger than every finite number's where one is not
// finite.
template <int W>
__device__ __forceinline__ uint32_t top_bits(const float x[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
#pragma unroll
  for (int d = 1; d < W; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
  return m;
}

__device__ __forceinline__ uint32_t codes8(const float x[8], float scale) {
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) w |= e2m1_code(x[i], scale) << (4 * i);
  return w;
}

// 8 channels' codes of a key block, its scale byte; all lanes of the block's
// four take part.  A power of two is the conversion's own scale.
__device__ __forceinline__ uint32_t key_codes(const float x[8], uint32_t &byte) {
  const uint32_t top = top_bits<4>(x);
  const bool finite = top < 0x7F800000u;
  byte = finite ? key_scale(__uint_as_float(top)) : 255u;
  const float scale = __uint_as_float(byte << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
  return finite ? w : 0u;
}

// 8 channels in dtype from their codes: keys with the exponent byte as the
// conversion's scale (255: infinity, which converts to NaN), values times theirs.
template <bool BF16>
__device__ __forceinline__ void store_keys(void *p, int64_t at, uint32_t codes, uint32_t byte) {
  const float scale = __uint_as_float(byte << 23);
  if constexpr (BF16) {
    u32x4 w;
    w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
    *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(p) + at) = w;
  } else {
    const float2v a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0);
    const float2v b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
    const float2v c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2);
    const float2v d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
    float4 *q = reinterpret_cast<float4 *>(static_cast<float *>(p) + at);
    q[0] = make_float4(a[0], a[1], b[0], b[1]);
    q[1] = make_float4(c[0], c[1], d[0], d[1]);
  }
}

template <bool BF16>
__device__ __forceinline__ void store_values(void *p, int64_t at, uint32_t codes, float scale) {
  float2v x[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0),
                  __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1),
                  __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 2),
                  __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 3)};
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = float2v{x[i][0] * scale, x[i][1] * scale};
  if constexpr (BF16) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x[i], bf16x2));
    *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(p) + at) = w;
  } else {
    float4 *q = reinterpret_cast<float4 *>(static_cast<float *>(p) + at);
    q[0] = make_float4(x[0][0], x[0][1], x[1][0], x[1][1]);
    q[1] = make_float4(x[2][0], x[2][1], x[3][0], x[3][1]);
  }
}

template <int D>
__device__ __forceinline__ uint32_t value_codes(const float x[8], uint32_t &scale) {
  const uint32_t top = top_bits<D / 8>(x);
  const bool finite = top < 0x7F800000u;
  scale = finite ? bf16_bits(__uint_as_float(top) * (1.0f / 6.0f)) : 0x7FC0u;
  return finite ? codes8(x, bf16_float(scale)) : 0u;
}

// ---- append ------------------------------------------------------------------

// Rows of at most one token: D / 8 lanes for each (row, head), 8 channels each.
// A value word is shared with seven other tokens of the slot, none of which the
// call writes: read, changed and written by one thread.  A chain of two loads
// (page id, word) and two stores; 512 rows x 8 heads are 4096 such chains: 4.6 us.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void append_one_kernel(CacheView cv, RowsView rv, const void *k,
                                                         int64_t ks, const void *v, int64_t vs,
                                                         uint32_t *status) {
  constexpr int L = D / 8;
  const int item = (blockIdx.x * 256 + threadIdx.x) / L, chunk = threadIdx.x % L;
  const int r = item / cv.Hkv, h = item % cv.Hkv;
  if (r >= rv.R) return;
  // the lanes of a wave may be of several rows: vector loads throughout
  const int t0 = rv.start ? rv.start[r] : r, t1 = rv.start ? rv.start[r + 1] : r + 1;
  const int slot = rv.slot ? rv.slot[r] : r, pos = rv.context[r];
  if (t0 >= t1 && t0 >= 0 && t1 <= rv.N) return;             // no token
  if (t0 < 0 || t1 > rv.N || t1 - t0 > 1 || slot < 0 || slot >= cv.n_slots || pos < 0 ||
      pos >= rv.max_context || pos / kPage >= cv.max_pages) {
    if (chunk == 0) set_bad(status);
    return;
  }
  const int id = cv.table[(int64_t)slot * cv.max_pages + pos / kPage];
  if (id < 0 || id >= cv.n_pages || (cv.refs && cv.refs[id] > 1)) {
    if (chunk == 0) set_bad(status);
    return;
  }
  uint8_t *page = cv.pages + ((int64_t)id * cv.Hkv + h) * cache_page_bytes(D);
  const int t = pos % kPage;
  float x[8], y[8];
  load8<BF16>(k, t0 * ks + h * D + chunk * 8, x);
  load8<BF16>(v, t0 * vs + h * D + chunk * 8, y);
  uint32_t *word[8], old[8];
  const int shift = 4 * value_nibble(t);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    word[i] = reinterpret_cast<uint32_t *>(
        page + value_word<D>(t >> 5, (t >> 2) & 3, chunk * 8 + i));
    old[i] = *word[i];
  }
  uint32_t byte, scale;
  const uint32_t kc = key_codes(x, byte), vc = value_codes<D>(y, scale);
  *reinterpret_cast<uint32_t *>(page + t * (D / 2) + chunk * 4) = kc;
  if (chunk % 4 == 0) page[key_scale_at<D>(t, chunk / 4)] = (uint8_t)byte;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    *word[i] = (old[i] & ~(0xFu << shift)) | ((vc >> (4 * i)) & 0xFu) << shift;
  if (chunk == 0) {
    *reinterpret_cast<uint16_t *>(page + value_scale_at<D>(t)) = (uint16_t)scale;
    if (cv.weight) cv.weight[((int64_t)slot * cv.Hkv + h) * cv.max_pages * kPage + pos] = 0.0f;
  }
}

// The stretches of TOK positions (a page, or half of one) that a row's tokens
// touch: at most tokens / TOK + 2, so the items of row r begin at
// start[r] / TOK + 2 r.
inline int64_t stretch_items(int32_t R, int32_t N, int tok) {
  return (int64_t)N / tok + 2 * (int64_t)R;
}

struct StretchItem {
  Span sp;
  int pos0;                  // its first position
  int lo, hi;                // positions of it that are the call's, lo < hi, else none
  uint8_t *page;             // of head 0
};

template <int D, int TOK, bool WRITE>
__device__ __forceinline__ StretchItem stretch_item(const CacheView &cv, const RowsView &rv,
                                                    uint32_t *status) {
  StretchItem it;
  const int64_t x = blockIdx.x;
  auto base = [&](int r) __attribute__((always_inline)) {
    return (int64_t)row_start(rv, r) / TOK + 2 * (int64_t)r;
  };
  const int r = find_row(rv.R, x, base);
  it.sp = row_span(cv, rv, r);
  const Span &s = it.sp;
  const int first = max(s.ctx, 0);
  const int64_t at = (int64_t)first / TOK + (x - base(r));
  const bool none = s.n == 0 || x < base(r) || at * TOK >= s.len;
  it.lo = it.hi = 0;
  it.pos0 = 0;
  it.page = nullptr;
  if ((s.bad || s.ctx < 0) && threadIdx.x == 0) set_bad(status);
  if (none) return it;
  it.pos0 = (int)at * TOK;
  it.lo = max(first - it.pos0, 0);
  it.hi = min(s.len - it.pos0, TOK);
  it.page = page_of<D, WRITE>(cv, s.slot, it.pos0 / kPage, 0);
  if (!it.page) {
    it.hi = it.lo;
    if (threadIdx.x == 0) set_bad(status);
  }
  return it;
}

// Workgroups that share out the heads of a stretch: all heads in one where there
// are enough for eight workgroups on each compute unit (the chain of loads
// to a page's address then counts once for all), fewer otherwise.  Append and read,
// 24 prompts of 100 to 400 tokens: 22.5 us, always one workgroup 47, always one for
// each head 23; 200 of 30 to 40: 33.5, 54 and 36; 2 of 100 to 400: 14, 36 and 14.
inline unsigned head_groups(int64_t items, int Hkv) {
  const int64_t want = (2048 + items - 1) / std::max<int64_t>(items, 1);
  return (unsigned)std::min<int64_t>(std::max<int64_t>(want, 1), Hkv);
}

// Any number of tokens: a workgroup for each half page and its share of the heads.
// Key codes go straight to the page (a lane's 8 channels are one word); value
// codes turn through LDS, so that each word of 8 tokens is written once, whole.
// 24 prompts of 100 to 400 tokens, 8 heads of 128 (31 MB): 15.5 us, two round trips
// of loads and a launch around 5 us of traffic (whole pages: 21 us).
template <int D, bool BF16>
__global__ __launch_bounds__(256) void append_kernel(CacheView cv, RowsView rv, const void *k,
                                                     int64_t ks, const void *v, int64_t vs,
                                                     uint32_t *status) {
  constexpr int L = D / 8, E = kHalf * L / 256;
  __shared__ uint32_t codes[2][kHalf][L + 1];
  const StretchItem it = stretch_item<D, kHalf, true>(cv, rv, status);
  if (it.lo >= it.hi) return;
  const int t0 = it.pos0 % kPage;                // the half's first token in the page
  int b = 0;
  for (int h = blockIdx.y; h < cv.Hkv; h += gridDim.y, b ^= 1) {
    uint8_t *page = it.page + (int64_t)h * cache_page_bytes(D);
    float x[E][8], y[E][8];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int at = threadIdx.x + 256 * i, t = at / L, chunk = at % L;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = y[i][e] = 0.0f;
      if (t >= it.lo && t < it.hi) {
        const int64_t tok = it.sp.t0 + (it.pos0 + t - it.sp.ctx);
        load8<BF16>(k, tok * ks + h * D + chunk * 8, x[i]);
        load8<BF16>(v, tok * vs + h * D + chunk * 8, y[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int at = threadIdx.x + 256 * i, t = at / L, chunk = at % L;
      const bool mine = t >= it.lo && t < it.hi;
      if (!__any(mine)) continue;
      uint32_t byte, scale;
      const uint32_t kc = key_codes(x[i], byte);
      codes[b][t][chunk] = value_codes<D>(y[i], scale);
      if (mine) {
        *reinterpret_cast<uint32_t *>(page + (t0 + t) * (D / 2) + chunk * 4) = kc;
        if (chunk % 4 == 0) page[key_scale_at<D>(t0 + t, chunk / 4)] = (uint8_t)byte;
        if (chunk == 0)
          *reinterpret_cast<uint16_t *>(page + value_scale_at<D>(t0 + t)) = (uint16_t)scale;
      }
    }
    if (cv.weight && (int)threadIdx.x >= it.lo && (int)threadIdx.x < it.hi)
      cv.weight[((int64_t)it.sp.slot * cv.Hkv + h) * cv.max_pages * kPage + it.pos0 +
                threadIdx.x] = 0.0f;
    __syncthreads();
    uint32_t *words = reinterpret_cast<uint32_t *>(page + 32 * D) + t0 / kHalf * 4 * D;
#pragma unroll
    for (int i = threadIdx.x; i < 4 * D; i += 256) {
      const int lane = (i >> 2) & 63, ct = (i >> 8) * 4 + (i & 3), m = lane & 15, g = lane >> 4;
      const int c = (m >> 2) * (D / 4) + 4 * ct + (m & 3);
      uint32_t w = 0, mask = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int t = (j >> 2) * 16 + 4 * g + (j & 3);
        const bool mine = t >= it.lo && t < it.hi;
        if (mine) {
          w |= ((codes[b][t][c >> 3] >> (4 * (c & 7))) & 0xFu) << (4 * j);
          mask |= 0xFu << (4 * j);
        }
      }
      if (mask == 0xFFFFFFFFu) words[i] = w;
      else if (mask) words[i] = (words[i] & ~mask) | w;
    }
  }
}

// ---- read --------------------------------------------------------------------

// Rows of at most one token, as append_one_kernel.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void read_one_kernel(CacheView cv, RowsView rv, void *k,
                                                       int64_t ks, void *v, int64_t vs,
                                                       uint32_t *status) {
  constexpr int L = D / 8;
  const int item = (blockIdx.x * 256 + threadIdx.x) / L, chunk = threadIdx.x % L;
  const int r = item / cv.Hkv, h = item % cv.Hkv;
  if (r >= rv.R) return;
  const int t0 = rv.start ? rv.start[r] : r, t1 = rv.start ? rv.start[r + 1] : r + 1;
  const int slot = rv.slot ? rv.slot[r] : r, pos = rv.context[r];
  if (t0 >= t1 && t0 >= 0 && t1 <= rv.N) return;
  if (t0 < 0 || t1 > rv.N || t1 - t0 > 1 || slot < 0 || slot >= cv.n_slots || pos < 0 ||
      pos >= rv.max_context || pos / kPage >= cv.max_pages) {
    if (chunk == 0) set_bad(status);
    return;
  }
  const int id = cv.table[(int64_t)slot * cv.max_pages + pos / kPage];
  if (id < 0 || id >= cv.n_pages) {
    if (chunk == 0) set_bad(status);
    return;
  }
  const uint8_t *page = cv.pages + ((int64_t)id * cv.Hkv + h) * cache_page_bytes(D);
  const int t = pos % kPage, shift = 4 * value_nibble(t);
  const uint32_t kc = *reinterpret_cast<const uint32_t *>(page + t * (D / 2) + chunk * 4);
  const uint32_t byte = page[key_scale_at<D>(t, chunk / 4)];
  const float vscale =
      bf16_float(*reinterpret_cast<const uint16_t *>(page + value_scale_at<D>(t)));
  uint32_t vc = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t w = *reinterpret_cast<const uint32_t *>(
        page + value_word<D>(t >> 5, (t >> 2) & 3, chunk * 8 + i));
    vc |= ((w >> shift) & 0xFu) << (4 * i);
  }
  store_keys<BF16>(k, t0 * ks + h * D + chunk * 8, kc, byte);
  store_values<BF16>(v, t0 * vs + h * D + chunk * 8, vc, vscale);
}

// A workgroup for each page and its share of the heads; the value words go
// through LDS, the next head's on their way while this one's are written.
// Writes 4 (bf16) or 8 times the bytes that it reads.  HBM bounds it: 32 rows of
// 2048 positions (8 heads of 128, bf16, 340 MB) 57 us, 5.9 TB/s.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void read_kernel(CacheView cv, RowsView rv, void *k, int64_t ks,
                                                   void *v, int64_t vs, uint32_t *status) {
  constexpr int L = D / 8, E = kPage * L / 256, V = (2 * D + 255) / 256;
  __shared__ u32x4 words[2][2 * D];
  const StretchItem it = stretch_item<D, kPage, false>(cv, rv, status);
  if (it.lo >= it.hi) return;
  u32x4 vw[V];
  uint32_t kc[E];
  uint8_t kb[E];
  uint16_t vb[E];
  auto fetch = [&](int h) __attribute__((always_inline)) {
    const uint8_t *page = it.page + (int64_t)h * cache_page_bytes(D);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int at = threadIdx.x + 256 * i;
      if (at < 2 * D) vw[i] = reinterpret_cast<const u32x4 *>(page + 32 * D)[at];
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int at = threadIdx.x + 256 * i, t = at / L, chunk = at % L;
      kc[i] = *reinterpret_cast<const uint32_t *>(page + t * (D / 2) + chunk * 4);
      kb[i] = page[key_scale_at<D>(t, chunk / 4)];
      vb[i] = *reinterpret_cast<const uint16_t *>(page + value_scale_at<D>(t));
    }
  };
  int b = 0;
  fetch(blockIdx.y);
  for (int h = blockIdx.y; h < cv.Hkv; h += gridDim.y, b ^= 1) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int at = threadIdx.x + 256 * i;
      if (at < 2 * D) words[b][at] = vw[i];
    }
    uint32_t kc0[E], kb0[E];
    float vb0[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      kc0[i] = kc[i];
      kb0[i] = kb[i];
      vb0[i] = bf16_float(vb[i]);
    }
    if (h + (int)gridDim.y < cv.Hkv) fetch(h + gridDim.y);
    __syncthreads();
    const uint32_t *w32 = reinterpret_cast<const uint32_t *>(words[b]);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int at = threadIdx.x + 256 * i, t = at / L, chunk = at % L;
      if (t < it.lo || t >= it.hi) continue;
      const int64_t tok = it.sp.t0 + (it.pos0 + t - it.sp.ctx);
      const int shift = 4 * value_nibble(t);
      uint32_t vc = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t w = w32[(value_word<D>(t >> 5, (t >> 2) & 3, chunk * 8 + e) - 32 * D) / 4];
        vc |= ((w >> shift) & 0xFu) << (4 * e);
      }
      store_keys<BF16>(k, tok * ks + h * D + chunk * 8, kc0[i], kb0[i]);
      store_values<BF16>(v, tok * vs + h * D + chunk * 8, vc, vb0[i]);
    }
  }
}

// ---- eviction ----------------------------------------------------------------

constexpr int kSelect = 1024, kSelectWaves = kSelect / 64;

// Ascending with the weight; NaN lowest, -0 as 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One workgroup for each row and head.  The m-th largest key of the old
// positions is found digit by digit (11, 11 and 10 bits, from the top): a
// histogram of the digit among the keys that match so far, then the digit at
// which the count from above reaches what is left of m.  Equal keys of a wave
// are counted once by a vote before the LDS atomics: most positions of a cache
// have received exactly nothing.  Then keys above the m-th, and the first of its
// equals, are written in order.  Blocks of 16 keys a thread, loaded together: of
// up to 16384 positions they stay in registers for all four passes.  A chain of
// histograms, scans and barriers of one workgroup: 16 us for 256 (row, head) of up
// to 5000 positions, 20 for 8 of 16384.
__global__ __launch_bounds__(kSelect) void evict_select_kernel(CacheView cv, EvictView ev) {
  constexpr int KEYS = 16, BLOCK = KEYS * kSelect;
  __shared__ uint32_t hist[2048];
  __shared__ uint32_t counts[KEYS * kSelectWaves], wave_sum[kSelectWaves];
  __shared__ uint32_t sh_digit, sh_left;
  const int h = blockIdx.x, r = blockIdx.y, tid = threadIdx.x;
  const int lane = tid & 63, wave = tid >> 6;
  const int slot = ev.slot ? ld_const(ev.slot, r) : r;
  int n = ld_const(ev.length, r);
  const int cap = min((int64_t)ev.max_length, (int64_t)cv.max_pages * kPage);
  const bool bad = slot < 0 || slot >= cv.n_slots || n < 0 || n > cap;
  if (bad) {
    n = slot < 0 || slot >= cv.n_slots ? 0 : min(max(n, 0), cap);
    if (tid == 0) set_bad(ev.status);
  }
  const int len = min(n, ev.keep);
  if (h == 0 && tid == 0) ev.length_out[r] = len;
  int32_t *kept = ev.kept + ((int64_t)r * cv.Hkv + h) * ev.keep;
  for (int i = len + tid; i < ev.keep; i += kSelect) kept[i] = -1;
  if (n <= ev.keep) {
    for (int i = tid; i < n; i += kSelect) kept[i] = i;
    return;
  }
  const int old = n - ev.recent, m = ev.keep - ev.recent;
  for (int i = tid; i < ev.recent; i += kSelect) kept[m + i] = old + i;
  if (m == 0) return;
  const float *w = cv.weight + ((int64_t)slot * cv.Hkv + h) * cv.max_pages * kPage;
  // key j of a block: position block + j kSelect + tid
  uint32_t key[KEYS];
  auto load = [&](int block) __attribute__((always_inline)) {
    float x[KEYS];
#pragma unroll
    for (int j = 0; j < KEYS; ++j) x[j] = w[min(block + j * kSelect + tid, old - 1)];
#pragma unroll
    for (int j = 0; j < KEYS; ++j) key[j] = weight_key(x[j]);
  };
  load(0);
  uint32_t prefix = 0, left = (uint32_t)m;
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const int bits = pass == 2 ? 10 : 11;
    for (int i = tid; i < 2048; i += kSelect) hist[i] = 0;
    __syncthreads();
    for (int block = 0; block < old; block += BLOCK) {
      if (old > BLOCK) load(block);
#pragma unroll
      for (int j = 0; j < KEYS; ++j) {
        const bool in = block + j * kSelect + tid < old &&
                        (pass == 0 || key[j] >> (shift + bits) == prefix);
        const uint32_t digit = (key[j] >> shift) & ((1u << bits) - 1u);
        const uint64_t live = __ballot(in);
        if (live == 0) continue;
        const int lead = __ffsll((unsigned long long)live) - 1;
        const uint32_t dl = (uint32_t)__shfl((int)digit, lead);
        const uint64_t same = __ballot(in && digit == dl);
        if (lane == lead) atomicAdd(&hist[dl], (uint32_t)__popcll(same));
        if (in && digit != dl) atomicAdd(&hist[digit], 1u);
      }
    }
    __syncthreads();
    // counts from the top: thread t holds digits 2047 - 2t and 2046 - 2t
    const uint32_t a = hist[2047 - 2 * tid], b = hist[2046 - 2 * tid];
    uint32_t sum = a + b;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t o = (uint32_t)__shfl_up((int)sum, d);
      if (lane >= d) sum += o;
    }
    if (lane == 63) wave_sum[wave] = sum;
    __syncthreads();
    for (int i = 0; i < wave; ++i) sum += wave_sum[i];
    const uint32_t before = sum - a - b;       // keys of higher digits
    if (before < left && sum >= left) {
      const bool first = before + a >= left;
      sh_digit = (uint32_t)(first ? 2047 - 2 * tid : 2046 - 2 * tid);
      sh_left = left - before - (first ? 0u : a);
    }
    __syncthreads();
    prefix = prefix << bits | sh_digit;
    left = sh_left;
  }
  // `left` of the keys equal to prefix stay.  counts: of each key index and wave
  // of a block, in position order, keys above (low half) and equal (high half)
  uint32_t gt = 0, eq = 0;                     // before the block
  const uint64_t below = (1ull << lane) - 1;
  for (int block = 0; block < old; block += BLOCK) {
    if (old > BLOCK) load(block);
#pragma unroll
    for (int j = 0; j < KEYS; ++j) {
      const bool in = block + j * kSelect + tid < old;
      const uint64_t bg = __ballot(in && key[j] > prefix), be = __ballot(in && key[j] == prefix);
      if (lane == 0) counts[j * kSelectWaves + wave] = __popcll(bg) | __popcll(be) << 16;
    }
    __syncthreads();
    uint32_t mine = 0, sum = 0;
    if (tid < KEYS * kSelectWaves) {
      mine = sum = counts[tid];
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = (uint32_t)__shfl_up((int)sum, d);
        if (lane >= d) sum += o;
      }
      if (lane == 63) wave_sum[wave] = sum;
    }
    __syncthreads();
    uint32_t all = 0;
#pragma unroll
    for (int i = 0; i < KEYS * kSelectWaves / 64; ++i) {
      if (i < wave) sum += wave_sum[i];
      all += wave_sum[i];
    }
    if (tid < KEYS * kSelectWaves) counts[tid] = sum - mine;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < KEYS; ++j) {
      const int i = block + j * kSelect + tid;
      const bool above = i < old && key[j] > prefix, equal = i < old && key[j] == prefix;
      const uint64_t bg = __ballot(above), be = __ballot(equal);
      const uint32_t c = counts[j * kSelectWaves + wave];
      const uint32_t my_gt = gt + (c & 0xFFFFu) + __popcll(bg & below);
      const uint32_t my_eq = eq + (c >> 16) + __popcll(be & below);
      if (above || (equal && my_eq < left)) kept[my_gt + min(my_eq, left)] = i;
    }
    gt += all & 0xFFFFu;
    eq += all >> 16;
    __syncthreads();                           // counts and wave_sum are read
  }
}

// A workgroup for each row, head and page of the new slot.  A lane makes four
// value words (16 bytes) from the 16-byte chunks of their 8 tokens.  32 rows of up
// to 5000 positions to 2048 (8 heads of 128): 51 us.  The kept positions are 142 MB
// to read and write; a kept token's codes are pieces of lines that hold its
// neighbours, so nearly all of the source's pages are read.
template <int D>
__global__ __launch_bounds__(256) void evict_move_kernel(CacheView from, CacheView to,
                                                         EvictView ev) {
  __shared__ const uint8_t *page[kPage];
  __shared__ int token[kPage];
  __shared__ uint32_t valid[kPage];
  const int h = blockIdx.x % from.Hkv, r = blockIdx.y, tid = threadIdx.x;
  const int at = blockIdx.x / from.Hkv, pos0 = at * kPage;
  const int slot = ev.slot ? ld_const(ev.slot, r) : r;
  const int len = ld_const(ev.length_out, r);
  if (pos0 >= len) return;
  const int count = min(len - pos0, kPage);
  uint8_t *dst = nullptr;
  if (r < to.n_slots && at < to.max_pages) dst = page_of<D, true>(to, r, at, h);
  if (!dst) {
    if (tid == 0) set_bad(ev.status);
    return;
  }
  if (tid < kPage) {
    const uint8_t *p = nullptr;
    int src = 0;
    if (tid < count) {
      src = ev.kept[((int64_t)r * from.Hkv + h) * ev.keep + pos0 + tid];
      const int id = from.table[(int64_t)slot * from.max_pages + src / kPage];
      if (id >= 0 && id < from.n_pages)
        p = from.pages + ((int64_t)id * from.Hkv + h) * cache_page_bytes(D);
      else
        set_bad(ev.status);
      if (to.weight) {
        const int64_t f = ((int64_t)slot * from.Hkv + h) * from.max_pages * kPage + src;
        to.weight[((int64_t)r * to.Hkv + h) * to.max_pages * kPage + pos0 + tid] =
            from.weight ? from.weight[f] : 0.0f;
      }
    }
    // (a position without a page is read from the destination and left out)
    page[tid] = p ? p : dst;
    token[tid] = src % kPage;
    valid[tid] = p ? 0xFu : 0u;
  }
  __syncthreads();
  // the loads of a thread's pieces go out together.  Keys: 16-byte chunks of 32
  // channels and their scale byte; values: chunk i is words [half][q][lane][0..3]
#pragma unroll
  for (int i = tid; i < 2 * D; i += 256) {
    const int kt = i / (D / 32), kb = i % (D / 32), ks = token[kt];
    const uint8_t *kp = page[kt];
    const u32x4 kx = *reinterpret_cast<const u32x4 *>(kp + ks * (D / 2) + kb * 16);
    const uint8_t kscale = kp[key_scale_at<D>(ks, kb)];
    const int lane = i & 63, g = lane >> 4, m = lane & 15, hq = i >> 6;
    const int half = hq / (D / 64), q = hq % (D / 64);
    u32x4 x[8];
    int shift[8];
    uint32_t mask[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int t = half * kHalf + (j >> 2) * 16 + 4 * g + (j & 3), s = token[t];
      const int from_at = (((s >> 5) * (D / 64) + q) * 64 + ((s >> 2) & 3) * 16 + m) * 16;
      x[j] = *reinterpret_cast<const u32x4 *>(page[t] + 32 * D + from_at);
      shift[j] = 4 * value_nibble(s);
      mask[j] = valid[t];
    }
    if (valid[kt]) {
      *reinterpret_cast<u32x4 *>(dst + kt * (D / 2) + kb * 16) = kx;
      dst[key_scale_at<D>(kt, kb)] = kscale;
    }
    u32x4 w = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] |= ((x[j][e] >> shift[j]) & mask[j]) << (4 * j);
    *reinterpret_cast<u32x4 *>(dst + 32 * D + i * 16) = w;
  }
  if (tid < kPage && valid[tid])
    *reinterpret_cast<uint16_t *>(dst + value_scale_at<D>(tid)) =
        *reinterpret_cast<const uint16_t *>(page[tid] + value_scale_at<D>(token[tid]));
}

template <int D, bool BF16>
void append_launch(const CacheView &cv, const RowsView &rv, const void *k, int64_t ks,
                   const void *v, int64_t vs, uint32_t *status, hipStream_t st) {
  if (rv.max_tokens <= 1) {
    const int64_t lanes = (int64_t)rv.R * cv.Hkv * (D / 8);
    hipLaunchKernelGGL((append_one_kernel<D, BF16>), dim3((unsigned)((lanes + 255) / 256)),
                       dim3(256), 0, st, cv, rv, k, ks, v, vs, status);
  } else {
    const int64_t items = stretch_items(rv.R, rv.N, kHalf);
    const dim3 grid((unsigned)items, head_groups(items, cv.Hkv));
    hipLaunchKernelGGL((append_kernel<D, BF16>), grid, dim3(256), 0, st, cv, rv, k, ks, v, vs,
                       status);
  }
}

template <int D, bool BF16>
void read_launch(const CacheView &cv, const RowsView &rv, void *k, int64_t ks, void *v, int64_t vs,
                 uint32_t *status, hipStream_t st) {
  if (rv.max_tokens <= 1) {
    const int64_t lanes = (int64_t)rv.R * cv.Hkv * (D / 8);
    hipLaunchKernelGGL((read_one_kernel<D, BF16>), dim3((unsigned)((lanes + 255) / 256)),
                       dim3(256), 0, st, cv, rv, k, ks, v, vs, status);
  } else {
    const int64_t items = stretch_items(rv.R, rv.N, kPage);
    const dim3 grid((unsigned)items, head_groups(items, cv.Hkv));
    hipLaunchKernelGGL((read_kernel<D, BF16>), grid, dim3(256), 0, st, cv, rv, k, ks, v, vs,
                       status);
  }
}

}  // namespace

hipError_t launch_cache_append(const CacheView &cv, const RowsView &rv, int D, bool bf16,
                               const void *k, int64_t ks, const void *v, int64_t vs,
                               uint32_t *status, hipStream_t st) {
  auto go = [&](auto d) {
    constexpr int W = decltype(d)::value;
    if (bf16) append_launch<W, true>(cv, rv, k, ks, v, vs, status, st);
    else append_launch<W, false>(cv, rv, k, ks, v, vs, status, st);
  };
  if (D == 64) go(std::integral_constant<int, 64>{});
  else if (D == 128) go(std::integral_constant<int, 128>{});
  else go(std::integral_constant<int, 256>{});
  return hipGetLastError();
}

hipError_t launch_cache_read(const CacheView &cv, const RowsView &rv, int D, bool bf16, void *k,
                             int64_t ks, void *v, int64_t vs, uint32_t *status, hipStream_t st) {
  auto go = [&](auto d) {
    constexpr int W = decltype(d)::value;
    if (bf16) read_launch<W, true>(cv, rv, k, ks, v, vs, status, st);
    else read_launch<W, false>(cv, rv, k, ks, v, vs, status, st);
  };
  if (D == 64) go(std::integral_constant<int, 64>{});
  else if (D == 128) go(std::integral_constant<int, 128>{});
  else go(std::integral_constant<int, 256>{});
  return hipGetLastError();
}

hipError_t launch_cache_evict(const CacheView &from, const CacheView &to, const EvictView &ev,
                              int D, hipStream_t st) {
  hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)from.Hkv, (unsigned)ev.R), dim3(kSelect),
                     0, st, from, ev);
  const int longest = min(ev.keep, ev.max_length);
  if (longest > 0) {
    const dim3 grid((unsigned)((longest + kPage - 1) / kPage * from.Hkv), (unsigned)ev.R);
    if (D == 64) hipLaunchKernelGGL(evict_move_kernel<64>, grid, dim3(256), 0, st, from, to, ev);
    else if (D == 128)
      hipLaunchKernelGGL(evict_move_kernel<128>, grid, dim3(256), 0, st, from, to, ev);
    else hipLaunchKernelGGL(evict_move_kernel<256>, grid, dim3(256), 0, st, from, to, ev);
  }
  return hipGetLastError();
}

}  // namespace mcd
