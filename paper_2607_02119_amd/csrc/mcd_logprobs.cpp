// Host side of the log probabilities: argument checks and launches.  Nothing here
// allocates device memory, synchronises or throws.
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>

#include "logprobs.h"

namespace {

mcd_status bad(const char *fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return mcd::record_error(MCD_E_INVALID, buf);
}

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
size_t round_up(size_t x) { return (x + 255) / 256 * 256; }

mcd_status check_sizes(int32_t n, int32_t K, int32_t V, int32_t T) {
  if (n < 0 || K < 1 || K > MCD_MAX_K || V < 1 || T < 0)
    return bad("bad sizes (n=%d K=%d V=%d T=%d)", n, K, V, T);
  if (V > mcd::kMostLogits || T > MCD_MAX_TOP) {
    char buf[128];
    snprintf(buf, sizeof buf, "at most %d logits and %d alternatives (V=%d T=%d)",
             mcd::kMostLogits, MCD_MAX_TOP, V, T);
    return mcd::record_error(MCD_E_UNSUPPORTED, buf);
  }
  // (items of a launch: a part of a vector each)
  if ((int64_t)n * K * ((V + 4095) / 4096) >= (int64_t)1 << 31) return bad("too many vectors");
  if (mcd::logprob_groups((int64_t)n * K, V) > mcd::kMostGroups)
    return mcd::record_error(MCD_E_UNSUPPORTED, "more vectors than a launch takes");
  return MCD_OK;
}

size_t sum_bytes(int64_t vectors, int32_t parts) {
  return parts > 1 ? round_up((size_t)vectors * parts * sizeof(float4)) : 0;
}
size_t top_bytes(int64_t vectors, int32_t parts, int32_t T) {
  return parts > 1 ? round_up((size_t)vectors * parts * T * sizeof(uint2)) : 0;
}

struct Bytes {
  const void *p;
  int64_t n;
};
bool overlap(const Bytes &a, const Bytes &b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return x && y && a.n > 0 && b.n > 0 && x < y + b.n && y < x + a.n;
}

}  // namespace

extern "C" {

size_t mcd_logprobs_workspace_bytes(int32_t n, int32_t K, int32_t V, int32_t T) {
  if (check_sizes(n, K, V, T) != MCD_OK) return 0;
  // parts of 4096 logits: fewer rows may be cut up finer, never finer than that
  const int64_t vectors = (int64_t)n * K;
  const int32_t parts = (V + 4095) / 4096;
  return mcd::kStatusBytes + sum_bytes(vectors, parts) + top_bytes(vectors, parts, T);
}

mcd_status mcd_logprobs(const mcd_logprobs_args *a, hipStream_t stream) {
  if (!a) return bad("null args");
  if (mcd_status s = check_sizes(a->n, a->K, a->V, a->T)) return s;
  if (a->dtype != MCD_F32 && a->dtype != MCD_BF16) return bad("bad dtype");
  mcd::LogprobView lv = {};
  int64_t width = 0;
  for (int k = 0; k < a->K; ++k) {
    const int32_t V = a->V_stream ? a->V_stream[k] : a->V;
    if (V < 1 || V > a->V) return bad("stream %d has %d ids, V=%d", k, V, a->V);
    lv.off.o[k] = (int32_t)width;
    width += V;
  }
  lv.off.o[a->K] = (int32_t)width;                 // (at most 32 * 2^19)
  if (a->pad_id >= 0 && a->pad_id < a->V) return bad("pad_id %d is an id of a stream", a->pad_id);
  if (a->n == 0) return MCD_OK;
  if (!a->logits || !a->tokens || !a->logprob) return bad("null array");
  const int64_t eb = a->dtype == MCD_BF16 ? 2 : 4, n = a->n, vectors = n * a->K;
  if (a->logits_stride < width || a->logits_stride > ((int64_t)1 << 30))
    return bad("logits: bad row stride");                // (n - 1 of them: below 2^61)
  if (a->token_rows < 1 || (!a->token_row && a->token_rows < a->n))
    return bad("tokens of %d rows", a->token_rows);
  if (a->T == 0 ? a->top_ids || a->top_logprobs : !a->top_ids && !a->top_logprobs)
    return bad("T=%d with%s arrays for alternatives", a->T, a->T ? "out" : "");
  if (!aligned(a->logits, (size_t)eb)) return bad("logits not aligned to their type");
  for (const void *p : {(const void *)a->tokens, (const void *)a->token_row,
                        (const void *)a->logprob, (const void *)a->entropy,
                        (const void *)a->top_ids, (const void *)a->top_logprobs})
    if (!aligned(p, 4)) return bad("array not aligned");
  const Bytes out[] = {{a->logprob, vectors * 4},
                       {a->entropy, vectors * 4},
                       {a->top_ids, vectors * a->T * 4},
                       {a->top_logprobs, vectors * a->T * 4}};
  const int64_t span = (n - 1) * a->logits_stride + width;
  if (span > ((int64_t)1 << 58)) return bad("logits: bad row stride");
  const Bytes in[] = {{a->logits, span * eb},
                      {a->tokens, (int64_t)a->token_rows * a->K * 4},
                      {a->token_row, n * 4}};
  for (int i = 0; i < 4; ++i) {
    for (const Bytes &x : in)
      if (overlap(out[i], x)) return bad("the arrays written must not overlap those read");
    for (int k = 0; k < i; ++k)
      if (overlap(out[i], out[k])) return bad("the arrays written must not overlap each other");
  }
  const size_t need = mcd_logprobs_workspace_bytes(a->n, a->K, a->V, a->T);
  if (!a->workspace || !aligned(a->workspace, 256))
    return bad("workspace must be 256-byte aligned");
  if (a->workspace_bytes < need) {
    char buf[128];
    snprintf(buf, sizeof buf, "workspace of %zu bytes, %zu needed", a->workspace_bytes, need);
    return mcd::record_error(MCD_E_WORKSPACE, buf);
  }
  const mcd::LogprobPlan p = mcd::logprob_plan(vectors, a->V);
  char *w = static_cast<char *>(a->workspace);
  lv.K = a->K;
  lv.T = a->T;
  lv.pad_id = a->pad_id;
  lv.parts = p.parts;
  lv.token_rows = a->token_rows;
  lv.vectors = vectors;
  lv.stride = a->logits_stride;
  lv.logits = a->logits;
  lv.tokens = a->tokens;
  lv.token_row = a->token_row;
  lv.logprob = a->logprob;
  lv.entropy = a->entropy;
  lv.top_ids = a->top_ids;
  lv.top_logprobs = a->top_logprobs;
  lv.status = reinterpret_cast<uint32_t *>(w);
  w += mcd::kStatusBytes;
  lv.part_sums = reinterpret_cast<float4 *>(w);
  w += sum_bytes(vectors, p.parts);
  lv.part_top = reinterpret_cast<uint2 *>(w);
  const hipError_t e = mcd::launch_logprobs(lv, p, a->dtype == MCD_BF16, stream);
  if (e == hipSuccess) return MCD_OK;
  char buf[256];
  snprintf(buf, sizeof buf, "log probabilities launch: %s", hipGetErrorString(e));
  return mcd::record_error(MCD_E_HIP, buf);
}

}  // extern "C"
