// Log probabilities (mcd.h, mcd_logprobs): what the host and the kernels share.
#pragma once

#include "mcd_internal.h"

namespace mcd {

constexpr int kMostTop = MCD_MAX_TOP;
constexpr int32_t kMostLogits = 64 * 8192;           // 64 parts: one lane for each

struct LogprobView {
  int32_t K, T, pad_id, parts, token_rows;
  int64_t vectors, stride;     // n K; elements between rows
  const void *logits;
  const int32_t *tokens, *token_row;
  float *logprob, *entropy, *top_logprobs;
  int32_t *top_ids;
  // workspace: [vectors][parts] {max, S, U}, and [T] {order, id}
  float4 *part_sums;
  uint2 *part_top;
  uint32_t *status;
  StreamOffsets off;
};

// Logits of a part, and parts of a vector (1: no second launch).
struct LogprobPlan {
  int32_t part, parts;
};
LogprobPlan logprob_plan(int64_t vectors, int32_t V);
// Workgroups of the largest launch.
int64_t logprob_groups(int64_t vectors, int32_t V);
hipError_t launch_logprobs(const LogprobView &lv, const LogprobPlan &p, bool bf16, hipStream_t st);

}  // namespace mcd
