// Arguments of the log-probability kernels (bs_token_logprobs), and the ranking of alternatives.
#pragma once
#include "common.h"

struct LogprobArgs {
  const void* logits;             // [rows][vocab]
  const int32_t *draft_len, *tokens, *n_tokens;
  int k_max, vocab, n_top;
  float inv_temp;
  float *logprob, *entropy, *top_logprobs;
  int32_t *top_tokens, *status;
};
constexpr int kLogprobMaxTop = 32;

// Ranking of alternatives: a larger logit first, equal ones by the lower index (-0 counts as +0); 0: no alternative (masked, NaN).
__device__ __forceinline__ unsigned long long logprob_key(float z, int j) {
  if (!(z > -INFINITY)) return 0;
  return (unsigned long long)filter_key(z) << 32 | (0xffffffffu - (uint32_t)j);
}

size_t logprob_workspace(int B, int k_max, int vocab, int n_top);
void launch_logprob(const LogprobArgs& a, int B, int dtype, void* workspace, hipStream_t st);
