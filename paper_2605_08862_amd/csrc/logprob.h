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
constexpr int kLogprobMaxTop = 32, kLogprobMaxVocab = 1 << 20, kLogprobMaxRows = 1 << 16;

size_t logprob_workspace(int B, int k_max, int vocab, int n_top);
void launch_logprob(const LogprobArgs& a, int B, int dtype, void* workspace, hipStream_t st);
