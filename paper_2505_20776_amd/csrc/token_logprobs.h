// Arguments of the logits kernels (token_logprobs.hip) and the cut of a row into slices.
#pragma once

#include "common.h"

namespace specext {

struct LogprobArgs {
  const void* logits;
  const int32_t* tokens;      // [n_rows][n_given]
  float* logprob;             // [n_rows][n_given]
  int32_t* top_id;            // [n_rows][k]
  float* top_logprob;         // [n_rows][k]; may be null, as lse and entropy
  float* lse;
  float* entropy;
  float* stats;               // workspace: [n_rows][slices][4]
  unsigned long long* keys;   // workspace: [n_rows][slices][k]
  int64_t row_stride;         // in values
  int32_t bf16, n_rows, vocab, n_given, k, slices;
  float logit_scale;
};

constexpr int kLogprobThreads = 512;
constexpr int kMaxVocab = 1 << 20;
constexpr int kMaxTop = 64;

// Values per thread (8, 16, 32 or 64) and slices of a row of `vocab` values.  A row's first address may lie up to seven values
// behind a multiple of 16 bytes, which the slices have to cover too.
struct LogprobCut {
  int per_thread, slices;
};
inline LogprobCut logprob_cut(int vocab) {
  const int values = vocab + 7;
  int per_thread = 8;
  while (per_thread < 64 && per_thread * kLogprobThreads < values) per_thread *= 2;
  return {per_thread, (values + per_thread * kLogprobThreads - 1) / (per_thread * kLogprobThreads)};
}

hipError_t launch_token_logprobs(const LogprobArgs& a, int per_thread, hipStream_t stream);

}  // namespace specext
