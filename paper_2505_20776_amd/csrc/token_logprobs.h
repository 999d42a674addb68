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
constexpr int kMaxSlices = 64;
// Slices are made smaller while there would be fewer than 128 workgroups.  us with 128 / 512, bf16 rows of 128256: 20 rows 9.1 / 9.8, 60 10.3 /
// 10.8; 60 fp32 rows of 32000 8.9 / 10.8; equal from 128 rows on and for one row.
constexpr int kLogprobWorkgroups = 128;

// 16-byte vectors per thread (1, 2, 4 or 8) and slices of a row of `vocab` values.  A row's first address may lie up to seven values
// behind a multiple of 16 bytes, which the slices have to cover too.
struct LogprobCut {
  int vectors, slices;
};
inline LogprobCut logprob_cut(int n_rows, int vocab, bool bf16) {
  const int per_vector = bf16 ? 8 : 4;
  const int values = vocab + per_vector - 1;
  auto slices_of = [&](int vectors) { return (values + vectors * per_vector * kLogprobThreads - 1) / (vectors * per_vector * kLogprobThreads); };
  int vectors = 8;
  while (vectors > 1 && static_cast<int64_t>(n_rows) * slices_of(vectors) < kLogprobWorkgroups) vectors /= 2;
  while (vectors < 8 && slices_of(vectors) > kMaxSlices) vectors *= 2;
  return {vectors, slices_of(vectors)};
}

hipError_t launch_token_logprobs(const LogprobArgs& a, int vectors, hipStream_t stream);

}  // namespace specext
