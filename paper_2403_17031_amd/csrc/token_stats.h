// Launchers of token_stats.hip.  With a null workspace they only return the bytes that they need.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rlhf {

enum { kTokensF32 = 0, kTokensBF16 = 1, kTokensF16 = 2 };
constexpr int kMaxTop = 64;           // alternatives of a row
constexpr int kMaxTokenVocab = 1 << 18;  // the part maxima of a row and the candidates of 64 alternatives fit 64 KB of LDS

struct TokenRows {  // a matrix whose rows are ld elements apart
  const void* p;
  int64_t ld;
  bool lies_well;  // token_rows_lie_well: read as it is, not through a packed copy in the workspace
};
// rows_as_k: the number of rows where a product sums over them (the backward pass), else 0.  (p 16-byte aligned)
bool token_rows_lie_well(int64_t ld, int d, int dtype, int rows_as_k);

struct TokenStatsArgs {
  TokenRows hidden, weight;
  const int32_t* targets;
  int T, d, V, dtype, top;
  float inv_t, inv_lo;  // 1 / temperature in two floats
  float *logprob, *entropy, *lse;
  int32_t* top_ids;
  float* top_logprob;
};
size_t token_stats_plan(const TokenStatsArgs& a, void* workspace, hipStream_t s, hipError_t* err);

struct TokenGradArgs {
  TokenRows hidden, weight;
  const int32_t* targets;
  const float *lse, *entropy, *d_logprob, *d_entropy;
  int T, d, V, dtype;
  float inv_t, inv_lo;  // 1 / temperature in two floats
  bool grad_f32;
  void *d_hidden, *d_weight;
};
size_t token_stats_backward_plan(const TokenGradArgs& a, void* workspace, hipStream_t s, hipError_t* err);

}  // namespace rlhf
