// Launchers of the operators at the ends of a block and of a tuning step (owq_dropout.hip, owq_norm.hip, owq_logprob.hip),
// called by the checked entry points in owq_ends.cpp.  All return a hipError_t as int.
#pragma once
#include <cstddef>
#include <cstdint>

#include "owq.h"

namespace owq {

// What dropout does with 16 random bits: an element stays where they are not below `threshold`, times `scale`.
struct Dropping {
  const uint64_t *rng;
  uint32_t threshold;      // 0 = none
  float scale;
  int32_t site;
};

struct DropoutArgs {
  const void *x, *residual;
  void *out;
  int64_t x_row, residual_row;
  int32_t n_rows, width;
  Dropping drop;
};
int launch_dropout(const DropoutArgs &a, int32_t type, void *stream);

struct NormArgs {
  const void *h, *branch, *gate, *post_w, *post_b, *w, *b;
  void *total_out, *y;                              // forward
  const void *dy, *dtotal, *total;                  // backward
  void *dh, *dbranch, *dgate;                       // dgate: of a token gate
  float *partial;                                   // backward: a row of n_sums sums of `pitch` columns per workgroup
  int64_t h_row, branch_row, gate_row, total_row, dy_row, dtotal_row;
  int32_t n_tokens, width, post, norm;
  int32_t n_sums, pitch;
  int32_t branch_side;                              // backward: something of the branch's is wanted
  int32_t sum_w, sum_b, sum_post_w, sum_post_b, sum_gate;   // which sum is whose, -1 = not wanted
  float eps, h_scale, branch_scale;
  Dropping drop;
};
// Workgroups of the backward and sums of each, from the description alone.
struct NormPlan {
  int32_t blocks, pitch;
};
NormPlan norm_backward_plan(const owq_norm_desc_t &d);
int launch_norm(const NormArgs &a, int32_t type, int32_t h_type, void *stream);
// Rows that registers do not hold (owq_norm_wide.hip).
int launch_norm_wide(const NormArgs &a, int32_t type, int32_t h_type, void *stream);
void launch_norm_backward_wide(const NormArgs &a, int32_t type, int32_t h_type, int32_t blocks, void *stream);
// sums: where the sum of each kind goes, in the order of their numbers in a
int launch_norm_backward(const NormArgs &a, int32_t type, int32_t h_type, const NormPlan &p, float *const *sums, void *stream);

struct LogprobArgs {
  const void *logits;
  const int32_t *targets;
  float *logprob, *top_logprob, *stats;
  int32_t *top_token;
  int64_t logits_row;
  int32_t n_rows, vocab, top;
  float scale;
};
int launch_logprobs(const LogprobArgs &a, int32_t type, void *stream);

struct LogprobBackwardArgs {
  const void *logits;
  const int32_t *targets;
  const float *stats, *dlogprob, *dentropy;
  void *dlogits;
  int64_t logits_row;
  int32_t n_rows, vocab;
  float scale;
};
int launch_logprobs_backward(const LogprobBackwardArgs &a, int32_t type, void *stream);

}  // namespace owq
