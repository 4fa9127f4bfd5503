// Launch interface of the training losses over logit rows (internal).
#pragma once

#include "device_util.h"

namespace pr {

// The logit rows of a loss and the gradient rows it writes.
struct LossRows {
  const void* logits;
  int64_t n_rows;
  int32_t V;
  int64_t row_stride;
  const int32_t* ids;
  const float* temperature;
  const float* weight;
  void* grad;  // NULL: not wanted
  int64_t grad_stride;
};

struct PolicyArgs {
  LossRows rows;
  const float* advantage;
  const float* old_logprob;
  const float* ref_logprob;  // NULL: no KL term
  double clip_lo, clip_hi;   // bounds of the clipped ratio
  double kl_coef;
  double grad_scale;
  float* loss;
  pr_policy_tokens_t out;
  int32_t G;         // workgroups per row of the parts (0: rows are not split)
  double* row_loss;  // the workspace, which starts with the rows' terms of the loss where they are not split
};

struct PreferenceArgs {
  LossRows rows;
  const int32_t* offsets;
  int32_t n_pairs;
  const float* ref_logprob;  // NULL: none
  double beta, label_smoothing, margin, grad_scale;
  float* loss;
  pr_preference_out_t out;
  int32_t G;  // workgroups per row of the statistics
  void* ws;
};

// Workgroups per row for a shape (0: rows are not split), with or without the
// gradient, and the workspace that either takes.
int policy_split(int64_t n_rows, int32_t V, pr_dtype dtype, bool grad);
size_t policy_workspace_bytes(int64_t n_rows, int32_t V, pr_dtype dtype);
hipError_t launch_policy(const PolicyArgs& a, pr_dtype dtype, hipStream_t stream);

// Workgroups per row for a shape, and the workspace it takes.
int preference_split(int64_t n_rows, int32_t V, pr_dtype dtype);
size_t preference_workspace_bytes(int64_t n_rows, int32_t n_pairs, int32_t G);
hipError_t launch_preference(const PreferenceArgs& a, pr_dtype dtype, hipStream_t stream);

}  // namespace pr
