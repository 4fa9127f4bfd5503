// Launch interface of the distillation loss (internal).
#pragma once

#include "loss.h"

namespace pr {

struct DistillArgs {
  LossRows rows;  // ids are not used
  const int32_t* top_ids;
  const float* top_logprob;
  int32_t k;
  int64_t top_stride;
  pr_tail tail;
  double grad_scale;
  float* loss;
  pr_distill_tokens_t out;
  void* ws;
};

size_t distill_workspace_bytes(int64_t n_rows, int32_t V, pr_dtype dtype, int32_t k);
hipError_t launch_distill(const DistillArgs& a, pr_dtype dtype, hipStream_t stream);

}  // namespace pr
