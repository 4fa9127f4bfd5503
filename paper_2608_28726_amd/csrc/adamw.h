// Launch interface of the optimizer's step over many tensors (internal).
#pragma once

#include "device_util.h"

namespace pr {

constexpr int kAdamBlock = PR_ADAMW_BLOCK;  // elements that share an exponent
constexpr int kAdamGrads = 400;             // gradient pointers that travel with a launch

// One tensor of the plan, on the device.
struct AdamTensor {
  void* param;
  const void* grad;
  uint16_t* copy;
  void* m;
  void* v;
  uint8_t* m_exp;
  uint8_t* v_exp;
  int64_t n;
  int64_t first_block;  // blocks of the tensors before it
};

// One workgroup's share: a chunk of a tensor.
struct AdamChunk {
  int32_t tensor;
  int32_t chunk;
};

// Elements of a chunk.
constexpr int64_t kAdamChunk = 4096;

struct AdamScalars {
  float beta1, one_minus_beta1, beta2, one_minus_beta2;
  float decay;      // 1 - lr weight_decay
  float rate;       // lr c1
  float c2, eps;
  float grad_scale;
  uint32_t key;     // of the step's random numbers
};

struct AdamPlan {
  const AdamTensor* tensors;
  const AdamChunk* chunks;
  pr_dtype param_dtype, grad_dtype;
  int32_t state_bits;
};

// Gradient pointers of the tensors from `first` on.
struct AdamGrads {
  const void* p[kAdamGrads];
};

// Chunks [begin, end) of the plan. grads: those of the tensors from `first`
// on, or NULL: the plan's own.
hipError_t launch_adamw(const AdamPlan& plan, int64_t begin, int64_t end, const AdamScalars& s, const AdamGrads* grads,
                        int32_t first, hipStream_t stream);

hipError_t launch_adamw_moments(const AdamPlan& plan, int64_t n_chunks, uint16_t* m, uint16_t* v, hipStream_t stream);

}  // namespace pr
