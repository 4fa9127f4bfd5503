// Launch interface of the optimizer's step over many tensors (internal).
#pragma once

#include "device_util.h"

namespace pr {

constexpr int kAdamBlock = PR_ADAMW_BLOCK;  // elements that share an exponent
constexpr int kAdamGrads = 400;             // gradient pointers that travel with a launch
constexpr int kAdamChunk = 2048;            // most elements of a chunk

// What one workgroup takes: a chunk of a tensor. The pointers are those of
// the chunk's first element, so that a workgroup's loads wait for one read of
// the plan.
struct AdamChunk {
  void* param;
  const void* grad;  // NULL: given at the step
  uint16_t* copy;
  void* m;
  void* v;
  uint8_t* m_exp;
  uint8_t* v_exp;
  int64_t first;     // the chunk's first element in its tensor
  int64_t block;     // and its block among those of all tensors
  int32_t n;
  int32_t tensor;
};

struct AdamScalars {
  float beta1, one_minus_beta1, beta2, one_minus_beta2;
  float decay;       // lr weight_decay
  float keep;        // 1 - lr weight_decay
  float rate;        // lr c1
  float c2, eps;
  float grad_scale;
  uint32_t key;      // of the step's random numbers
  int32_t tiny_eps;  // eps does not dwarf c2 times the roots of values that the fast square root takes for 0
};

struct AdamPlan {
  const AdamChunk* chunks;
  pr_dtype param_dtype, grad_dtype;
  int32_t state_bits;
  bool streamed;  // a step touches more than the last-level cache holds
};

// Bytes of the last-level cache: a step over more gains by going past the
// caches (216 million elements, 32-bit states: 1,196 -> 1,078 us, 8-bit ones
// 650 -> 599), a smaller one finds there what the pass before it left.
constexpr int64_t kAdamCached = int64_t{256} << 20;

// Gradient pointers of the tensors from `first` on.
struct AdamGrads {
  int32_t first;
  const void* p[kAdamGrads];
};

// Chunks [begin, end) of the plan, with these gradients or (NULL) the plan's own.
hipError_t launch_adamw(const AdamPlan& plan, int64_t begin, int64_t end, const AdamScalars& s, const AdamGrads* grads,
                        hipStream_t stream);

hipError_t launch_adamw_moments(const AdamPlan& plan, int64_t n_chunks, uint16_t* m, uint16_t* v, hipStream_t stream);

}  // namespace pr
