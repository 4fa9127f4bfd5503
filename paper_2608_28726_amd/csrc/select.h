// Launch interface of the largest logits of rows and of beam search's selection,
// and of the reordering of states (internal).
#pragma once

#include "row_features.h"

namespace pr {

struct TopArgs {
  const void* logits;
  int64_t n_rows;
  int32_t V;
  int64_t row_stride;
  const float* temperature;
  int32_t k;
  int32_t* ids;    // [n_rows][k]
  float* logprob;  // [n_rows][k]
  float* lse;      // [n_rows]
  uint32_t* flags;
  int G;  // workgroups per row (set by the launch)
  void* ws;
};

struct BeamArgs {
  const void* logits;
  int32_t n_req, B;
  int32_t V;
  int64_t row_stride;
  const float* temperature;
  const float* scores;  // [n_req][B]
  const uint8_t* done;  // [n_req][B], NULL: none
  int32_t done_token;
  int32_t k;
  pr_beam_out_t out;
  int G;  // workgroups per row (set by the launch)
  void* ws;
};

size_t top_workspace_bytes(int64_t n_rows, int32_t V, pr_dtype dtype, int32_t k);
hipError_t launch_top(const TopArgs& a, pr_dtype dtype, hipStream_t stream);

size_t beam_workspace_bytes(int64_t n_rows, int32_t V, pr_dtype dtype, int32_t k);
hipError_t launch_beam(const BeamArgs& a, pr_dtype dtype, hipStream_t stream);

// Rows of bytes that move together: row rows[i B + b] (i B + b when rows is
// NULL) of each state takes what row rows[i B + parent[i B + b]] held.
constexpr int kStates = 96;  // of one launch, by value
struct StateList {
  pr_beam_state s[kStates];
  int32_t n;
};

hipError_t launch_reorder(const StateList& states, const int32_t* rows, int32_t n_rows, const int32_t* parent,
                          int32_t n_req, int32_t B, hipStream_t stream);

}  // namespace pr
