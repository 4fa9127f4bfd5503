// C ABI of the verifier library: argument checks, launch-shape selection and
// the streaming state object. Every compute step runs in the kernels of
// row_features.hip, topp.hip and aggregate.hip.
#include <algorithm>
#include <cmath>
#include <mutex>
#include <new>
#include <vector>

#include "adamw.h"
#include "aggregate.h"
#include "calibrate.h"
#include "distill.h"
#include "head.h"
#include "loss.h"
#include "select.h"
#include "topp.h"

using namespace pr;

// Scratch of pr_token_features_noalloc: the split-row partial states of small
// batches, in a file-scope device array instead of a caller's workspace. Each
// GPU the library runs on holds its own copy until the process ends. In host
// code this name is only a stand-in for the symbol: its device address comes
// from hipGetSymbolAddress (see noalloc_scratch below), never from the name.
static __device__ __align__(256) unsigned char scratch[PR_NOALLOC_SCRATCH_BYTES];

struct pr_stream {
  int device;
  StreamDev dev;
  pr_agg_params params;
  Partial* ws;  // split-row workspace for up to max_slots rows of kStreamMaxSplit workgroups
  void* block;  // single allocation backing everything above
};

struct pr_adamw {
  int device;
  AdamPlan plan;
  std::vector<int64_t> chunk_begin;  // [n_tensors + 1] first chunk of each tensor
  bool has_grads;                    // every tensor of the plan has a gradient of its own
  uint64_t seed;                     // of the stochastic rounding
  void* block;                       // single allocation backing the plan
};

namespace {

constexpr int kStreamMaxSplit = 32;
// The top-p histogram packs a bin's count into 24 bits.
constexpr int32_t kTopPMaxVocab = 1 << 24;

inline hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline size_t dtype_size(pr_dtype d) { return d == PR_BF16 ? 2 : 4; }

bool features_complete(const pr_token_features_t* o) {
  return o && o->max_logit && o->lse && o->entropy && o->logprob && o->maxprob && o->margin && o->rank &&
         o->argmax && o->cutoff && o->flags;
}

pr_status check_rows(const void* logits, pr_dtype dtype, int64_t n_rows, int32_t V, int64_t row_stride,
                     const int32_t* ids, const float* temps) {
  if (dtype != PR_F32 && dtype != PR_BF16) return PR_ERR_INVALID_ARG;
  if (n_rows < 0 || V < 2 || row_stride < V) return PR_ERR_INVALID_ARG;
  if (n_rows > 0 && (!logits || !ids || !temps)) return PR_ERR_INVALID_ARG;
  if (logits && !aligned(logits, dtype_size(dtype))) return PR_ERR_INVALID_ARG;
  // Grid limits: rows * split must stay far below 2^31 workgroups.
  if (n_rows > (int64_t{1} << 26)) return PR_ERR_UNSUPPORTED;
  return PR_OK;
}

// Whether the one launch of the row kernels takes n rows, or that of the request
// kernels n requests: it has fewer than 2^32 threads (more are cut off without an
// error), 256 a row or request, 512 a row with top-p.
bool launch_fits(int64_t n, bool top_p = false) { return n < (int64_t{1} << (top_p ? 23 : 24)); }

pr_status hip_status(hipError_t e) {
  if (e == hipSuccess) return PR_OK;
  if (e == hipErrorOutOfMemory) return PR_ERR_NO_MEMORY;
  if (e == hipErrorNotSupported) return PR_ERR_UNSUPPORTED;
  return PR_ERR_HIP;
}

pr_agg_params default_params() {
  pr_agg_params p;
  p.q = 0.1;
  for (double& w : p.w) w = 0.0;
  p.w[1] = 1.0;  // mean(maxprob)
  p.b = 0.0;
  p.link = 0;
  return p;
}

// Device address of `scratch` on the device that runs `stream` (the current
// device for the NULL stream), looked up once per device with that device
// current and kept. No allocation happens here or later.
constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_ptr[kMaxDevices] = {};

pr_status noalloc_scratch(hipStream_t stream, void** out) {
  int cur = 0;
  if (hipGetDevice(&cur) != hipSuccess) return PR_ERR_HIP;
  int dev = cur;
  if (stream) {
    hipDevice_t d = 0;
    if (hipStreamGetDevice(stream, &d) != hipSuccess) return PR_ERR_HIP;
    dev = static_cast<int>(d);
  }
  if (dev < 0 || dev >= kMaxDevices) return PR_ERR_UNSUPPORTED;
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    if (dev != cur && hipSetDevice(dev) != hipSuccess) return PR_ERR_HIP;
    void* p = nullptr;
    const hipError_t e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
    if (dev != cur && hipSetDevice(cur) != hipSuccess) return PR_ERR_HIP;
    if (e != hipSuccess || !p) return PR_ERR_HIP;
    g_scratch_ptr[dev] = p;
  }
  *out = g_scratch_ptr[dev];
  return PR_OK;
}

// What a loss needs of its rows and its gradient, checked on the host.
pr_status check_loss(const void* logits, pr_dtype dtype, int64_t n_rows, int32_t V, int64_t row_stride,
                     const int32_t* ids, const float* temps, const float* weight, const float* loss, const void* grad,
                     int64_t grad_stride) {
  const pr_status st = check_rows(logits, dtype, n_rows, V, row_stride, ids, temps);
  if (st != PR_OK) return st;
  if (!loss || (n_rows > 0 && !weight)) return PR_ERR_INVALID_ARG;
  if (!grad || n_rows == 0) return PR_OK;
  if (grad_stride < V || !aligned(grad, dtype_size(dtype))) return PR_ERR_INVALID_ARG;
  if (grad == logits && grad_stride == row_stride) return PR_OK;
  // Rows of at most 2^31 elements, at most 2^26 of them: strides beyond 2^34
  // would overflow the byte offsets below and address no memory there is.
  constexpr int64_t kMostStride = int64_t{1} << 34;
  if (row_stride > kMostStride || grad_stride > kMostStride) return PR_ERR_INVALID_ARG;
  const uintptr_t item = dtype_size(dtype), n = static_cast<uintptr_t>(n_rows) - 1, v = static_cast<uintptr_t>(V);
  const uintptr_t z0 = reinterpret_cast<uintptr_t>(logits), g0 = reinterpret_cast<uintptr_t>(grad);
  const uintptr_t z1 = z0 + (n * static_cast<uintptr_t>(row_stride) + v) * item;
  const uintptr_t g1 = g0 + (n * static_cast<uintptr_t>(grad_stride) + v) * item;
  return z0 < g1 && g0 < z1 ? PR_ERR_INVALID_ARG : PR_OK;
}

LossRows loss_rows(const void* logits, int64_t n_rows, int32_t V, int64_t row_stride, const int32_t* ids,
                   const float* temps, const float* weight, void* grad, int64_t grad_stride) {
  LossRows a{};
  a.logits = logits;
  a.n_rows = n_rows;
  a.V = V;
  a.row_stride = row_stride;
  a.ids = ids;
  a.temperature = temps;
  a.weight = weight;
  a.grad = grad;
  a.grad_stride = grad_stride;
  return a;
}

// Upper 32 bits of SplitMix64's output (Steele, Lea and Flood, OOPSLA 2014)
// for a step: the key of its random numbers.
uint32_t step_key(uint64_t seed, int64_t step) {
  uint64_t x = seed + static_cast<uint64_t>(step) * 0x9E3779B97F4A7C15ull;
  x = (x ^ (x >> 30)) * 0xBF58476D1CE4E5B9ull;
  x = (x ^ (x >> 27)) * 0x94D049BB133111EBull;
  return static_cast<uint32_t>((x ^ (x >> 31)) >> 32);
}

pr_status check_beams(int32_t n_req, int32_t n_beams) {
  if (n_req < 0 || n_beams < 1) return PR_ERR_INVALID_ARG;
  if (n_beams > PR_MAX_BEAMS || n_req > INT32_MAX / n_beams) return PR_ERR_UNSUPPORTED;
  return PR_OK;
}

// Whether two states share a byte: their rows' bytes from the first to the last
// do, and they do not lie side by side in rows of one stride.
bool states_overlap(const pr_beam_state& a, const pr_beam_state& b, int64_t n) {
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.rows), b0 = reinterpret_cast<uintptr_t>(b.rows);
  const uintptr_t a1 = a0 + static_cast<uintptr_t>((n - 1) * a.row_stride + a.row_bytes);
  const uintptr_t b1 = b0 + static_cast<uintptr_t>((n - 1) * b.row_stride + b.row_bytes);
  if (a1 <= b0 || b1 <= a0) return false;
  if (a.row_stride != b.row_stride) return true;
  const int64_t s = a.row_stride, d = static_cast<int64_t>((b0 > a0 ? b0 - a0 : a0 - b0) % static_cast<uintptr_t>(s));
  const int64_t lo = b0 > a0 ? a.row_bytes : b.row_bytes, hi = b0 > a0 ? b.row_bytes : a.row_bytes;
  return d < lo || d + hi > s;
}

bool params_ok(const pr_agg_params& p) {
  if (!(p.q >= 0.0 && p.q <= 1.0)) return false;
  if (p.link != 0 && p.link != 1) return false;
  return true;
}

}  // namespace

extern "C" {

const char* pr_status_string(pr_status status) {
  switch (status) {
    case PR_OK:
      return "ok";
    case PR_ERR_INVALID_ARG:
      return "invalid argument";
    case PR_ERR_UNSUPPORTED:
      return "unsupported";
    case PR_ERR_HIP:
      return "HIP runtime error";
    case PR_ERR_NO_MEMORY:
      return "out of device memory";
  }
  return "unknown status";
}

void pr_agg_params_default(pr_agg_params* params) {
  if (params) *params = default_params();
}

size_t pr_token_features_workspace(pr_dtype dtype, int64_t n_rows, int32_t vocab, int32_t top_p_on) {
  if (n_rows <= 0 || vocab < 2) return 0;
  if (top_p_on) return topp_workspace(dtype, n_rows, vocab);
  return split_workspace_bytes(n_rows, row_split(n_rows, vocab, dtype));
}

size_t pr_token_features_workspace_full(pr_dtype dtype, int64_t n_rows, int32_t vocab, int32_t top_p_on) {
  if (n_rows <= 0 || vocab < 2) return 0;
  return top_p_on ? topp_split_workspace(n_rows, vocab, false) : pr_token_features_workspace(dtype, n_rows, vocab, 0);
}

pr_status pr_token_features(const void* logits, pr_dtype dtype, int64_t n_rows, int32_t vocab,
                            int64_t row_stride, const int32_t* sampled_ids, const float* temperature,
                            const float* top_p, const pr_token_features_t* out, void* workspace,
                            size_t workspace_bytes, void* stream) {
  return pr_token_features_ws(logits, dtype, n_rows, vocab, row_stride, sampled_ids, temperature, top_p, out,
                              top_p ? nullptr : workspace, top_p ? 0 : workspace_bytes, stream);
}

pr_status pr_token_features_ws(const void* logits, pr_dtype dtype, int64_t n_rows, int32_t vocab,
                               int64_t row_stride, const int32_t* sampled_ids, const float* temperature,
                               const float* top_p, const pr_token_features_t* out, void* workspace,
                               size_t workspace_bytes, void* stream) {
  pr_status st = check_rows(logits, dtype, n_rows, vocab, row_stride, sampled_ids, temperature);
  if (st != PR_OK) return st;
  if (!features_complete(out)) return PR_ERR_INVALID_ARG;
  const size_t need = pr_token_features_workspace(dtype, n_rows, vocab, top_p ? 1 : 0);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return PR_ERR_INVALID_ARG;
  if (top_p && workspace && !aligned(workspace, 16)) return PR_ERR_INVALID_ARG;
  if (n_rows == 0) return PR_OK;
  RowArgs a{};
  a.logits = logits;
  a.n_rows = n_rows;
  a.V = vocab;
  a.row_stride = row_stride;
  a.sampled_ids = sampled_ids;
  a.temperature = temperature;
  a.top_p = top_p;
  a.out = *out;
  if ((top_p && vocab >= kTopPMaxVocab) || !launch_fits(n_rows, top_p)) return PR_ERR_UNSUPPORTED;
  if (top_p) return hip_status(launch_topp(a, dtype, workspace, workspace_bytes, as_stream(stream)));
  a.G = row_split(n_rows, vocab, dtype);
  a.ws = static_cast<Partial*>(workspace);
  return hip_status(launch_row_features(a, dtype, as_stream(stream)));
}

pr_status pr_token_features_noalloc(const void* logits, pr_dtype dtype, int64_t n_rows, int32_t vocab,
                                    int64_t row_stride, const int32_t* sampled_ids, const float* temperature,
                                    const float* top_p, const pr_token_features_t* out, void* stream) {
  pr_status st = check_rows(logits, dtype, n_rows, vocab, row_stride, sampled_ids, temperature);
  if (st != PR_OK) return st;
  if (!features_complete(out)) return PR_ERR_INVALID_ARG;
  const size_t need = pr_token_features_workspace(dtype, n_rows, vocab, top_p ? 1 : 0);
  if (need > PR_NOALLOC_SCRATCH_BYTES) return PR_ERR_UNSUPPORTED;
  if (n_rows == 0) return PR_OK;
  void* ws = nullptr;
  if (need > 0) {
    st = noalloc_scratch(as_stream(stream), &ws);
    if (st != PR_OK) return st;
  }
  return pr_token_features(logits, dtype, n_rows, vocab, row_stride, sampled_ids, temperature, top_p, out, ws,
                           need, stream);
}

size_t pr_feature_sequence_workspace(pr_dtype dtype, int64_t n_rows, int32_t vocab, int32_t top_p_on) {
  if (vocab < 2) return 0;
  return top_p_on ? topp_split_workspace(n_rows, vocab, true) : lane_workspace_bytes(n_rows, vocab, dtype, true, false);
}

pr_status pr_feature_sequence(const void* logits, pr_dtype dtype, int64_t n_rows, int32_t vocab,
                              int64_t row_stride, const int32_t* sampled_ids, const float* temperature,
                              const float* top_p, const int32_t* offsets, int32_t n_req, int32_t top_k,
                              float* X, const pr_token_features_t* features, void* stream) {
  return pr_feature_sequence_ws(logits, dtype, n_rows, vocab, row_stride, sampled_ids, temperature, top_p, offsets,
                                n_req, top_k, X, features, nullptr, 0, stream);
}

pr_status pr_feature_sequence_ws(const void* logits, pr_dtype dtype, int64_t n_rows, int32_t vocab,
                                 int64_t row_stride, const int32_t* sampled_ids, const float* temperature,
                                 const float* top_p, const int32_t* offsets, int32_t n_req, int32_t top_k,
                                 float* X, const pr_token_features_t* features, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  pr_status st = check_rows(logits, dtype, n_rows, vocab, row_stride, sampled_ids, temperature);
  if (st != PR_OK) return st;
  if (top_k < 1 || top_k > PR_MAX_TOP_K || n_req < 0) return PR_ERR_INVALID_ARG;
  if (features && !features_complete(features)) return PR_ERR_INVALID_ARG;
  if (n_rows == 0) return PR_OK;
  if (n_req == 0 || !offsets || !X || !aligned(X, 16)) return PR_ERR_INVALID_ARG;
  RowArgs a{};
  a.logits = logits;
  a.n_rows = n_rows;
  a.V = vocab;
  a.row_stride = row_stride;
  a.sampled_ids = sampled_ids;
  a.temperature = temperature;
  a.top_p = top_p;
  if (features) a.out = *features;
  a.G = 1;
  a.X = X;
  a.offsets = offsets;
  a.n_req = n_req;
  a.top_k = top_k;
  if ((top_p && vocab >= kTopPMaxVocab) || !launch_fits(n_rows, top_p)) return PR_ERR_UNSUPPORTED;
  if (workspace && !aligned(workspace, 16)) return PR_ERR_INVALID_ARG;
  if (top_p) return hip_status(launch_topp(a, dtype, workspace, workspace_bytes, as_stream(stream)));
  const size_t need = lane_workspace_bytes(n_rows, vocab, dtype, true, false);
  if (workspace && need > 0 && workspace_bytes >= need) {
    a.G = lane_split(n_rows, vocab, dtype);
    a.ws = static_cast<Partial*>(workspace);
  }
  return hip_status(launch_feature_sequence(a, dtype, as_stream(stream)));
}

size_t pr_sample_features_workspace(pr_dtype dtype, int64_t n_rows, int32_t vocab, int32_t sequence_on) {
  return vocab < 2 ? 0 : lane_workspace_bytes(n_rows, vocab, dtype, sequence_on != 0, true);
}

pr_status pr_sample_features(const void* logits, pr_dtype dtype, int64_t n_rows, int32_t vocab, int64_t row_stride,
                             const float* temperature, uint64_t seed, uint64_t offset, int32_t* sampled_ids,
                             const pr_token_features_t* features, const int32_t* offsets, int32_t n_req,
                             int32_t top_k, float* X, void* stream) {
  return pr_sample_features_ws(logits, dtype, n_rows, vocab, row_stride, temperature, seed, offset, sampled_ids,
                               features, offsets, n_req, top_k, X, nullptr, 0, stream);
}

pr_status pr_sample_features_ws(const void* logits, pr_dtype dtype, int64_t n_rows, int32_t vocab,
                                int64_t row_stride, const float* temperature, uint64_t seed, uint64_t offset,
                                int32_t* sampled_ids, const pr_token_features_t* features, const int32_t* offsets,
                                int32_t n_req, int32_t top_k, float* X, void* workspace, size_t workspace_bytes,
                                void* stream) {
  if (dtype != PR_F32 && dtype != PR_BF16) return PR_ERR_INVALID_ARG;
  if (n_rows < 0 || vocab < 2 || row_stride < vocab) return PR_ERR_INVALID_ARG;
  if (!launch_fits(n_rows)) return PR_ERR_UNSUPPORTED;
  if (features && !features_complete(features)) return PR_ERR_INVALID_ARG;
  if (X && (top_k < 1 || top_k > PR_MAX_TOP_K || n_req < 0)) return PR_ERR_INVALID_ARG;
  if (n_rows == 0) return PR_OK;
  if (!logits || !temperature || !sampled_ids || !aligned(logits, dtype_size(dtype))) return PR_ERR_INVALID_ARG;
  if (X && (n_req == 0 || !offsets || !aligned(X, 16))) return PR_ERR_INVALID_ARG;
  RowArgs a{};
  a.logits = logits;
  a.n_rows = n_rows;
  a.V = vocab;
  a.row_stride = row_stride;
  a.sampled_ids = nullptr;
  a.temperature = temperature;
  if (features) a.out = *features;
  a.G = 1;
  a.X = X;
  a.offsets = offsets;
  a.n_req = n_req;
  a.top_k = top_k;
  a.sampled_out = sampled_ids;
  // One key per (seed, offset): the offset is spread by an odd multiplier
  // (a bijection of 64-bit words), so each offset gives its own key.
  const uint64_t key = seed ^ (offset * 0x9E3779B97F4A7C15ull);
  a.key0 = static_cast<uint32_t>(key);
  a.key1 = static_cast<uint32_t>(key >> 32);
  if (workspace && !aligned(workspace, 16)) return PR_ERR_INVALID_ARG;
  const size_t need = lane_workspace_bytes(n_rows, vocab, dtype, X != nullptr, true);
  if (workspace && need > 0 && workspace_bytes >= need) {
    a.G = lane_split(n_rows, vocab, dtype);
    a.ws = static_cast<Partial*>(workspace);
  }
  return hip_status(launch_sample(a, dtype, as_stream(stream)));
}

size_t pr_verifier_head_workspace(int64_t n_rows) { return n_rows > 0 ? head_tiles_workspace_bytes(n_rows) : 0; }

size_t pr_verifier_head_workspace_full(int64_t n_rows) { return n_rows > 0 ? head_workspace_bytes(n_rows) : 0; }

pr_status pr_verifier_head(const float* X, int64_t n_rows, const int32_t* offsets, int32_t n_req, int32_t max_len,
                           const float* weights, float* scores, void* workspace, size_t workspace_bytes,
                           void* stream) {
  if (n_rows < 0 || n_req < 0 || max_len < 1) return PR_ERR_INVALID_ARG;
  if (n_rows > (int64_t{1} << 30) || max_len > (1 << 20)) return PR_ERR_UNSUPPORTED;  // grid limits
  if (n_req == 0) return PR_OK;
  if (!offsets || !weights || !scores || !aligned(weights, 16)) return PR_ERR_INVALID_ARG;
  if (n_rows > 0 && (!X || !aligned(X, 4))) return PR_ERR_INVALID_ARG;
  const size_t need = pr_verifier_head_workspace(n_rows);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return PR_ERR_INVALID_ARG;
  HeadArgs a{};
  a.X = X;
  a.n_rows = n_rows;
  a.offsets = offsets;
  a.n_req = n_req;
  a.max_len = max_len;
  a.weights = weights;
  a.scores = scores;
  a.ws = workspace;
  if (workspace_bytes < pr_verifier_head_workspace_full(n_rows)) return hip_status(launch_head_tiles(a, as_stream(stream)));
  return hip_status(launch_head(a, as_stream(stream)));
}

pr_status pr_request_aggregate(const pr_token_features_t* feats, const int32_t* offsets, int32_t n_req,
                               const pr_agg_params* params, const pr_request_agg_t* out, void* stream) {
  if (n_req < 0 || !out) return PR_ERR_INVALID_ARG;
  if (n_req == 0) return PR_OK;
  if (!feats || !offsets || !feats->logprob || !feats->maxprob || !feats->entropy || !feats->margin)
    return PR_ERR_INVALID_ARG;
  const pr_agg_params p = params ? *params : default_params();
  if (!params_ok(p)) return PR_ERR_INVALID_ARG;
  if (!launch_fits(n_req)) return PR_ERR_UNSUPPORTED;
  return hip_status(launch_aggregate(*feats, offsets, n_req, p, *out, as_stream(stream)));
}

pr_status pr_route(const float* scores, int32_t n_req, float threshold, uint8_t* ship, int32_t* n_ship,
                   void* stream) {
  if (n_req < 0) return PR_ERR_INVALID_ARG;
  if (n_req > 0 && (!scores || !ship)) return PR_ERR_INVALID_ARG;
  if (n_req == 0 && !n_ship) return PR_OK;
  return hip_status(launch_route(scores, n_req, threshold, ship, n_ship, as_stream(stream)));
}

size_t pr_calibrate_workspace(int32_t n) { return n < 0 ? 0 : calibrate_workspace_bytes(n); }

pr_status pr_calibrate_threshold(const float* scores, int32_t n, double ship_fraction, float* tau, int32_t* n_ship,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  if (n < 0 || !tau || (n > 0 && !scores)) return PR_ERR_INVALID_ARG;
  if (!(ship_fraction >= 0.0 && ship_fraction <= 1.0)) return PR_ERR_INVALID_ARG;
  const size_t need = calibrate_workspace_bytes(n);
  if (need && (!workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 4 != 0))
    return PR_ERR_INVALID_ARG;
  return hip_status(launch_calibrate(scores, n, ship_fraction, tau, n_ship, workspace, as_stream(stream)));
}

pr_status pr_validate_offsets(const int32_t* offsets, int32_t n_req, int64_t n_rows, void* stream) {
  if (!offsets || n_req < 0) return PR_ERR_INVALID_ARG;
  int32_t* host = new (std::nothrow) int32_t[static_cast<size_t>(n_req) + 1];
  if (!host) return PR_ERR_NO_MEMORY;
  hipError_t e = hipMemcpyAsync(host, offsets, (static_cast<size_t>(n_req) + 1) * sizeof(int32_t),
                                hipMemcpyDeviceToHost, as_stream(stream));
  if (e == hipSuccess) e = hipStreamSynchronize(as_stream(stream));
  pr_status st = hip_status(e);
  if (st == PR_OK) {
    if (host[0] != 0 || host[n_req] != n_rows) st = PR_ERR_INVALID_ARG;
    for (int32_t i = 0; st == PR_OK && i < n_req; ++i)
      if (host[i + 1] < host[i]) st = PR_ERR_INVALID_ARG;
  }
  delete[] host;
  return st;
}

pr_status pr_stream_create(int32_t max_slots, int32_t max_len, const pr_agg_params* params, pr_stream** state) {
  if (!state || max_slots <= 0 || max_len < 0) return PR_ERR_INVALID_ARG;
  *state = nullptr;
  const pr_agg_params p = params ? *params : default_params();
  if (!params_ok(p)) return PR_ERR_INVALID_ARG;
  const size_t S = static_cast<size_t>(max_slots);
  const size_t L = static_cast<size_t>(max_len);
  auto up = [](size_t b) { return (b + 255) & ~size_t{255}; };
  const size_t b_ws = up(split_workspace_bytes(static_cast<int64_t>(S), kStreamMaxSplit));
  const size_t b_sum = up(S * 4 * sizeof(double));
  const size_t b_hist = up(S * 4 * L * sizeof(float));
  const size_t b_min = up(S * 4 * sizeof(float));
  const size_t b_cnt = up(S * sizeof(int32_t));
  const size_t b_nan = up(S * sizeof(uint32_t));
  const bool bounded = max_len == 0;  // P-square markers instead of the history
  const size_t b_p2q = bounded ? up(S * 20 * sizeof(double)) : 0;
  const size_t b_p2n = bounded ? up(S * 16 * sizeof(int32_t)) : 0;
  const size_t total = b_ws + b_sum + b_hist + b_min + b_cnt + b_nan + b_p2q + b_p2n;
  pr_stream* s = new (std::nothrow) pr_stream();
  if (!s) return PR_ERR_NO_MEMORY;
  hipError_t e = hipGetDevice(&s->device);
  if (e == hipSuccess) e = hipMalloc(&s->block, total);
  if (e != hipSuccess) {
    delete s;
    return hip_status(e);
  }
  char* b = static_cast<char*>(s->block);
  s->ws = reinterpret_cast<Partial*>(b);
  b += b_ws;
  s->dev.sum = reinterpret_cast<double*>(b);
  b += b_sum;
  s->dev.hist = reinterpret_cast<float*>(b);
  b += b_hist;
  s->dev.minv = reinterpret_cast<float*>(b);
  b += b_min;
  s->dev.count = reinterpret_cast<int32_t*>(b);
  b += b_cnt;
  s->dev.nanbits = reinterpret_cast<uint32_t*>(b);
  b += b_nan;
  s->dev.p2q = bounded ? reinterpret_cast<double*>(b) : nullptr;
  b += b_p2q;
  s->dev.p2n = bounded ? reinterpret_cast<int32_t*>(b) : nullptr;
  s->dev.p2p = p.q;
  if (bounded) s->dev.hist = nullptr;
  s->dev.max_slots = max_slots;
  s->dev.max_len = max_len;
  s->params = p;
  e = launch_stream_clear(s->dev, nullptr, 0, nullptr);
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    (void)hipFree(s->block);
    delete s;
    return hip_status(e);
  }
  *state = s;
  return PR_OK;
}

size_t pr_stream_step_workspace(pr_dtype, int32_t n_active, int32_t vocab, int32_t top_p_on) {
  return top_p_on ? topp_split_workspace(n_active, vocab, false) : 0;
}

pr_status pr_stream_step(pr_stream* state, const void* logits, pr_dtype dtype, int32_t n_active, int32_t vocab,
                         int64_t row_stride, const int32_t* slot_ids, const int32_t* sampled_ids,
                         const float* temperature, const float* top_p, const pr_token_features_t* out,
                         void* stream) {
  return pr_stream_step_ws(state, logits, dtype, n_active, vocab, row_stride, slot_ids, sampled_ids, temperature,
                           top_p, out, nullptr, 0, stream);
}

pr_status pr_stream_step_ws(pr_stream* state, const void* logits, pr_dtype dtype, int32_t n_active, int32_t vocab,
                            int64_t row_stride, const int32_t* slot_ids, const int32_t* sampled_ids,
                            const float* temperature, const float* top_p, const pr_token_features_t* out,
                            void* workspace, size_t workspace_bytes, void* stream) {
  if (!state) return PR_ERR_INVALID_ARG;
  pr_status st = check_rows(logits, dtype, n_active, vocab, row_stride, sampled_ids, temperature);
  if (st != PR_OK) return st;
  if (n_active > state->dev.max_slots) return PR_ERR_INVALID_ARG;
  if (n_active > 0 && !slot_ids) return PR_ERR_INVALID_ARG;
  if ((top_p && vocab >= kTopPMaxVocab) || !launch_fits(n_active, top_p)) return PR_ERR_UNSUPPORTED;
  if (out && !features_complete(out)) return PR_ERR_INVALID_ARG;
  if (workspace && !aligned(workspace, 16)) return PR_ERR_INVALID_ARG;
  if (n_active == 0) return PR_OK;
  RowArgs a{};
  a.logits = logits;
  a.n_rows = n_active;
  a.V = vocab;
  a.row_stride = row_stride;
  a.sampled_ids = sampled_ids;
  a.temperature = temperature;
  a.top_p = top_p;
  if (out) a.out = *out;
  int G = row_split(n_active, vocab, dtype);
  if (G > kStreamMaxSplit) G = kStreamMaxSplit;
  a.G = G;
  a.ws = state->ws;
  a.slot_ids = slot_ids;
  a.st = state->dev;
  if (top_p) return hip_status(launch_topp(a, dtype, workspace, workspace_bytes, as_stream(stream)));
  return hip_status(launch_row_features(a, dtype, as_stream(stream)));
}

pr_status pr_stream_finish(pr_stream* state, const int32_t* slots, int32_t n, float threshold,
                           const pr_request_agg_t* out, uint8_t* ship, void* stream) {
  if (!state || n < 0) return PR_ERR_INVALID_ARG;
  if (n == 0) return PR_OK;
  if (!slots) return PR_ERR_INVALID_ARG;
  if (!launch_fits(n)) return PR_ERR_UNSUPPORTED;
  pr_request_agg_t o{};
  if (out) o = *out;
  return hip_status(
      launch_stream_finish(state->dev, slots, n, state->params, threshold, o, ship, as_stream(stream)));
}

pr_status pr_stream_reset_slots(pr_stream* state, const int32_t* slots, int32_t n, void* stream) {
  if (!state || n < 0) return PR_ERR_INVALID_ARG;
  if (n == 0) return PR_OK;
  if (!slots) return PR_ERR_INVALID_ARG;
  return hip_status(launch_stream_clear(state->dev, slots, n, as_stream(stream)));
}

pr_status pr_stream_reorder(pr_stream* state, const int32_t* slots, const int32_t* parent, int32_t n_req,
                            int32_t n_beams, void* stream) {
  if (!state) return PR_ERR_INVALID_ARG;
  const pr_status st = check_beams(n_req, n_beams);
  if (st != PR_OK) return st;
  if (n_req == 0) return PR_OK;
  if (!slots || !parent) return PR_ERR_INVALID_ARG;
  int device = 0;
  if (hipGetDevice(&device) != hipSuccess) return PR_ERR_HIP;
  if (device != state->device) return PR_ERR_INVALID_ARG;
  const StreamDev& d = state->dev;
  StateList list{};
  auto add = [&](void* p, int64_t bytes) {
    if (p && bytes > 0) list.s[list.n++] = pr_beam_state{p, bytes, bytes};
  };
  add(d.hist, static_cast<int64_t>(d.max_len) * 16);
  add(d.sum, 32);
  add(d.minv, 16);
  add(d.count, 4);
  add(d.nanbits, 4);
  add(d.p2q, 160);
  add(d.p2n, 64);
  return hip_status(launch_reorder(list, slots, d.max_slots, parent, n_req, n_beams, as_stream(stream)));
}

void pr_stream_destroy(pr_stream* state) {
  if (!state) return;
  int prev = 0;
  (void)hipGetDevice(&prev);
  (void)hipSetDevice(state->device);
  (void)hipDeviceSynchronize();
  (void)hipFree(state->block);
  (void)hipSetDevice(prev);
  delete state;
}

size_t pr_top_logits_workspace(pr_dtype dtype, int64_t n_rows, int32_t vocab, int32_t k) {
  return vocab < 2 || k < 1 ? 0 : top_workspace_bytes(n_rows, vocab, dtype, k);
}

pr_status pr_top_logits(const void* logits, pr_dtype dtype, int64_t n_rows, int32_t vocab, int64_t row_stride,
                        const float* temperature, int32_t k, int32_t* ids, float* logprob, float* lse,
                        uint32_t* flags, void* workspace, size_t workspace_bytes, void* stream) {
  const pr_status st = check_rows(logits, dtype, n_rows, vocab, row_stride, ids, temperature);
  if (st != PR_OK) return st;
  if (k < 1 || k > PR_MAX_TOP_LOGITS || (n_rows > 0 && !logprob)) return PR_ERR_INVALID_ARG;
  const size_t need = pr_top_logits_workspace(dtype, n_rows, vocab, k);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return PR_ERR_INVALID_ARG;
  if (n_rows == 0) return PR_OK;
  TopArgs a{};
  a.logits = logits;
  a.n_rows = n_rows;
  a.V = vocab;
  a.row_stride = row_stride;
  a.temperature = temperature;
  a.k = k;
  a.ids = ids;
  a.logprob = logprob;
  a.lse = lse;
  a.flags = flags;
  a.ws = workspace;
  return hip_status(launch_top(a, dtype, as_stream(stream)));
}

size_t pr_beam_select_workspace(pr_dtype dtype, int32_t n_req, int32_t n_beams, int32_t vocab, int32_t k) {
  if (n_req < 1 || n_beams < 1 || vocab < 2 || k < 1) return 0;
  return beam_workspace_bytes(static_cast<int64_t>(n_req) * n_beams, vocab, dtype, k);
}

pr_status pr_beam_select(const void* logits, pr_dtype dtype, int32_t n_req, int32_t n_beams, int32_t vocab,
                         int64_t row_stride, const float* temperature, const float* scores, const uint8_t* done,
                         int32_t done_token, int32_t k, const pr_beam_out_t* out, void* workspace,
                         size_t workspace_bytes, void* stream) {
  pr_status st = check_beams(n_req, n_beams);
  if (st != PR_OK) return st;
  const int64_t n = static_cast<int64_t>(n_req) * n_beams;
  st = check_rows(logits, dtype, n, vocab, row_stride, reinterpret_cast<const int32_t*>(scores), temperature);
  if (st != PR_OK) return st;
  if (k < 1 || k > PR_MAX_TOP_LOGITS || !out) return PR_ERR_INVALID_ARG;
  if (n > (1 << 23)) return PR_ERR_UNSUPPORTED;
  if (n_req == 0) return PR_OK;
  if (!out->scores || !out->parent || !out->token) return PR_ERR_INVALID_ARG;
  const size_t need = pr_beam_select_workspace(dtype, n_req, n_beams, vocab, k);
  if (!workspace || workspace_bytes < need || !aligned(workspace, 16)) return PR_ERR_INVALID_ARG;
  BeamArgs a{};
  a.logits = logits;
  a.n_req = n_req;
  a.B = n_beams;
  a.V = vocab;
  a.row_stride = row_stride;
  a.temperature = temperature;
  a.scores = scores;
  a.done = done;
  a.done_token = done_token;
  a.k = k;
  a.out = *out;
  a.ws = workspace;
  return hip_status(launch_beam(a, dtype, as_stream(stream)));
}

pr_status pr_beam_reorder(const pr_beam_state* states, int32_t n_states, const int32_t* parent, int32_t n_req,
                          int32_t n_beams, void* stream) {
  const pr_status st = check_beams(n_req, n_beams);
  if (st != PR_OK) return st;
  if (n_states < 0 || (n_states > 0 && !states)) return PR_ERR_INVALID_ARG;
  const int64_t n = static_cast<int64_t>(n_req) * n_beams;
  // No device holds more; byte offsets stay below 2^63.
  constexpr int64_t kMostBytes = int64_t{1} << 42;
  for (int32_t j = 0; j < n_states; ++j) {
    const pr_beam_state& s = states[j];
    if (s.row_bytes < 0 || s.row_stride < s.row_bytes || (n > 0 && s.row_stride > kMostBytes / n))
      return PR_ERR_INVALID_ARG;
    if (n > 0 && s.row_bytes > 0 && !s.rows) return PR_ERR_INVALID_ARG;
  }
  if (n_req == 0 || n_states == 0) return PR_OK;
  if (!parent) return PR_ERR_INVALID_ARG;
  const uintptr_t p0 = reinterpret_cast<uintptr_t>(parent), p1 = p0 + static_cast<uintptr_t>(n) * sizeof(int32_t);
  for (int32_t j = 0; j < n_states; ++j) {
    const uintptr_t s0 = reinterpret_cast<uintptr_t>(states[j].rows);
    const uintptr_t s1 = s0 + static_cast<uintptr_t>((n - 1) * states[j].row_stride + states[j].row_bytes);
    if (states[j].row_bytes > 0 && s0 < p1 && p0 < s1) return PR_ERR_INVALID_ARG;
  }
  try {
    // By their first byte: a state can share bytes only with those that start before its end.
    std::vector<pr_beam_state> by(states, states + n_states);
    std::sort(by.begin(), by.end(), [](const pr_beam_state& a, const pr_beam_state& b) {
      return reinterpret_cast<uintptr_t>(a.rows) < reinterpret_cast<uintptr_t>(b.rows);
    });
    for (size_t i = 0; i < by.size(); ++i) {
      if (by[i].row_bytes == 0) continue;
      const uintptr_t end =
          reinterpret_cast<uintptr_t>(by[i].rows) + static_cast<uintptr_t>((n - 1) * by[i].row_stride + by[i].row_bytes);
      for (size_t j = i + 1; j < by.size() && reinterpret_cast<uintptr_t>(by[j].rows) < end; ++j)
        if (by[j].row_bytes > 0 && states_overlap(by[i], by[j], n)) return PR_ERR_INVALID_ARG;
    }
  } catch (...) {
    return PR_ERR_NO_MEMORY;
  }
  for (int32_t at = 0; at < n_states; at += kStates) {
    StateList list{};
    for (int32_t j = at; j < n_states && j < at + kStates; ++j)
      if (states[j].row_bytes > 0) list.s[list.n++] = states[j];
    if (list.n == 0) continue;
    const hipError_t e = launch_reorder(list, nullptr, 0, parent, n_req, n_beams, as_stream(stream));
    if (e != hipSuccess) return hip_status(e);
  }
  return PR_OK;
}

void pr_policy_params_default(pr_policy_params* params) {
  if (params) *params = pr_policy_params{0.2, 0.2, 0.0, 1.0};
}

size_t pr_policy_loss_workspace(pr_dtype dtype, int64_t n_rows, int32_t vocab) {
  return vocab < 2 ? 0 : policy_workspace_bytes(n_rows, vocab, dtype);
}

pr_status pr_policy_loss(const void* logits, pr_dtype dtype, int64_t n_rows, int32_t vocab, int64_t row_stride,
                         const int32_t* ids, const float* temperature, const float* weight, const float* advantage,
                         const float* old_logprob, const float* ref_logprob, const pr_policy_params* params,
                         float* loss, const pr_policy_tokens_t* out, void* grad, int64_t grad_stride,
                         void* workspace, size_t workspace_bytes, void* stream) {
  const pr_status st =
      check_loss(logits, dtype, n_rows, vocab, row_stride, ids, temperature, weight, loss, grad, grad_stride);
  if (st != PR_OK) return st;
  if (n_rows > 0 && (!advantage || !old_logprob)) return PR_ERR_INVALID_ARG;
  pr_policy_params p;
  pr_policy_params_default(&p);
  if (params) p = *params;
  if (!(p.clip_low >= 0.0 && p.clip_low <= 1.0) || !(p.clip_high >= 0.0) || !(p.kl_coef >= 0.0) ||
      !std::isfinite(p.kl_coef) || !std::isfinite(p.grad_scale) || (p.kl_coef > 0.0 && !ref_logprob && n_rows > 0))
    return PR_ERR_INVALID_ARG;
  const size_t need = pr_policy_loss_workspace(dtype, n_rows, vocab);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return PR_ERR_INVALID_ARG;
  PolicyArgs a{};
  a.rows = loss_rows(logits, n_rows, vocab, row_stride, ids, temperature, weight, grad, grad_stride);
  a.advantage = advantage;
  a.old_logprob = old_logprob;
  a.ref_logprob = ref_logprob;
  a.clip_lo = 1.0 - p.clip_low;
  a.clip_hi = 1.0 + p.clip_high;
  a.kl_coef = p.kl_coef;
  a.grad_scale = p.grad_scale;
  a.loss = loss;
  if (out) a.out = *out;
  a.G = policy_split(n_rows, vocab, dtype, grad != nullptr);
  a.row_loss = static_cast<double*>(workspace);
  return hip_status(launch_policy(a, dtype, as_stream(stream)));
}

void pr_preference_params_default(pr_preference_params* params) {
  if (params) *params = pr_preference_params{0.1, 0.0, 0.0, 1.0};
}

size_t pr_preference_loss_workspace(pr_dtype dtype, int64_t n_rows, int32_t vocab, int32_t n_pairs) {
  if (vocab < 2) return 0;
  return preference_workspace_bytes(n_rows, n_pairs, preference_split(n_rows, vocab, dtype));
}

pr_status pr_preference_loss(const void* logits, pr_dtype dtype, int64_t n_rows, int32_t vocab, int64_t row_stride,
                             const int32_t* ids, const float* temperature, const float* weight,
                             const int32_t* offsets, int32_t n_pairs, const float* ref_logprob,
                             const pr_preference_params* params, float* loss, const pr_preference_out_t* out,
                             void* grad, int64_t grad_stride, void* workspace, size_t workspace_bytes, void* stream) {
  const pr_status st =
      check_loss(logits, dtype, n_rows, vocab, row_stride, ids, temperature, weight, loss, grad, grad_stride);
  if (st != PR_OK) return st;
  if (n_pairs < 0 || (n_pairs > 0 && !offsets) || (n_pairs == 0 && n_rows > 0)) return PR_ERR_INVALID_ARG;
  if (n_pairs > (1 << 30) - 1) return PR_ERR_UNSUPPORTED;  // 2 n_pairs + 1 offsets are counted in 32 bits
  pr_preference_params p;
  pr_preference_params_default(&p);
  if (params) p = *params;
  if (!(p.beta > 0.0) || !std::isfinite(p.beta) || !(p.label_smoothing >= 0.0 && p.label_smoothing <= 1.0) ||
      !std::isfinite(p.margin) || !std::isfinite(p.grad_scale))
    return PR_ERR_INVALID_ARG;
  const size_t need = pr_preference_loss_workspace(dtype, n_rows, vocab, n_pairs);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return PR_ERR_INVALID_ARG;
  PreferenceArgs a{};
  a.rows = loss_rows(logits, n_rows, vocab, row_stride, ids, temperature, weight, grad, grad_stride);
  a.offsets = offsets;
  a.n_pairs = n_pairs;
  a.ref_logprob = ref_logprob;
  a.beta = p.beta;
  a.label_smoothing = p.label_smoothing;
  a.margin = p.margin;
  a.grad_scale = p.grad_scale;
  a.loss = loss;
  if (out) a.out = *out;
  a.G = preference_split(n_rows, vocab, dtype);
  a.ws = workspace;
  return hip_status(launch_preference(a, dtype, as_stream(stream)));
}

void pr_distill_params_default(pr_distill_params* params) {
  if (params) *params = pr_distill_params{PR_TAIL_REST, 1.0};
}

size_t pr_distill_loss_workspace(pr_dtype dtype, int64_t n_rows, int32_t vocab, int32_t k) {
  return vocab < 2 ? 0 : distill_workspace_bytes(n_rows, vocab, dtype, k);
}

pr_status pr_distill_loss(const void* logits, pr_dtype dtype, int64_t n_rows, int32_t vocab, int64_t row_stride,
                          const int32_t* top_ids, const float* top_logprob, int32_t k, int64_t top_stride,
                          const float* temperature, const float* weight, const pr_distill_params* params, float* loss,
                          const pr_distill_tokens_t* out, void* grad, int64_t grad_stride, void* workspace,
                          size_t workspace_bytes, void* stream) {
  // The rows' ids may be missing where there are no entries.
  const int32_t* ids = k > 0 ? top_ids : reinterpret_cast<const int32_t*>(weight);
  const pr_status st =
      check_loss(logits, dtype, n_rows, vocab, row_stride, ids, temperature, weight, loss, grad, grad_stride);
  if (st != PR_OK) return st;
  if (k < 0 || k > PR_MAX_TOP_LOGITS || top_stride < k || (k > 0 && n_rows > 0 && !top_logprob))
    return PR_ERR_INVALID_ARG;
  pr_distill_params p;
  pr_distill_params_default(&p);
  if (params) p = *params;
  if (p.tail < PR_TAIL_DROP || p.tail > PR_TAIL_REST || !std::isfinite(p.grad_scale)) return PR_ERR_INVALID_ARG;
  const size_t need = pr_distill_loss_workspace(dtype, n_rows, vocab, k);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return PR_ERR_INVALID_ARG;
  DistillArgs a{};
  a.rows = loss_rows(logits, n_rows, vocab, row_stride, nullptr, temperature, weight, grad, grad_stride);
  a.top_ids = top_ids;
  a.top_logprob = top_logprob;
  a.k = k;
  a.top_stride = top_stride;
  a.tail = p.tail;
  a.grad_scale = p.grad_scale;
  a.loss = loss;
  if (out) a.out = *out;
  a.ws = workspace;
  return hip_status(launch_distill(a, dtype, as_stream(stream)));
}

pr_status pr_adamw_create(const pr_adamw_tensor* tensors, int32_t n_tensors, pr_dtype param_dtype,
                          pr_dtype grad_dtype, int32_t state_bits, uint64_t seed, pr_adamw** handle) {
  if (!handle) return PR_ERR_INVALID_ARG;
  *handle = nullptr;
  if (n_tensors < 0 || (n_tensors > 0 && !tensors)) return PR_ERR_INVALID_ARG;
  if (n_tensors > (1 << 20)) return PR_ERR_UNSUPPORTED;
  if ((param_dtype != PR_F32 && param_dtype != PR_BF16) || (grad_dtype != PR_F32 && grad_dtype != PR_BF16) ||
      (state_bits != 8 && state_bits != 32))
    return PR_ERR_INVALID_ARG;
  const size_t state = state_bits == 8 ? 1 : 4;
  for (int32_t j = 0; j < n_tensors; ++j) {
    const pr_adamw_tensor& t = tensors[j];
    if (t.n < 0 || t.n > (int64_t{1} << 38)) return PR_ERR_INVALID_ARG;  // more than a device holds
    if (t.n == 0) continue;
    if (!t.param || !t.m || !t.v || !aligned(t.param, dtype_size(param_dtype)) || !aligned(t.m, state) ||
        !aligned(t.v, state) || (t.grad && !aligned(t.grad, dtype_size(grad_dtype))))
      return PR_ERR_INVALID_ARG;
    if (state_bits == 8 && (!t.m_exp || !t.v_exp)) return PR_ERR_INVALID_ARG;
    if (t.copy && (param_dtype != PR_F32 || !aligned(t.copy, 2))) return PR_ERR_INVALID_ARG;
  }
  try {
    pr_adamw* h = new pr_adamw();
    h->block = nullptr;
    h->has_grads = true;
    std::vector<AdamChunk> chunks;
    hipError_t e = hipSuccess;
    int64_t elements = 0;
    const int64_t element_bytes = static_cast<int64_t>(dtype_size(param_dtype) + dtype_size(grad_dtype) + 2 * state);
    try {
      h->chunk_begin.resize(static_cast<size_t>(n_tensors) + 1);
      int64_t block = 0, total = 0;
      for (int32_t j = 0; j < n_tensors; ++j) {
        total += (tensors[j].n + kAdamChunk - 1) / kAdamChunk;
        elements += tensors[j].n;
      }
      chunks.reserve(static_cast<size_t>(total));
      const int64_t p_item = static_cast<int64_t>(dtype_size(param_dtype)), s_item = static_cast<int64_t>(state);
      const int64_t g_item = static_cast<int64_t>(dtype_size(grad_dtype));
      auto past = [](auto* p, int64_t bytes) -> decltype(p) {
        return p ? (decltype(p))((const char*)p + bytes) : nullptr;
      };
      for (int32_t j = 0; j < n_tensors; ++j) {
        const pr_adamw_tensor& t = tensors[j];
        h->chunk_begin[static_cast<size_t>(j)] = static_cast<int64_t>(chunks.size());
        if (t.n > 0 && !t.grad) h->has_grads = false;
        for (int64_t at = 0; at < t.n; at += kAdamChunk) {
          const int64_t n = t.n - at < kAdamChunk ? t.n - at : kAdamChunk, k = at / kAdamBlock;
          chunks.push_back(AdamChunk{past(t.param, at * p_item), past(t.grad, at * g_item),
                                     past(static_cast<uint16_t*>(t.copy), at * 2), past(t.m, at * s_item),
                                     past(t.v, at * s_item), past(t.m_exp, k), past(t.v_exp, k), at, block + k,
                                     static_cast<int32_t>(n), j});
        }
        block += (t.n + kAdamBlock - 1) / kAdamBlock;
      }
      h->chunk_begin[static_cast<size_t>(n_tensors)] = static_cast<int64_t>(chunks.size());
      const size_t bytes = chunks.size() * sizeof(AdamChunk);
      e = hipGetDevice(&h->device);
      if (e == hipSuccess && bytes > 0) {
        e = hipMalloc(&h->block, bytes);
        if (e == hipSuccess) e = hipMemcpy(h->block, chunks.data(), bytes, hipMemcpyHostToDevice);
        h->plan.chunks = static_cast<const AdamChunk*>(h->block);
      }
    } catch (...) {
      delete h;
      throw;
    }
    if (e != hipSuccess) {
      if (h->block) (void)hipFree(h->block);
      delete h;
      return hip_status(e);
    }
    h->plan.param_dtype = param_dtype;
    h->plan.grad_dtype = grad_dtype;
    h->plan.state_bits = state_bits;
    h->plan.streamed = elements * element_bytes > kAdamCached;
    h->seed = seed;
    *handle = h;
    return PR_OK;
  } catch (...) {
    return PR_ERR_NO_MEMORY;
  }
}

pr_status pr_adamw_step(pr_adamw* handle, const void* const* grads, const pr_adamw_params* params, void* stream) {
  if (!handle || !params) return PR_ERR_INVALID_ARG;
  const pr_adamw_params& p = *params;
  for (const double v : {p.lr, p.beta1, p.beta2, p.eps, p.weight_decay, p.grad_scale})
    if (!std::isfinite(v)) return PR_ERR_INVALID_ARG;
  if (!(p.beta1 >= 0.0 && p.beta1 < 1.0) || !(p.beta2 >= 0.0 && p.beta2 < 1.0) || !(p.eps >= 0.0) || p.step < 1)
    return PR_ERR_INVALID_ARG;
  if (!grads && !handle->has_grads) return PR_ERR_INVALID_ARG;
  AdamScalars s{};
  s.beta1 = static_cast<float>(p.beta1);
  s.one_minus_beta1 = static_cast<float>(1.0 - p.beta1);
  s.beta2 = static_cast<float>(p.beta2);
  s.one_minus_beta2 = static_cast<float>(1.0 - p.beta2);
  s.decay = static_cast<float>(p.lr * p.weight_decay);
  s.keep = static_cast<float>(1.0 - p.lr * p.weight_decay);
  s.rate = static_cast<float>(p.lr / (1.0 - std::pow(p.beta1, static_cast<double>(p.step))));
  s.c2 = static_cast<float>(1.0 / std::sqrt(1.0 - std::pow(p.beta2, static_cast<double>(p.step))));
  s.eps = static_cast<float>(p.eps);
  s.grad_scale = static_cast<float>(p.grad_scale);
  // Roots of values below 2^-126 are below 1.1e-19: times c2 a part in 10^7 of such an eps.
  s.tiny_eps = p.eps < 1e-12 * static_cast<double>(s.c2);
  s.key = step_key(handle->seed, p.step);
  const int32_t n = static_cast<int32_t>(handle->chunk_begin.size()) - 1;
  if (!grads)
    return hip_status(
        launch_adamw(handle->plan, 0, handle->chunk_begin[static_cast<size_t>(n)], s, nullptr, as_stream(stream)));
  const size_t item = dtype_size(handle->plan.grad_dtype);
  for (int32_t j = 0; j < n; ++j)
    if (grads[j] && !aligned(grads[j], item)) return PR_ERR_INVALID_ARG;
  for (int32_t j = 0; j < n; j += kAdamGrads) {
    const int32_t to = n - j < kAdamGrads ? n : j + kAdamGrads;
    AdamGrads g{};
    g.first = j;
    for (int32_t i = j; i < to; ++i) g.p[i - j] = grads[i];
    const hipError_t e = launch_adamw(handle->plan, handle->chunk_begin[static_cast<size_t>(j)],
                                      handle->chunk_begin[static_cast<size_t>(to)], s, &g, as_stream(stream));
    if (e != hipSuccess) return hip_status(e);
  }
  return PR_OK;
}

pr_status pr_adamw_moments(pr_adamw* handle, void* m, void* v, void* stream) {
  if (!handle) return PR_ERR_INVALID_ARG;
  if (handle->plan.state_bits != 8) return PR_ERR_UNSUPPORTED;
  const int64_t chunks = handle->chunk_begin.back();
  if (chunks == 0) return PR_OK;
  if (!m || !v || !aligned(m, 2) || !aligned(v, 2)) return PR_ERR_INVALID_ARG;
  return hip_status(launch_adamw_moments(handle->plan, chunks, static_cast<uint16_t*>(m), static_cast<uint16_t*>(v),
                                         as_stream(stream)));
}

void pr_adamw_destroy(pr_adamw* handle) {
  if (!handle) return;
  int prev = 0;
  (void)hipGetDevice(&prev);
  (void)hipSetDevice(handle->device);
  (void)hipDeviceSynchronize();
  (void)hipFree(handle->block);
  (void)hipSetDevice(prev);
  delete handle;
}

}  // extern "C"
