// Rows that a workgroup holds in registers between their sum and their gradient
// (internal, device code only).
#pragma once

#include "loss.h"
#include "row_sum.h"

namespace pr {

constexpr int kCUs = 256;  // compute units of the device

template <typename Tin>
__device__ __forceinline__ const Tin* row_ptr(const LossRows& a, int64_t r) {
  return static_cast<const Tin*>(a.logits) + r * a.row_stride;
}

// Makes the compiler forget what it knows of a vector, so that it unpacks it
// anew in each pass instead of keeping 8 floats of each through all of them.
__device__ __forceinline__ void forget(vec4u& v) { asm volatile("" : "+v"(v)); }

// A row as the fused kernels see it: its vectors start at the first 16-byte
// boundary, h elements in; up to 2 x 7 elements before and after are scalars.
template <typename Tin>
struct RowView {
  const Tin* row;
  Tin* out;
  int32_t h, nvec;

  __device__ __forceinline__ RowView(const LossRows& a, int64_t r) {
    row = row_ptr<Tin>(a, r);
    out = static_cast<Tin*>(a.grad) + r * a.grad_stride;
    h = static_cast<int32_t>(head_elems<Tin>(row, a.V));
    nvec = (a.V - h) / Elem<Tin>::kVec;
  }
  __device__ __forceinline__ int32_t tail() const { return h + nvec * Elem<Tin>::kVec; }
  // Vector at + t of the row and of its gradient: a place that the wave shares
  // plus 16 t, so that an address takes one register of a lane.
  __device__ __forceinline__ const vec4u* in(int32_t at, uint32_t t) const {
    return reinterpret_cast<const vec4u*>(reinterpret_cast<const char*>(row + h) + static_cast<int64_t>(at) * 16 +
                                          t * 16u);
  }
  __device__ __forceinline__ Tin* to(int32_t at, uint32_t t) const {
    return reinterpret_cast<Tin*>(reinterpret_cast<char*>(out + h) + static_cast<int64_t>(at) * 16 + t * 16u);
  }
};

// Vectors of the rows that policy_row_kernel holds, by its two sizes (two and
// one workgroups a compute unit). Shorter rows than the least take two passes:
// what a workgroup spends on a row beside its vectors then costs more than the
// second read. 1.2 GB of rows that all count, held and in two passes (us, in
// brackets the row's vectors): bfloat16 16,384 logits a row (2,048) 710 and
// 615, 24,000 (3,000) 593 and 580, 32,000 (4,000) 535 and 575, 50,257 510 and
// 596, 65,536 475 and 569, 70,000 (8,750, the larger size) 496 and 588, 100,000
// 487 and 570, 151,936 484 and 574; float32 8,192 (2,048) 669 and 601, 12,000
// (3,000) 566 and 571, 16,000 (4,000) 521 and 580, 32,000 484 and 565, 40,000
// (10,000, the larger size) 464 and 585. Fewer rows of 32,000 bfloat16 logits:
// 128 rows 11.7 and 13.6, 512 18.4 and 23.9, 1,000 31 and 39. Batches that the
// last-level cache keeps between two passes are the exception, and only long
// rows among them: of 151,936 bfloat16 logits 300 rows 62 and 54, 512 79.6 and
// 79.8, 1,024 143 and 155.
constexpr int64_t kLeastRowVectors = 3500, kSmallRowVectors = 19 * 7 * kWave, kRowVectors = 20 * 15 * kWave;
inline bool held_row(int64_t nvec) { return nvec >= kLeastRowVectors && nvec <= kRowVectors; }

// Below this many rows a row may be spread over workgroups. Spread and whole,
// preference loss: 64 rows of 50,257 bfloat16 logits 14.4 and 17.1 us, of
// 151,936 float32 logits 30.5 and 41.0; 128 rows 17.5 and 19.6, 47.2 and 53.7;
// 200 rows 23.1 and 22.3, 66.8 and 68.5; 256 rows 25.1 and 24.7, 83.1 and 80.5;
// 400 rows 32.7 and 31.2, 126 and 124.
constexpr int64_t kSplitRows = 256;

// Few rows whose gradient is wanted are spread over the device although they
// fit a workgroup: one compute unit alone takes 20 us for 304 KB. Captured
// calls, spread and held: 16 rows of 151,936 bfloat16 logits 11.7 and 21.6 us,
// 64 rows 19.5 and 24.2, 96 rows 24.5 and 24.9, 128 rows 29.3 and 25.7, of 40,000
// float32 logits 32 rows 11.0 and 12.3, 64 rows 14.2 and 13.5; 16 rows of 32,000
// float32 logits 8.5 and 11.0, 32 rows 11.2 and 11.4, 64 rows 12.6 and 12.0.
constexpr int64_t kFewRows = 64, kFewSmallRows = 32;

// Most workgroups that each work out their own row's factors: it saves a
// launch, 1 to 2 us, and costs more than that past this many.
constexpr int64_t kFewGroups = 512;

// Most rows whose order a kernel works out for itself.
constexpr int64_t kListedRows = 65536;
constexpr int kListed = kListedRows / kCUs + 1;

// The rows of workgroup b of G: of the rows that count (weight not 0) those of
// rank b, b + G, .., and likewise of the others, as lists when there are more
// rows than workgroups and no more than kListedRows. Each thread counts a stretch
// of rows; the counts' prefix sums give the ranks. Every thread of the WAVES
// waves calls it; sh_n has WAVES entries.
struct RowDeal {
  bool listed;
  uint32_t n_on, n_off;  // of the lists
};

template <int WAVES>
__device__ __forceinline__ RowDeal deal_rows(const float* weight, int64_t n, int64_t G, int32_t* rows_on,
                                             int32_t* rows_off, uint32_t* sh_n) {
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
  RowDeal d{n > G && n <= kListedRows, 0, 0};
  if (!d.listed) return d;
  const uint32_t per = static_cast<uint32_t>((n + blockDim.x - 1) / blockDim.x);
  const uint32_t lo = min(static_cast<uint32_t>(n), threadIdx.x * per), hi = min(static_cast<uint32_t>(n), lo + per);
  uint32_t on = 0;
  for (uint32_t i = lo; i < hi; ++i) on += weight[i] != 0.0f ? 1u : 0u;
  const uint32_t scan = wave_incl_scan_u(on);
  if (lane == kWave - 1) sh_n[wave] = scan;
  __syncthreads();
  uint32_t rank = scan - on;
  for (int k = 0; k < WAVES; ++k) {
    if (k < wave) rank += sh_n[k];
    d.n_on += sh_n[k];
  }
  d.n_off = static_cast<uint32_t>(n) - d.n_on;
  for (uint32_t i = lo; i < hi; ++i) {
    const bool counts = weight[i] != 0.0f;
    const uint32_t k = counts ? rank : i - rank;
    if (k % static_cast<uint32_t>(G) == blockIdx.x) (counts ? rows_on : rows_off)[k / G] = static_cast<int32_t>(i);
    rank += counts ? 1u : 0u;
  }
  __syncthreads();
  const uint32_t b = blockIdx.x, g = static_cast<uint32_t>(G);
  d.n_on = d.n_on > b ? (d.n_on - b - 1) / g + 1 : 0u;
  d.n_off = d.n_off > b ? (d.n_off - b - 1) / g + 1 : 0u;
  return d;
}

}  // namespace pr
