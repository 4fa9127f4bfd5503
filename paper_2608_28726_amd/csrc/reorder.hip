// Beam search's reordering of states: rows of bytes that take another row's
// place within their request, in place.
//
// A thread owns 16 bytes of the rows of one request: it reads them of every row
// that another row takes, then writes them, so that nothing is overwritten
// before it is read and no scratch is needed. Rows that stay are neither read
// (unless another takes them) nor written. Memory bounds it: 64 requests of 4
// beams, 798 MB read and written in 129 us (6.2 TB/s).
#include "select.h"

namespace pr {
namespace {

constexpr int kBlock = 256;

// States start and end at any byte; global loads and stores need no alignment.
typedef uint32_t Bytes16 __attribute__((ext_vector_type(4), aligned(1)));

// Past the caches (PAST) only where the states are far larger than the last-level
// cache and a thread holds few rows. Cached and past the caches, us: 64 requests
// of 4 beams, eight states of 128 tokens of 512 bytes (134 MB) 27.7 and 33.4, of
// 256 tokens 52.6 and 65.8, of 512 tokens (537 MB) 134.8 and 129.2; as many bytes
// as 32 x 8 beams 162 and 167, 16 x 16 187 and 197, 8 x 32 223 and 220, 4 x 64
// (cached) 235: from 9 beams on the row numbers, which all lanes share, exceed the
// scalar registers (79, 308 and 863 are spilled with up to 16, 32 and 64 beams),
// and with more than 16 the rows' vectors leave 3 and 1 waves a SIMD.
constexpr int64_t kCachedStates = 400'000'000;

// Workgroups along a row: 8, 16, 32 and 64 of them took 154, 140, 129 and 129 us
// for the 537 MB above.
constexpr int64_t kMostParts = 64;

template <bool NT>
__device__ __forceinline__ vec4u load16(const char* p) {
  const Bytes16* q = reinterpret_cast<const Bytes16*>(p);
  if (NT) return static_cast<vec4u>(__builtin_nontemporal_load(q));
  return static_cast<vec4u>(*q);
}
template <bool NT>
__device__ __forceinline__ void store16(char* p, vec4u v) {
  Bytes16* q = reinterpret_cast<Bytes16*>(p);
  if (NT) __builtin_nontemporal_store(static_cast<Bytes16>(v), q);
  else *q = static_cast<Bytes16>(v);
}

template <int MOST, bool PAST>
__global__ __launch_bounds__(kBlock) void reorder_kernel(StateList states, const int32_t* rows, int32_t n_rows,
                                                         const int32_t* parent, int32_t B) {
  __shared__ int32_t sh_to[MOST], sh_from[MOST];
  const int64_t first = static_cast<int64_t>(blockIdx.y) * B;
  const pr_beam_state s = states.s[blockIdx.z];
  if (threadIdx.x < MOST) {
    const int b = threadIdx.x;
    int32_t to = -1, from = -1;
    if (b < B) {
      const int32_t p = parent[first + b];
      if (p >= 0 && p < B && p != b) {
        to = rows ? rows[first + b] : static_cast<int32_t>(first + b);
        from = rows ? rows[first + p] : static_cast<int32_t>(first + p);
        if (to < 0 || to >= n_rows || from < 0 || from >= n_rows) to = -1;
      }
    }
    sh_to[b] = to;
    sh_from[b] = from;
  }
  __syncthreads();
  // As wave-uniform values, so that a row that stays costs a branch.
  int32_t to[MOST], from[MOST];
#pragma unroll
  for (int b = 0; b < MOST; ++b) {
    to[b] = __builtin_amdgcn_readfirstlane(sh_to[b]);
    from[b] = __builtin_amdgcn_readfirstlane(sh_from[b]);
  }
  char* const base = static_cast<char*>(s.rows);
  const int64_t whole = s.row_bytes / 16;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kBlock;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x; i < whole; i += step) {
    vec4u v[MOST];
#pragma unroll
    for (int b = 0; b < MOST; ++b)
      if (to[b] >= 0) v[b] = load16<PAST>(base + from[b] * s.row_stride + i * 16);
#pragma unroll
    for (int b = 0; b < MOST; ++b)
      if (to[b] >= 0) store16<PAST>(base + to[b] * s.row_stride + i * 16, v[b]);
  }
  // The up to 15 bytes after them, one a thread.
  const int64_t last = whole * 16 + threadIdx.x;
  if (blockIdx.x == 0 && last < s.row_bytes) {
    char v[MOST];
#pragma unroll
    for (int b = 0; b < MOST; ++b)
      if (to[b] >= 0) v[b] = base[from[b] * s.row_stride + last];
#pragma unroll
    for (int b = 0; b < MOST; ++b)
      if (to[b] >= 0) base[to[b] * s.row_stride + last] = v[b];
  }
}

}  // namespace

hipError_t launch_reorder(const StateList& states, const int32_t* rows, int32_t n_rows, const int32_t* parent,
                          int32_t n_req, int32_t B, hipStream_t stream) {
  int64_t most = 0, bytes = 0;
  for (int j = 0; j < states.n; ++j) {
    most = states.s[j].row_bytes > most ? states.s[j].row_bytes : most;
    bytes += states.s[j].row_bytes * n_req * B;
  }
  const int64_t parts = (most / 16 + kBlock - 1) / kBlock;
  constexpr int32_t kMostY = 32768;
  for (int32_t at = 0; at < n_req; at += kMostY) {
    const int32_t reqs = n_req - at < kMostY ? n_req - at : kMostY;
    const dim3 grid(static_cast<unsigned>(parts < 1 ? 1 : parts > kMostParts ? kMostParts : parts), static_cast<unsigned>(reqs),
                    static_cast<unsigned>(states.n));
    StateList list = states;
    const int64_t skip = static_cast<int64_t>(at) * B;
    if (!rows)
      for (int j = 0; j < list.n; ++j)
        list.s[j].rows = static_cast<char*>(list.s[j].rows) + skip * list.s[j].row_stride;
    auto run = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, stream, list, rows ? rows + skip : nullptr,
                         rows ? n_rows : reqs * B, parent + skip, B);
    };
    const bool past = B <= 4 && bytes > kCachedStates;
    if (past)
      run(reorder_kernel<4, true>);
    else if (B <= 4)
      run(reorder_kernel<4, false>);
    else if (B <= 8)
      run(reorder_kernel<8, false>);
    else if (B <= 16)
      run(reorder_kernel<16, false>);
    else if (B <= 32)
      run(reorder_kernel<32, false>);
    else
      run(reorder_kernel<64, false>);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace pr
