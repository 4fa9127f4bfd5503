// The k largest logits of each row with their log-probs, and beam search's
// selection over the beams of a request.
//
// A row's tokens are in the order of the verifier's features: larger logit
// first, equal ones by lower index. As numbers: the logit's order-preserving
// key above the complement of the index, 64 bits, all different; larger is
// earlier and 0 is none. A logit of -inf is none. What is selected is exact.
//
// Log-probs are those of the losses: the row's float32 sum of exps, compensated
// per lane; what follows in 64 bits. A beam's candidates follow its own tokens'
// order, so the k best of a request are among the k first tokens of each beam.
#include "select.h"
#include "row_sum.h"

namespace pr {
namespace {

constexpr int kMaxTop = PR_MAX_TOP_LOGITS;
constexpr int kRowBlock = 256;
constexpr int kBeamBlock = 256;
static_assert(kRowBlock >= kMaxTop && kBeamBlock >= kMaxTop, "a thread for each of the selected");

__device__ __forceinline__ uint64_t place_key(float z, int64_t i) {
  return z == -INFINITY ? 0u : static_cast<uint64_t>(float_key(z)) << 32 | (0xffffffffu - static_cast<uint32_t>(i));
}
__device__ __forceinline__ float key_logit(uint64_t k) { return key_float(static_cast<uint32_t>(k >> 32)); }
__device__ __forceinline__ int32_t key_index(uint64_t k) {
  return static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(k));
}

// Order-preserving key of a finite double.
__device__ __forceinline__ uint64_t score_key(double s) {
  const uint64_t b = static_cast<uint64_t>(__double_as_longlong(s == 0.0 ? 0.0 : s));
  return b >> 63 ? ~b : b | 0x8000000000000000ull;
}

struct CutLds {
  uint32_t hist[256];
  uint32_t digit, need, bin, total;
};

// Which keys are the k largest: those with (key & mask) >= value, and `more`
// says that of those with (key & mask) == value only `need` are among them.
struct Cut {
  uint64_t value, mask;
  uint32_t need;
  bool more;
  __device__ __forceinline__ bool takes(uint64_t key) const { return key != 0 && (key & mask) >= value; }
  __device__ __forceinline__ bool above(uint64_t key) const { return key != 0 && (key & mask) > value; }
};

// The cut of the k largest of the keys that the workgroup's threads pass to
// `keys` (each calls keys(fn), and fn(key) for each of its keys; 0 is no key),
// by digits of 8 bits from the top until a digit's keys are all taken. SKIP:
// digits, counted from the top by bits, that are the same for all keys whose
// earlier digits are. Every thread calls it; a barrier follows its last read.
template <int BLOCK, uint32_t SKIP, typename Keys>
__device__ Cut find_cut(Keys&& keys, uint32_t k, CutLds& s) {
  Cut c{0, 0, k, false};
  for (int pass = 0; pass < 8; ++pass) {
    if (SKIP >> pass & 1u) continue;
    const int shift = 56 - 8 * pass;
    for (int b = threadIdx.x; b < 256; b += BLOCK) s.hist[b] = 0;
    __syncthreads();
    keys([&](uint64_t key) {
      if (key != 0 && (key & c.mask) == c.value) atomicAdd(&s.hist[key >> shift & 255u], 1u);
    });
    __syncthreads();
    if (threadIdx.x < kWave) {
      // lane l holds digits 255 - 4l .. 252 - 4l: descending order
      const int l = threadIdx.x;
      uint32_t n[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += n[i] = s.hist[255 - 4 * l - i];
      const uint32_t incl = wave_incl_scan_u(sum);
      uint32_t before = incl - sum;
      if (l == kWave - 1) s.total = incl;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (c.need > before && c.need <= before + n[i]) {
          s.digit = 255u - 4u * static_cast<uint32_t>(l) - static_cast<uint32_t>(i);
          s.need = c.need - before;
          s.bin = n[i];
        }
        before += n[i];
      }
    }
    __syncthreads();
    if (pass == 0 && s.total <= k) {  // all of them
      __syncthreads();
      return c;
    }
    c.value |= static_cast<uint64_t>(s.digit) << shift;
    c.mask |= 255ull << shift;
    c.need = s.need;
    c.more = s.bin != s.need;
    __syncthreads();
    if (!c.more) return c;
  }
  return c;
}

// The tokens of a row, for find_cut: every element's key.
template <typename Tin, int BLOCK, typename Fn>
__device__ __forceinline__ void row_keys(const Tin* row, int32_t V, Fn&& fn) {
  constexpr int VEC = Elem<Tin>::kVec;
  const int32_t h = static_cast<int32_t>(head_elems<Tin>(row, V)), nvec = (V - h) / VEC, tail = h + nvec * VEC;
  const int t = threadIdx.x;
  if (t < h) fn(place_key(Elem<Tin>::load1(row, t), t));
  if (t < V - tail) fn(place_key(Elem<Tin>::load1(row, tail + t), tail + t));
  for (int32_t j = t; j < nvec; j += BLOCK) {
    float z[VEC];
    Elem<Tin>::unpack(reinterpret_cast<const vec4u*>(row + h)[j], z);
#pragma unroll
    for (int u = 0; u < VEC; ++u) fn(place_key(z[u], h + j * VEC + u));
  }
}

// The first k tokens of a row in no order, by one workgroup; returns how many there are.
struct RowLds {
  CutLds cut;
  uint32_t n;
  uint64_t key[kMaxTop];
};

template <typename Tin, int BLOCK>
__device__ int list_row(const Tin* row, int32_t V, int k, RowLds& s) {
  // Of a bfloat16's key the low 16 bits follow from its sign.
  constexpr uint32_t SKIP = sizeof(Tin) == 2 ? 0x0cu : 0u;
  if (threadIdx.x == 0) s.n = 0;
  const Cut cut = find_cut<BLOCK, SKIP>([&](auto fn) { row_keys<Tin, BLOCK>(row, V, fn); }, static_cast<uint32_t>(k),
                                        s.cut);
  row_keys<Tin, BLOCK>(row, V, [&](uint64_t key) {
    if (!cut.takes(key)) return;
    const uint32_t at = atomicAdd(&s.n, 1u);
    if (at < static_cast<uint32_t>(kMaxTop)) s.key[at] = key;
  });
  __syncthreads();
  return static_cast<int>(min(s.n, static_cast<uint32_t>(k)));
}

// What log-probs of a row come from: log p of a logit is (z - m) / T - lnS.
struct RowNorm {
  double lnS;
  float m, T;
  uint32_t flags;
  __device__ __forceinline__ double logprob(float z) const {
    return (static_cast<double>(z) - static_cast<double>(m)) / static_cast<double>(T) - lnS;
  }
};

__device__ __forceinline__ RowNorm row_norm(const RowSum& p, float T) {
  RowNorm x;
  x.m = p.m;
  x.T = T;
  x.flags = 0;
  if (!temperature_ok(T)) x.flags |= PR_FLAG_BAD_TP;
  if (!(fabsf(p.S) < INFINITY) || p.m == INFINITY || p.m == -INFINITY) x.flags |= PR_FLAG_NONFINITE;
  if (!x.flags && fabsf(p.m) > ldexpf(T, 100)) x.flags |= PR_FLAG_BAD_TP;
  const float c = scale_of(T), A = p.m * c;
  x.lnS = log(static_cast<double>(p.S)) - static_cast<double>(fmaf(p.m, c, -A)) * 0.69314718055994530942;
  return x;
}

// Writes a row's first tokens in order from the n listed ones.
__device__ __forceinline__ void write_top(const TopArgs& a, int64_t r, const RowNorm& x, const uint64_t* key, int n) {
  const int t = threadIdx.x;
  const bool bad = x.flags != 0;
  if (t == 0) {
    if (a.lse) a.lse[r] = bad ? __uint_as_float(0x7fc00000u)
                              : static_cast<float>(static_cast<double>(x.m) / static_cast<double>(x.T) + x.lnS);
    if (a.flags) a.flags[r] = x.flags;
  }
  if (t >= a.k) return;
  int at = t;
  int32_t id = -1;
  float lp = bad ? __uint_as_float(0x7fc00000u) : -INFINITY;
  if (!bad && t < n) {
    const uint64_t mine = key[t];
    at = 0;
    for (int i = 0; i < n; ++i) at += key[i] > mine ? 1 : 0;
    id = key_index(mine);
    lp = static_cast<float>(x.logprob(key_logit(mine)));
  }
  a.ids[r * a.k + at] = id;
  a.logprob[r * a.k + at] = lp;
}

template <typename Tin>
__global__ __launch_bounds__(kRowBlock) void top_kernel(TopArgs a, int64_t first) {
  __shared__ RowLds s;
  const int64_t r = first + blockIdx.x;
  const Tin* row = static_cast<const Tin*>(a.logits) + r * a.row_stride;
  const float T = a.temperature[r];
  const RowSum sum = stretch_sum<Tin, kRowBlock>(row, a.V, 0, 1, scale_of(T));
  const RowNorm x = row_norm(sum, T);
  const int n = x.flags ? 0 : list_row<Tin, kRowBlock>(row, a.V, a.k, s);
  write_top(a, r, x, s.key, n);
}

// ---------------------------------------------------------------------------
// Beams

// Whether a beam's row is read, and the flags of one that is not.
__device__ __forceinline__ bool beam_live(const BeamArgs& a, int64_t r, uint32_t* flags) {
  const float s = a.scores[r];
  *flags = 0;
  if (!(s < INFINITY)) *flags = PR_FLAG_NONFINITE;
  else if (s == -INFINITY || (a.done && a.done[r])) *flags = PR_FLAG_MASKED;
  return *flags == 0;
}

// The first k tokens of each live beam's row, and its sum of exps.
template <typename Tin>
__global__ __launch_bounds__(kRowBlock) void beam_rows_kernel(BeamArgs a, RowSum* sums, uint64_t* list) {
  __shared__ RowLds s;
  const int64_t r = blockIdx.x;
  uint32_t flags;
  if (!beam_live(a, r, &flags)) return;
  const Tin* row = static_cast<const Tin*>(a.logits) + r * a.row_stride;
  const float T = a.temperature[r];
  const RowSum sum = stretch_sum<Tin, kRowBlock>(row, a.V, 0, 1, scale_of(T));
  const int n = row_norm(sum, T).flags ? 0 : list_row<Tin, kRowBlock>(row, a.V, a.k, s);
  const int t = threadIdx.x;
  if (t == 0) sums[r] = sum;
  if (t < a.k) list[r * a.k + t] = t < n ? s.key[t] : 0;
}

// A candidate of a request in the order of the selection: score, lower beam,
// the beam's own order.
struct Candidate {
  uint64_t score, token;
  int32_t beam;
  __device__ __forceinline__ bool before(const Candidate& o) const {
    if (score != o.score) return score > o.score;
    if (beam != o.beam) return beam < o.beam;
    return token > o.token;
  }
};

// The k best candidates of a request, by one workgroup.
__global__ __launch_bounds__(kBeamBlock) void beam_merge_kernel(BeamArgs a, const RowSum* sums, const uint64_t* list) {
  __shared__ RowNorm norm[PR_MAX_BEAMS];
  __shared__ double base[PR_MAX_BEAMS];
  __shared__ int state[PR_MAX_BEAMS];  // 0: no candidates, 1: its tokens, 2: itself
  __shared__ CutLds cut_lds;
  __shared__ Candidate best[kMaxTop];
  __shared__ uint32_t n_best;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * a.B;
  const int t = threadIdx.x;
  if (t < a.B) {
    uint32_t flags;
    const bool live = beam_live(a, first + t, &flags);
    RowNorm x{0.0, 0.0f, 1.0f, 0};
    if (live) {
      x = row_norm(sums[first + t], a.temperature[first + t]);
      flags = x.flags;
    }
    norm[t] = x;
    base[t] = static_cast<double>(a.scores[first + t]);
    state[t] = live ? (flags ? 0 : 1) : (flags == PR_FLAG_MASKED && a.scores[first + t] > -INFINITY ? 2 : 0);
    if (a.out.flags) a.out.flags[first + t] = flags;
  }
  if (t == 0) n_best = 0;
  __syncthreads();
  const uint64_t* mine = list + first * a.k;
  // Each candidate of thread t: its score's key, beam and token.
  auto candidates = [&](auto fn) {
    for (int e = t; e < a.B * a.k; e += kBeamBlock) {
      const int b = e / a.k;
      if (state[b] == 1) {
        const uint64_t key = mine[e];
        if (key != 0) fn(score_key(base[b] + norm[b].logprob(key_logit(key))), b, key);
      } else if (state[b] == 2 && e % a.k == 0) {
        fn(score_key(base[b]), b, uint64_t{1});
      }
    }
  };
  const Cut by_score = find_cut<kBeamBlock, 0>([&](auto fn) {
    candidates([&](uint64_t s, int, uint64_t) { fn(s); });
  }, static_cast<uint32_t>(a.k), cut_lds);
  Cut by_beam{0, 0, 0, false}, by_token{0, 0, 0, false};
  if (by_score.more) {  // equal scores: by beam, then by token
    by_beam = find_cut<kBeamBlock, 0x7fu>([&](auto fn) {
      candidates([&](uint64_t s, int b, uint64_t) { fn(s == by_score.value ? static_cast<uint64_t>(255 - b) : 0); });
    }, by_score.need, cut_lds);
    if (by_beam.more)
      by_token = find_cut<kBeamBlock, 0>([&](auto fn) {
        candidates([&](uint64_t s, int b, uint64_t key) {
          fn(s == by_score.value && static_cast<uint64_t>(255 - b) == by_beam.value ? key : 0);
        });
      }, by_beam.need, cut_lds);
  }
  candidates([&](uint64_t s, int b, uint64_t key) {
    bool take = by_score.takes(s);
    if (take && by_score.more && s == by_score.value) {
      const uint64_t kb = static_cast<uint64_t>(255 - b);
      take = by_beam.takes(kb) && (!by_beam.more || by_beam.above(kb) || by_token.takes(key));
    }
    if (!take) return;
    const uint32_t at = atomicAdd(&n_best, 1u);
    if (at < static_cast<uint32_t>(kMaxTop)) best[at] = Candidate{s, key, b};
  });
  __syncthreads();
  const int n = static_cast<int>(min(n_best, static_cast<uint32_t>(a.k)));
  if (t >= a.k) return;
  int at = t;
  float score = -INFINITY, lp = -INFINITY;
  int32_t parent = -1, token = -1;
  if (t < n) {
    const Candidate c = best[t];
    at = 0;
    for (int i = 0; i < n; ++i) at += best[i].before(c) ? 1 : 0;
    parent = c.beam;
    const bool itself = state[c.beam] == 2;
    const double l = itself ? 0.0 : norm[c.beam].logprob(key_logit(c.token));
    token = itself ? a.done_token : key_index(c.token);
    lp = static_cast<float>(l);
    score = static_cast<float>(base[c.beam] + l);
  }
  const int64_t o = static_cast<int64_t>(blockIdx.x) * a.k + at;
  a.out.scores[o] = score;
  a.out.parent[o] = parent;
  a.out.token[o] = token;
  if (a.out.logprob) a.out.logprob[o] = lp;
}

constexpr int64_t kMostGroups = int64_t{1} << 23;  // a grid holds less than 2^32 threads

template <typename Tin>
hipError_t top(const TopArgs& a, hipStream_t stream) {
  for (int64_t at = 0; at < a.n_rows; at += kMostGroups) {
    const int64_t rows = a.n_rows - at < kMostGroups ? a.n_rows - at : kMostGroups;
    hipLaunchKernelGGL(top_kernel<Tin>, dim3(static_cast<unsigned>(rows)), dim3(kRowBlock), 0, stream, a, at);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename Tin>
hipError_t beam(const BeamArgs& a, hipStream_t stream) {
  const int64_t n = static_cast<int64_t>(a.n_req) * a.B;
  uint64_t* list = static_cast<uint64_t*>(a.ws);
  RowSum* sums = reinterpret_cast<RowSum*>(list + n * a.k);
  hipLaunchKernelGGL(beam_rows_kernel<Tin>, dim3(static_cast<unsigned>(n)), dim3(kRowBlock), 0, stream, a, sums, list);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(beam_merge_kernel, dim3(static_cast<unsigned>(a.n_req)), dim3(kBeamBlock), 0, stream, a, sums,
                     list);
  return hipGetLastError();
}

}  // namespace

size_t top_workspace_bytes(int64_t, int32_t, pr_dtype, int32_t) { return 0; }

hipError_t launch_top(const TopArgs& a, pr_dtype dtype, hipStream_t stream) {
  return dtype == PR_BF16 ? top<uint16_t>(a, stream) : top<float>(a, stream);
}

size_t beam_workspace_bytes(int64_t n_rows, int32_t, pr_dtype, int32_t k) {
  const size_t n = n_rows < 0 ? 0 : static_cast<size_t>(n_rows);
  return n * (static_cast<size_t>(k) * sizeof(uint64_t) + sizeof(RowSum));
}

hipError_t launch_beam(const BeamArgs& a, pr_dtype dtype, hipStream_t stream) {
  return dtype == PR_BF16 ? beam<uint16_t>(a, stream) : beam<float>(a, stream);
}

}  // namespace pr
