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

// A stretch of a row: its vectors [vb, ve), counted from element 0 wherever the
// row lies (unaligned 16-byte loads), so that equal rows have equal sums; the
// row's last stretch also has the elements after the vectors.
template <typename Tin>
struct Stretch {
  static constexpr int VEC = Elem<Tin>::kVec;
  typedef typename GradVec<Tin>::Store Vec;  // 16 bytes of an element's alignment
  const Tin* row;
  int32_t vb, ve, tail, n_tail;

  __device__ __forceinline__ Stretch(const Tin* r, int32_t V, int g, int G) : row(r) {
    const int64_t nvec = V / VEC;
    vb = static_cast<int32_t>(nvec * g / G);
    ve = static_cast<int32_t>(nvec * (g + 1) / G);
    tail = static_cast<int32_t>(nvec * VEC);
    n_tail = g == G - 1 ? V - tail : 0;
  }
  __device__ __forceinline__ const Vec* vectors() const { return reinterpret_cast<const Vec*>(row); }
  __device__ __forceinline__ float tail_logit(int t) const { return t < n_tail ? Elem<Tin>::load1(row, tail + t) : -INFINITY; }
  // fn(key) for each of the thread's elements.
  template <int BLOCK, typename Fn>
  __device__ __forceinline__ void keys(Fn&& fn) const {
    fn(place_key(tail_logit(threadIdx.x), tail + threadIdx.x));
    for (int32_t j = vb + static_cast<int32_t>(threadIdx.x); j < ve; j += BLOCK) {
      float z[VEC];
      Elem<Tin>::unpack(static_cast<vec4u>(vectors()[j]), z);
#pragma unroll
      for (int u = 0; u < VEC; ++u) fn(place_key(z[u], static_cast<int64_t>(j) * VEC + u));
    }
  }
};

constexpr int kCap = 2048;  // keys listed of a stretch

template <int BLOCK>
struct ListLds {
  uint64_t key[kCap];
  alignas(16) uint32_t hist[256];
  CutLds cut;
  float low[BLOCK / kWave], top[BLOCK / kWave];
  float floor;  // at least k logits of the stretch are not below it
  uint32_t n;
};

// The largest value, to 16 bits of its key, that at least j of the wave's
// lanes' v are not below (-inf: there is none). j <= 64.
__device__ __forceinline__ float wave_floor(float v, int j) {
  const uint32_t key = float_key(v);
  uint32_t at = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t up = at | 1u << bit;
    if (__popcll(__ballot(key >= up)) >= j) at = up;
  }
  return at <= 0x007f0000u ? -INFINITY : key_float(at);
}

// Which of the 256 bins holds the k-th largest of what they count (0 where
// there are fewer). One wave calls it.
__device__ __forceinline__ int cut_bin(const uint32_t* hist, uint32_t k) {
  const int l = static_cast<int>(__lane_id());  // bins 255 - 4l .. 252 - 4l
  const vec4u n = *reinterpret_cast<const vec4u*>(hist + 252 - 4 * l);
  const uint32_t incl = wave_incl_scan_u(n.x + n.y + n.z + n.w), before = incl - (n.x + n.y + n.z + n.w);
  const uint64_t full = __ballot(incl >= k);
  if (full == 0) return 0;
  int bin = 252 - 4 * l;
  if (before + n.w >= k)
    bin += 3;
  else if (before + n.w + n.z >= k)
    bin += 2;
  else if (before + n.w + n.z + n.y >= k)
    bin += 1;
  return __builtin_amdgcn_readlane(bin, static_cast<int>(__builtin_ctzll(full)));
}

// The k largest logits of a stretch and others beside them, as keys in s.key;
// returns how many. One pass: the first vectors of all lanes give a floor that
// k logits reach; from there on what reaches the floor is listed and counted in
// 256 bins between it and the largest logit of the first vectors, and every
// `k` listed logits the wave that lists the last of them raises the floor to the
// bin that the k-th largest is in. The waves do not wait for each other: a floor
// read late lists more. Rows in which far too many logits reach the floor (many
// equal ones, or rising ones) are selected from by digits (find_cut).
template <typename Tin, int BLOCK>
__device__ int list_stretch(const Stretch<Tin>& x, int k, float c, ListLds<BLOCK>& s, RowSum* sum) {
  constexpr int VEC = Elem<Tin>::kVec, NW = BLOCK / kWave, LD = 4;
  const int t = threadIdx.x, wave = t / kWave;
  const bool lead = t % kWave == 0;
  vec4u v[LD];
  scan::vector_prefetch<Tin, BLOCK, LD>(x.vectors(), x.vb, x.ve, v);
  const float zt = x.tail_logit(t);
  for (int i = t; i < 256; i += BLOCK) s.hist[i] = 0;
  if (t == 0) s.n = 0;
  float first = zt;
#pragma unroll
  for (int u = 0; u < LD; ++u) {
    float z[VEC];
    Elem<Tin>::unpack(v[u], z);
#pragma unroll
    for (int i = 0; i < VEC; ++i) first = fmaxf(first, z[i]);
  }
  const float low = wave_floor(first, (k + NW - 1) / NW), high = wave_max(first);
  if (lead) {
    s.low[wave] = low;
    s.top[wave] = high;
  }
  __syncthreads();
  float floor0 = s.low[0], top0 = s.top[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) {
    floor0 = fminf(floor0, s.low[w]);
    top0 = fmaxf(top0, s.top[w]);
  }
  floor0 = fmaxf(floor0, kNegSentinel);  // any finite logit
  const float width = (top0 - floor0) * (1.0f / 255.0f), scale = width > 0.0f && width < INFINITY ? 1.0f / width : 0.0f;
  auto bin_of = [&](float z) { return min(255, static_cast<int>(fmaxf((z - floor0) * scale, 0.0f))); };
  if (t == 0) s.floor = floor0;
  __syncthreads();

  const uint32_t every = static_cast<uint32_t>(k < 64 ? 64 : k);
  LaneSum<true> L;
  auto list = [&](float z, int64_t i, bool& raise) {
    const uint32_t at = atomicAdd(&s.n, 1u);
    if (at < static_cast<uint32_t>(kCap)) {
      s.key[at] = place_key(z, i);
      atomicAdd(&s.hist[bin_of(z)], 1u);
      raise |= at % every == every - 1;
    } else {
      raise = true;
    }
  };
  auto raise_floor = [&](bool raise) {
    if (!__any(raise)) return;
    const int b = cut_bin(s.hist, static_cast<uint32_t>(k));
    const bool full = s.n > static_cast<uint32_t>(kCap);  // list no more
    // A sixteenth of a bin below its edge: the bins' own roundings are less.
    const float f = full ? INFINITY : floor0 + (static_cast<float>(b) - 0.0625f) * width;
    if ((b > 0 || full) && lead) __hip_atomic_store(&s.floor, f, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  };
  scan::stream_stretch<Tin, BLOCK, 2, LD>(x.vectors(), x.vb, x.ve, v, [&](const vec4u* vv, int64_t j) {
    const float floor = __hip_atomic_load(&s.floor, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    float z[2 * VEC];
    Elem<Tin>::unpack(vv[0], z);
    Elem<Tin>::unpack(vv[1], z + VEC);
    const float top = L.add(z, c);
    if (!__any(top >= floor)) return;
    bool raise = false;
    if (top >= floor) {
#pragma unroll
      for (int i = 0; i < 2 * VEC; ++i)
        if (z[i] >= floor) list(z[i], (j + (i / VEC) * BLOCK) * VEC + i % VEC, raise);
    }
    raise_floor(raise);
  });
  L.add1(zt, c);
  bool unused = false;
  if (zt >= floor0) list(zt, x.tail + t, unused);
  *sum = merge_block<BLOCK>(L, c);  // its barrier ends the listing
  const uint32_t n = s.n;
  if (n > static_cast<uint32_t>(kCap)) {
    // Of a bfloat16's key the low 16 bits follow from its sign.
    constexpr uint32_t SKIP = sizeof(Tin) == 2 ? 0x0cu : 0u;
    const Cut cut = find_cut<BLOCK, SKIP>([&](auto fn) { x.template keys<BLOCK>(fn); }, static_cast<uint32_t>(k), s.cut);
    __syncthreads();
    if (t == 0) s.n = 0;
    __syncthreads();
    x.template keys<BLOCK>([&](uint64_t key) {
      if (!cut.takes(key)) return;
      const uint32_t at = atomicAdd(&s.n, 1u);
      if (at < static_cast<uint32_t>(kCap)) s.key[at] = key;
    });
    __syncthreads();
    return static_cast<int>(min(s.n, static_cast<uint32_t>(k)));
  }
  if (n <= static_cast<uint32_t>(k) + 16) return static_cast<int>(n);
  // Those from the k-th's bin on.
  const int b = cut_bin(s.hist, static_cast<uint32_t>(k));
  constexpr int PER = kCap / BLOCK;
  uint64_t mine[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint32_t e = static_cast<uint32_t>(t + i * BLOCK);
    mine[i] = e < n ? s.key[e] : 0;
  }
  __syncthreads();
  if (t == 0) s.n = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (mine[i] != 0 && bin_of(key_logit(mine[i])) >= b) s.key[atomicAdd(&s.n, 1u)] = mine[i];
  __syncthreads();
  return static_cast<int>(s.n);
}

// The places of the n listed keys among themselves: fn(place, key) for each,
// from 0, the largest's.
template <int BLOCK, typename Fn>
__device__ __forceinline__ void in_order(const uint64_t* key, int n, Fn&& fn) {
  for (int e = threadIdx.x; e < n; e += BLOCK) {
    const uint64_t mine = key[e];
    int place = 0;
#pragma unroll 4
    for (int i = 0; i < n; ++i) place += key[i] > mine ? 1 : 0;
    fn(place, mine);
  }
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

// Writes a row's first k tokens in order from the n listed ones.
template <int BLOCK>
__device__ __forceinline__ void write_top(const TopArgs& a, int64_t r, const RowNorm& x, const uint64_t* key, int n) {
  const int t = threadIdx.x;
  const bool bad = x.flags != 0;
  const float nan = __uint_as_float(0x7fc00000u);
  if (t == 0) {
    if (a.lse) a.lse[r] = bad ? nan : static_cast<float>(static_cast<double>(x.m) / static_cast<double>(x.T) + x.lnS);
    if (a.flags) a.flags[r] = x.flags;
  }
  if (bad) n = 0;
  in_order<BLOCK>(key, n, [&](int place, uint64_t mine) {
    if (place >= a.k) return;
    a.ids[r * a.k + place] = key_index(mine);
    a.logprob[r * a.k + place] = static_cast<float>(x.logprob(key_logit(mine)));
  });
  if (t >= n && t < a.k) {
    a.ids[r * a.k + t] = -1;
    a.logprob[r * a.k + t] = bad ? nan : -INFINITY;
  }
}

template <typename Tin, int BLOCK>
__global__ __launch_bounds__(BLOCK) void top_kernel(TopArgs a, int64_t first) {
  __shared__ ListLds<BLOCK> s;
  const int64_t r = first + blockIdx.x;
  const float T = a.temperature[r];
  const Stretch<Tin> x(static_cast<const Tin*>(a.logits) + r * a.row_stride, a.V, 0, 1);
  RowSum sum;
  const int n = list_stretch<Tin, BLOCK>(x, a.k, scale_of(T), s, &sum);
  write_top<BLOCK>(a, r, row_norm(sum, T), s.key, n);
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
  __shared__ ListLds<kRowBlock> s;
  const int64_t r = blockIdx.x;
  uint32_t flags;
  if (!beam_live(a, r, &flags)) return;
  const float T = a.temperature[r];
  const Stretch<Tin> x(static_cast<const Tin*>(a.logits) + r * a.row_stride, a.V, 0, 1);
  RowSum sum;
  int n = list_stretch<Tin, kRowBlock>(x, a.k, scale_of(T), s, &sum);
  if (row_norm(sum, T).flags) n = 0;
  const int t = threadIdx.x;
  if (t == 0) sums[r] = sum;
  in_order<kRowBlock>(s.key, n, [&](int place, uint64_t key) {
    if (place < a.k) list[r * a.k + place] = key;
  });
  if (t >= n && t < a.k) list[r * a.k + t] = 0;
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
    hipLaunchKernelGGL((top_kernel<Tin, kRowBlock>), dim3(static_cast<unsigned>(rows)), dim3(kRowBlock), 0, stream, a, at);
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
