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

// The same to float32: keys in one order have theirs in the same or equal. 0 stays 0.
__device__ __forceinline__ uint32_t near_key(uint64_t k) {
  if (k == 0) return 0;
  const uint64_t b = k >> 63 ? k & 0x7fffffffffffffffull : ~k;
  return float_key(static_cast<float>(__longlong_as_double(static_cast<long long>(b))));
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
// by digits of 8 bits from the top until a digit's keys are all taken. skip:
// digits, counted from the top by bits, that are the same for all keys whose
// earlier digits are. Every thread calls it; a barrier follows its last read.
template <int BLOCK, typename Keys>
__device__ Cut find_cut(Keys&& keys, uint32_t k, CutLds& s, uint32_t skip = 0) {
  Cut c{0, 0, k, false};
  for (int pass = 0; pass < 8; ++pass) {
    if (skip >> pass & 1u) continue;
    const int shift = 56 - 8 * pass;
    for (int b = threadIdx.x; b < 256; b += BLOCK) s.hist[b] = 0;
    __syncthreads();
    keys([&](uint64_t key) {
      if (key == 0 || (key & c.mask) != c.value) return;
      // Equal logits have equal digits: lanes that agree add once.
      const uint32_t digit = static_cast<uint32_t>(key >> shift) & 255u;
      const uint32_t one = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(digit)));
      const uint64_t here = __ballot(true);
      if (__ballot(digit == one) != here)
        atomicAdd(&s.hist[digit], 1u);
      else if (static_cast<int>(__lane_id()) == __builtin_ctzll(here))
        atomicAdd(&s.hist[one], static_cast<uint32_t>(__popcll(here)));
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

// The loads of a stretch and the loop over its vectors: those of scan::
// stretch_prefetch and scan::stream_stretch (row_scan.h), for vectors of an
// element's alignment. v holds the lane's first LD vectors; body(vv, j) reduces
// the U vectors vv[0..U) of indices j + u BLOCK; lanes past the end see -inf.
template <typename Tin>
__device__ __forceinline__ vec4u load_vector(const typename Stretch<Tin>::Vec* p) {
  return static_cast<vec4u>(__builtin_nontemporal_load(p));
}

template <typename Tin, int BLOCK, int LD>
__device__ __forceinline__ void prefetch(const Stretch<Tin>& x, vec4u (&v)[LD]) {
  const auto* vp = x.vectors();
  const int32_t i = x.vb + static_cast<int32_t>(threadIdx.x);
  if (x.vb + scan::wave_first_thread() + (kWave - 1) + (LD - 1) * BLOCK < x.ve) {
#pragma unroll
    for (int u = 0; u < LD; ++u) v[u] = load_vector<Tin>(vp + i + u * BLOCK);
  } else {
#pragma unroll
    for (int u = 0; u < LD; ++u) {
      const int32_t j = i + u * BLOCK;
      v[u] = j < x.ve ? load_vector<Tin>(vp + j) : neg_inf_vec<Tin>();
    }
  }
}

template <typename Tin, int BLOCK, int U, int LD, typename Body>
__device__ __forceinline__ void stream(const Stretch<Tin>& x, vec4u (&v)[LD], Body&& body) {
  const auto* vp = x.vectors();
  const int64_t ve = x.ve;
  int64_t i = x.vb + static_cast<int32_t>(threadIdx.x);
  int64_t i0 = x.vb + scan::wave_first_thread();
  if (i0 + (kWave - 1) + (LD - 1) * BLOCK < ve) {
    // Two buffers: the loads of one are issued before the other is reduced.
    for (; i0 + (kWave - 1) + (3 * LD - 1) * BLOCK < ve; i += 2 * LD * BLOCK, i0 += 2 * LD * BLOCK) {
      vec4u w[LD];
#pragma unroll
      for (int u = 0; u < LD; ++u) w[u] = load_vector<Tin>(vp + i + (LD + u) * BLOCK);
#pragma unroll
      for (int c = 0; c < LD; c += U) body(v + c, i + c * BLOCK);
#pragma unroll
      for (int u = 0; u < LD; ++u) v[u] = load_vector<Tin>(vp + i + (2 * LD + u) * BLOCK);
#pragma unroll
      for (int c = 0; c < LD; c += U) body(w + c, i + (LD + c) * BLOCK);
    }
    for (; i0 < ve; i += LD * BLOCK, i0 += LD * BLOCK) {
      vec4u w[LD];
#pragma unroll
      for (int u = 0; u < LD; ++u) {
        const int64_t j = i + (LD + u) * BLOCK;
        w[u] = j < ve ? load_vector<Tin>(vp + j) : neg_inf_vec<Tin>();
      }
#pragma unroll
      for (int c = 0; c < LD; c += U) body(v + c, i + c * BLOCK);
#pragma unroll
      for (int u = 0; u < LD; ++u) v[u] = w[u];
    }
  } else if (i0 < ve) {
#pragma unroll
    for (int c = 0; c < LD; c += U) body(v + c, i + c * BLOCK);
  }
}

// What a stretch lists: vectors, later keys in their place. KMAX: the largest k
// that the lists are made for (a row of ordinary logits lists about
// k (1 + log(the row / the first vectors)) vectors).
template <int KMAX>
constexpr int list_cap() {
  return KMAX <= 64 ? 768 : 2048;
}

template <int BLOCK, int KMAX>
struct ListLds {
  static constexpr int CAP = list_cap<KMAX>();  // vectors
  static constexpr int KEYS = 2 * CAP;          // keys in the vectors' place
  union {
    struct {
      vec4u vec[CAP];
      int32_t at[CAP];
    };
    alignas(16) uint64_t key[KEYS + 4];
  };
  alignas(16) uint32_t hist[256];
  CutLds cut;
  float low[BLOCK / kWave], top[BLOCK / kWave], bottom[BLOCK / kWave];
  float floor;  // at least k logits of the stretch are not below it
  uint32_t n;
};

// The largest value, to 16 bits of its key, that at least j of the N values of
// each of the wave's lanes are not below (-inf: there is none). j <= 64 N.
template <int N>
__device__ __forceinline__ float wave_floor(const float (&v)[N], int j) {
  uint32_t key[N];
#pragma unroll
  for (int u = 0; u < N; ++u) key[u] = float_key(v[u]);
  uint32_t at = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t up = at | 1u << bit;
    int n = 0;
#pragma unroll
    for (int u = 0; u < N; ++u) n += __popcll(__ballot(key[u] >= up));
    if (n >= j) at = up;
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

// The places of the n listed keys among themselves: fn(place, key) for each,
// from 0, the largest's. The list is 16-byte aligned and closed by four zeros
// (close_list, after which the threads have met).
__device__ __forceinline__ int close_list(uint64_t* key, int n) {
  if (threadIdx.x < 4) key[n + threadIdx.x] = 0;
  __syncthreads();
  return n;
}
typedef uint64_t Keys2 __attribute__((ext_vector_type(2)));
template <int BLOCK, typename Fn>
__device__ __forceinline__ void in_order(const uint64_t* key, int n, Fn&& fn) {
  const Keys2* pair = reinterpret_cast<const Keys2*>(key);
  for (int e = threadIdx.x; e < n; e += BLOCK) {
    const uint64_t mine = key[e];
    int place = 0;
    for (int i = 0; i < n; i += 4) {
      const Keys2 p = pair[i / 2], q = pair[i / 2 + 1];
      place += (p.x > mine ? 1 : 0) + (p.y > mine ? 1 : 0) + (q.x > mine ? 1 : 0) + (q.y > mine ? 1 : 0);
    }
    fn(place, mine);
  }
}

// The same for longer lists, each key counted against those of its bin alone
// (larger keys are in the same bin or a larger one); `to` has room for the list.
// 280 keys took 5.8 us the other way.
template <int BLOCK, typename Bin, typename Fn>
__device__ __forceinline__ void in_order_by_bins(const uint64_t* key, uint64_t* to, int n, uint32_t* hist, Bin&& bin_of,
                                                 Fn&& fn) {
  constexpr int kFew = 128;
  if (n <= kFew) return in_order<BLOCK>(key, n, fn);
  __shared__ uint32_t start[256], end[256];
  for (int b = threadIdx.x; b < 256; b += BLOCK) hist[b] = 0;
  __syncthreads();
  for (int e = threadIdx.x; e < n; e += BLOCK) atomicAdd(&hist[bin_of(key[e])], 1u);
  __syncthreads();
  if (threadIdx.x < kWave) {
    const int b = 252 - 4 * static_cast<int>(threadIdx.x);  // bins b + 3 .. b: descending order
    const uint32_t n3 = hist[b + 3], n2 = hist[b + 2], n1 = hist[b + 1], n0 = hist[b];
    const uint32_t s3 = wave_incl_scan_u(n3 + n2 + n1 + n0) - (n3 + n2 + n1 + n0);
    start[b + 3] = end[b + 3] = s3;
    start[b + 2] = end[b + 2] = s3 + n3;
    start[b + 1] = end[b + 1] = s3 + n3 + n2;
    start[b] = end[b] = s3 + n3 + n2 + n1;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < n; e += BLOCK) to[atomicAdd(&end[bin_of(key[e])], 1u)] = key[e];
  __syncthreads();
  for (int e = threadIdx.x; e < n; e += BLOCK) {
    const uint64_t mine = to[e];
    const int b = bin_of(mine);
    int place = static_cast<int>(start[b]);
    for (uint32_t i = start[b]; i < end[b]; ++i) place += to[i] > mine ? 1 : 0;
    fn(place, mine);
  }
}

// 256 bins of logits from `low` on; larger logits are in the same bin or a larger one.
struct Bins {
  float low, scale;
  __device__ __forceinline__ int of(float z) const {
    return static_cast<int>(fminf(fmaxf((z - low) * scale, 0.0f), 255.0f));
  }
  __device__ __forceinline__ int operator()(uint64_t key) const { return of(key_logit(key)); }
};

// The k largest logits of a stretch and a few beside them, as keys in s.key;
// returns how many. One pass: the first vectors of all lanes give a floor that
// k logits reach; from there on every vector with a logit that reaches the floor
// is listed, and its largest logit counted in 256 bins from the floor on; the
// wave that lists a k-th one raises the floor to the bin that the k-th largest
// counted is in. The waves do not wait for each other: a floor read late lists
// more. Where more vectors reach the floor than are held, the stretch is read
// again with the floor that those give; where that does not help (many equal
// logits, or ever larger ones), it is selected from by digits. 512 rows of
// 151,936 bfloat16 logits, 8 of each, take 30 us, 59 where the first 16,384 are
// masked, 303 where they rise, 446 where all are equal. A lane has four vectors in
// flight until the floor is made, 16 rounds of ballots and two barriers; its next
// loads are issued behind them. bins: the last bins.
template <typename Tin, int BLOCK, int KMAX>
__device__ int list_stretch(const Stretch<Tin>& x, int k, float c, ListLds<BLOCK, KMAX>& s, RowSum* sum, Bins* bins) {
  constexpr int VEC = Elem<Tin>::kVec, NW = BLOCK / kWave, LD = 4, CAP = ListLds<BLOCK, KMAX>::CAP;
  const int t = threadIdx.x, wave = t / kWave;
  const bool lead = t % kWave == 0;
  vec4u v[LD];
  prefetch<Tin, BLOCK>(x, v);
  const float zt = x.tail_logit(t);
  for (int i = t; i < 256; i += BLOCK) s.hist[i] = 0;
  if (t == 0) s.n = 0;
  auto largest = [](const float (&z)[VEC]) {
    float m = z[0];
#pragma unroll
    for (int i = 1; i < VEC; ++i) m = fmaxf(m, z[i]);
    return m;
  };
  float first[LD];  // each vector's largest
#pragma unroll
  for (int u = 0; u < LD; ++u) {
    float z[VEC];
    Elem<Tin>::unpack(v[u], z);
    first[u] = fmaxf(largest(z), u == 0 ? zt : -INFINITY);
  }
  float floor0, bin0, width;
  // The floor, and the bins above it, that the largest logits of some vectors give.
  auto set_floor = [&](const auto& best) {
    constexpr int N = sizeof(best) / sizeof(float);
    const float low = wave_floor(best, (k + NW - 1) / NW);
    float high = -INFINITY, least = INFINITY;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      high = fmaxf(high, best[u]);
      least = fminf(least, best[u] > -INFINITY ? best[u] : INFINITY);
    }
    high = wave_max(high);
    least = -wave_max(-least);
    if (lead) {
      s.low[wave] = low;
      s.top[wave] = high;
      s.bottom[wave] = least;
    }
    __syncthreads();
    floor0 = s.low[0];
    bin0 = s.bottom[0];
    float top0 = s.top[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) {
      floor0 = fminf(floor0, s.low[w]);
      top0 = fmaxf(top0, s.top[w]);
      bin0 = fminf(bin0, s.bottom[w]);
    }
    // Where many vectors are masked whole any finite logit is listed, and the bins
    // start at the least vector's largest.
    bin0 = floor0 > -INFINITY ? floor0 : bin0;
    floor0 = fmaxf(floor0, kNegSentinel);
    // Half as far again above the first vectors' largest: where the k-th of a long
    // row is above that one, the floor would not come near it.
    width = (top0 - bin0) * (1.5f / 255.0f);
    *bins = Bins{bin0, width > 0x1p-120f && width < INFINITY ? 1.0f / width : 0.0f};
    if (t == 0) s.floor = floor0;
    __syncthreads();
  };
  set_floor(first);
  auto bin_of = [&](float z) { return bins->of(z); };

  const uint32_t every = static_cast<uint32_t>(k < 64 ? 64 : k);
  auto list = [&](const vec4u& p, int32_t at, float top, bool& raise) {
    const uint32_t n = atomicAdd(&s.n, 1u);
    raise |= n >= static_cast<uint32_t>(CAP) || n % every == every - 1;
    if (n < static_cast<uint32_t>(CAP)) {
      s.vec[n] = p;
      s.at[n] = at;
      atomicAdd(&s.hist[bin_of(top)], 1u);
    }
  };
  auto edge = [&](int b) {  // a sixteenth of a bin below it: the bins' own roundings are less
    return bin0 + (static_cast<float>(b) - 0.0625f) * width;
  };
  auto raise_floor = [&](bool raise) {
    if (!__any(raise)) return;
    const int b = cut_bin(s.hist, static_cast<uint32_t>(k));
    const bool full = s.n > static_cast<uint32_t>(CAP);  // list no more
    if ((b > 0 || full) && lead)
      __hip_atomic_store(&s.floor, full ? INFINITY : edge(b), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  };
  LaneSum<true> L;
  stream<Tin, BLOCK, 2>(x, v, [&](const vec4u* vv, int64_t j) {
    const float floor = __hip_atomic_load(&s.floor, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    float z[2 * VEC], top[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float y[VEC];
      Elem<Tin>::unpack(vv[u], y);
      top[u] = largest(y);
#pragma unroll
      for (int i = 0; i < VEC; ++i) z[u * VEC + i] = y[i];
    }
    const float both = fmaxf(top[0], top[1]);
    L.add_top(z, both, c);
    if (!__any(both >= floor)) return;
    bool raise = false;
#pragma unroll
    for (int u = 0; u < 2; ++u)
      if (top[u] >= floor) list(vv[u], (static_cast<int32_t>(j) + u * BLOCK) * VEC, top[u], raise);
    raise_floor(raise);
  });
  L.add1(zt, c);
  *sum = merge_block<BLOCK>(L, c);  // its barrier ends the listing
  uint32_t n = s.n;
  auto digits = [&](auto keys) {  // exactly the k largest of the keys that keys(fn) passes
    // Of a bfloat16's key the low 16 bits follow from its sign; of an index the
    // high bits are those of the row's length.
    const uint32_t skip = (sizeof(Tin) == 2 ? 0x0cu : 0u) | (x.tail < (1 << 24) - VEC ? 0x10u : 0u);
    const Cut cut = find_cut<BLOCK>(keys, static_cast<uint32_t>(k), s.cut, skip);
    if (t == 0) s.n = 0;
    __syncthreads();
    keys([&](uint64_t key) {
      if (cut.takes(key)) s.key[atomicAdd(&s.n, 1u)] = key;
    });
    __syncthreads();
    return close_list(s.key, static_cast<int>(s.n));
  };
  auto row_keys = [&](auto fn) { x.template keys<BLOCK>(fn); };
  constexpr int PER = (CAP + BLOCK - 1) / BLOCK;
  if (n > static_cast<uint32_t>(CAP)) {
    float best[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      float z[VEC];
      Elem<Tin>::unpack(t + i * BLOCK < CAP ? s.vec[t + i * BLOCK] : neg_inf_vec<Tin>(), z);
      best[i] = largest(z);
    }
    __syncthreads();
    for (int i = t; i < 256; i += BLOCK) s.hist[i] = 0;
    if (t == 0) s.n = 0;
    set_floor(best);
    for (int32_t j = x.vb + t; __any(j < x.ve); j += BLOCK) {
      const vec4u p = j < x.ve ? load_vector<Tin>(x.vectors() + j) : neg_inf_vec<Tin>();
      float z[VEC];
      Elem<Tin>::unpack(p, z);
      const float floor = __hip_atomic_load(&s.floor, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      const float top = largest(z);
      bool raise = false;
      if (top >= floor) list(p, j * VEC, top, raise);
      raise_floor(raise);
    }
    __syncthreads();
    n = s.n;
    if (n > static_cast<uint32_t>(CAP)) {
      __syncthreads();
      return digits(row_keys);
    }
  }
  // The listed vectors' logits from the k-th's bin on.
  const int b = cut_bin(s.hist, static_cast<uint32_t>(k));
  vec4u mine[PER];
  int32_t at[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint32_t e = static_cast<uint32_t>(t + i * BLOCK);
    mine[i] = e < n ? s.vec[e] : neg_inf_vec<Tin>();
    at[i] = e < n ? s.at[e] : 0;
  }
  __syncthreads();
  if (t == 0) s.n = 0;
  __syncthreads();
  auto keep = [&](float z, int32_t i) {
    if (!(z > -INFINITY) || bin_of(z) < b) return;
    const uint32_t m = atomicAdd(&s.n, 1u);
    if (m < static_cast<uint32_t>(ListLds<BLOCK, KMAX>::KEYS)) s.key[m] = place_key(z, i);
  };
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    float z[VEC];
    Elem<Tin>::unpack(mine[i], z);
    if (largest(z) > -INFINITY) {
#pragma unroll
      for (int u = 0; u < VEC; ++u) keep(z[u], at[i] + u);
    }
  }
  keep(zt, x.tail + t);
  __syncthreads();
  n = s.n;
  if (n > static_cast<uint32_t>(ListLds<BLOCK, KMAX>::KEYS)) {
    __syncthreads();
    return digits(row_keys);
  }
  if (n <= static_cast<uint32_t>(k + k / 2 + 64)) return close_list(s.key, static_cast<int>(n));
  constexpr int MOST = 2 * PER;
  uint64_t key[MOST];
#pragma unroll
  for (int i = 0; i < MOST; ++i) {
    const uint32_t e = static_cast<uint32_t>(t + i * BLOCK);
    key[i] = e < n ? s.key[e] : 0;
  }
  return digits([&](auto fn) {
#pragma unroll
    for (int i = 0; i < MOST; ++i) fn(key[i]);
  });
}

// The places of the keys that list_stretch has left.
template <int BLOCK, int KMAX, typename Fn>
__device__ __forceinline__ void list_order(ListLds<BLOCK, KMAX>& s, int n, const Bins& bins, Fn&& fn) {
  if constexpr (KMAX <= 64)
    in_order<BLOCK>(s.key, n, fn);
  else
    in_order_by_bins<BLOCK>(s.key, s.key + ListLds<BLOCK, KMAX>::KEYS / 2, n, s.hist, bins, fn);
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
  const RowRef ref = row_ref(p.m, scale_of(T));
  x.lnS = log(static_cast<double>(p.S)) - static_cast<double>(fmaf(p.m, ref.c, -ref.A)) * 0.69314718055994530942;
  return x;
}

// Writes a row's first k tokens in order from the n listed ones. order(n, fn)
// gives the list's places.
template <int BLOCK, typename Order>
__device__ __forceinline__ void write_top(const TopArgs& a, int64_t r, const RowNorm& x, int n, Order&& order) {
  const int t = threadIdx.x;
  const bool bad = x.flags != 0;
  const float nan = __uint_as_float(0x7fc00000u);
  if (t == 0) {
    if (a.lse) a.lse[r] = bad ? nan : static_cast<float>(static_cast<double>(x.m) / static_cast<double>(x.T) + x.lnS);
    if (a.flags) a.flags[r] = x.flags;
  }
  if (bad) n = 0;
  order(n, [&](int place, uint64_t mine) {
    if (place >= a.k) return;
    a.ids[r * a.k + place] = key_index(mine);
    a.logprob[r * a.k + place] = static_cast<float>(x.logprob(key_logit(mine)));
  });
  if (t >= n && t < a.k) {
    a.ids[r * a.k + t] = -1;
    a.logprob[r * a.k + t] = bad ? nan : -INFINITY;
  }
}

// One workgroup per row. The read bounds it: 16,972 rows of 151,936 bfloat16
// logits, 64 of each, 799 us (6.46 TB/s); 512 rows of 32,000 float32 logits, 20 of
// each, 16.6 us, of which a chain of barriers, which the loads wait for, about 5.
template <typename Tin, int BLOCK, int KMAX>
__global__ __launch_bounds__(BLOCK) void top_kernel(TopArgs a, int64_t first) {
  __shared__ ListLds<BLOCK, KMAX> s;
  const int64_t r = first + blockIdx.x;
  const float T = a.temperature[r];
  const Stretch<Tin> x(static_cast<const Tin*>(a.logits) + r * a.row_stride, a.V, 0, 1);
  RowSum sum;
  Bins bins;
  const int n = list_stretch<Tin, BLOCK, KMAX>(x, a.k, scale_of(T), s, &sum, &bins);
  write_top<BLOCK>(a, r, row_norm(sum, T), n, [&](int m, auto fn) { list_order<BLOCK, KMAX>(s, m, bins, fn); });
}

// The first k tokens of a part of a row in order, 0 after the last, and the part's sum.
template <typename Tin, int BLOCK, int KMAX>
__device__ __forceinline__ void write_part(const Stretch<Tin>& x, int k, float c, ListLds<BLOCK, KMAX>& s, uint64_t* list,
                                           RowSum* to) {
  RowSum sum;
  Bins bins;
  const int t = threadIdx.x, n = list_stretch<Tin, BLOCK, KMAX>(x, k, c, s, &sum, &bins);
  if (t == 0) *to = sum;
  list_order<BLOCK, KMAX>(s, n, bins, [&](int place, uint64_t mine) {
    if (place < k) list[place] = mine;
  });
  if (t >= n && t < k) list[t] = 0;
}

// Rows over G workgroups each: the parts' tokens and sums (32 rows of 262,144
// float32 logits, k = 64, with the merge 21 us),
template <typename Tin, int BLOCK, int KMAX>
__global__ __launch_bounds__(BLOCK) void top_parts_kernel(TopArgs a, uint64_t* list, RowSum* sums) {
  __shared__ ListLds<BLOCK, KMAX> s;
  const int64_t r = blockIdx.x / a.G;
  const Stretch<Tin> x(static_cast<const Tin*>(a.logits) + r * a.row_stride, a.V, blockIdx.x % a.G, a.G);
  write_part<Tin, BLOCK, KMAX>(x, a.k, scale_of(a.temperature[r]), s, list + static_cast<int64_t>(blockIdx.x) * a.k,
                               sums + blockIdx.x);
}

// The m-th largest of the wave's values, N of each lane, to its upper 20 bits (0:
// there are fewer above 0). m <= 64 N; `used` of the N are looked at.
template <int N>
__device__ __forceinline__ uint32_t wave_nth(const uint32_t (&v)[N], int used, int m) {
  uint32_t at = 0;
#pragma unroll 1
  for (int bit = 31; bit >= 12; --bit) {
    const uint32_t up = at | 1u << bit;
    int n = 0;
#pragma unroll
    for (int u = 0; u < N; ++u)
      if (N == 1 || u < used) n += __popcll(__ballot(v[u] >= up));
    if (n >= m) at = up;
  }
  return at;
}

// and the rows'. Where m parts have a j-th key not below some value and m j is
// at least k, no key below it is among the first k: each wave takes its own j.
// From what is left the k-th is looked for as in list_stretch.
__global__ __launch_bounds__(kRowBlock) void top_merge_kernel(TopArgs a, const uint64_t* list, const RowSum* sums) {
  constexpr int NW = kRowBlock / kWave, PER = kMaxSplit * kMaxTop / kRowBlock;
  __shared__ alignas(16) uint64_t key[kMaxSplit * kMaxTop + 4];
  __shared__ alignas(16) uint32_t hist[256];
  __shared__ CutLds cut_lds;
  __shared__ uint32_t bound[NW], n_key;
  const int64_t r = blockIdx.x;
  const int t = threadIdx.x, lane = t % kWave, wave = t / kWave, N = a.G * a.k;
  const uint64_t* mine = list + r * N;
  uint64_t x[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) x[i] = t + i * kRowBlock < N ? mine[t + i * kRowBlock] : 0;
  const bool part = lane < a.G;
  const RowSum e = part ? sums[r * a.G + lane] : RowSum{-INFINITY, 0.0f};
  const float T = a.temperature[r];
  const int share = (a.k + a.G - 1) / a.G, j = wave == NW - 1 ? a.k : min(a.k, share << wave);
  const uint32_t jth[1] = {part ? static_cast<uint32_t>(mine[lane * a.k + j - 1] >> 32) : 0u};
  const uint32_t b = wave_nth(jth, 1, (a.k + j - 1) / j);
  if (lane == 0) bound[wave] = b;
  hist[t] = 0;
  if (t == 0) n_key = 0;
  __syncthreads();
  uint32_t floor = 0;
  for (int w = 0; w < NW; ++w) floor = max(floor, bound[w]);
  const RowNorm norm = row_norm(merge_lanes(e, scale_of(T)), T);
  // All keys are between the floor and the row's largest logit.
  const float low = key_float(floor), width = (norm.m - low) * (1.0f / 255.0f);
  const float scale = floor > 0 && width > 0.0f && width < INFINITY ? 1.0f / width : 0.0f;
  auto bin_of = [&](uint64_t v) {
    return scale > 0.0f ? static_cast<int>(fminf(fmaxf((key_logit(v) - low) * scale, 0.0f), 255.0f)) : 255;
  };
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (static_cast<uint32_t>(x[i] >> 32) < floor) x[i] = 0;
    if (x[i] != 0) atomicAdd(&hist[bin_of(x[i])], 1u);
  }
  __syncthreads();
  const int from = cut_bin(hist, static_cast<uint32_t>(a.k));
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (x[i] != 0 && bin_of(x[i]) >= from) key[atomicAdd(&n_key, 1u)] = x[i];
  __syncthreads();
  if (n_key > static_cast<uint32_t>(a.k + a.k / 2 + 64)) {
    const Cut cut = find_cut<kRowBlock>([&](auto fn) {
#pragma unroll
      for (int i = 0; i < PER; ++i) fn(x[i]);
    }, static_cast<uint32_t>(a.k), cut_lds);
    if (t == 0) n_key = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (cut.takes(x[i])) key[atomicAdd(&n_key, 1u)] = x[i];
    __syncthreads();
  }
  const int n = close_list(key, static_cast<int>(n_key));
  write_top<kRowBlock>(a, r, norm, n, [&](int m, auto fn) {
    in_order_by_bins<kRowBlock>(key, key + kMaxSplit * kMaxTop / 2, m, hist, bin_of, fn);
  });
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

// The first k tokens of each part of the live beams' rows, and its sum of exps.
// 256 rows of 151,936 bfloat16 logits 20.7 us (3.8 TB/s), 410 live of 512 rows of
// 262,144 float32 logits 69 us (6.2 TB/s).
template <typename Tin, int BLOCK, int KMAX>
__global__ __launch_bounds__(BLOCK) void beam_rows_kernel(BeamArgs a, RowSum* sums, uint64_t* list, int64_t first) {
  __shared__ ListLds<BLOCK, KMAX> s;
  const int64_t r = first + blockIdx.x / a.G, at = first + blockIdx.x;  // first: 0 unless G = 1
  uint32_t flags;
  if (!beam_live(a, r, &flags)) return;
  const Stretch<Tin> x(static_cast<const Tin*>(a.logits) + r * a.row_stride, a.V, blockIdx.x % a.G, a.G);
  write_part<Tin, BLOCK, KMAX>(x, a.k, scale_of(a.temperature[r]), s, list + at * a.k, sums + at);
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

// The k best candidates of a request, by one workgroup. The parts' lists are in
// order: where m of them have a j-th candidate not below some score and m j is
// at least k, no candidate below it is among the best. With j in powers of two
// fewer than 2 k (1 + log2 k) are above the largest of these scores, however they
// spread over the lists; the bound itself keeps 20 bits of a float32 score's key
// (11 of its fraction: 0.008 nats at -20, 0.5 at -2,000), and candidates that are
// equal or in that band below it are looked at too. Of larger requests up to
// kListed are cut by 256 bins of their scores; what is left is counted against each
// other, or, where it is more than kCounted, selected from by digits. SMALL: a
// request has at most kHeld candidates, which the threads read at once and hold. A
// chain of a few reads and barriers bounds it: 5.1 us for one request, 6.2 for 64.
// With the rows' kernel, k = 128, 64 beams of 151,936 bfloat16 logits whose scores
// differ take 77 us, alike 59. (Rows in eight parts: 99 and 67; with three j beside
// k and no bins 1,234 and 51.)
constexpr int kCounted = 512, kHeld = 4 * kBeamBlock, kListed = 4096;

template <bool SMALL>
__global__ __launch_bounds__(kBeamBlock) void beam_merge_kernel(BeamArgs a, const RowSum* sums, const uint64_t* list) {
  constexpr int NW = kBeamBlock / kWave, HELD = SMALL ? kHeld / kBeamBlock : 1;
  __shared__ RowNorm norm[PR_MAX_BEAMS];
  __shared__ double base[PR_MAX_BEAMS];
  __shared__ int state[PR_MAX_BEAMS];  // 0: no candidates, 1: its tokens, 2: itself
  __shared__ Candidate best[kCounted];
  __shared__ alignas(16) uint32_t near[kCounted + 4];
  __shared__ uint32_t held[SMALL ? kHeld : 1];
  // Of larger requests the candidates from the floor on: their scores and entries.
  __shared__ uint32_t listed[SMALL ? 1 : kListed];
  __shared__ int32_t entry[SMALL ? 1 : kListed];
  __shared__ alignas(16) uint32_t hist[SMALL ? 4 : 256];
  __shared__ uint32_t n_listed, least, most;
  __shared__ uint32_t bound[NW], n_best;
  __shared__ CutLds cut_lds;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * a.B;
  const int t = threadIdx.x, lane = t % kWave, wave = t / kWave;
  const int per = a.G * a.k, N = a.B * per, lists = a.B * a.G;  // per: entries of a beam
  const uint64_t* mine = list + first * per;
  uint64_t token[HELD];
  if constexpr (SMALL) {
#pragma unroll
    for (int i = 0; i < HELD; ++i) token[i] = t + i * kBeamBlock < N ? mine[t + i * kBeamBlock] : 0;
  }
  if (t < a.B) {
    // (The sums of a beam that is not live are read all the same: at once with its score.)
    const float score = a.scores[first + t], T = a.temperature[first + t];
    const RowNorm y = row_norm(merge_parts(sums + (first + t) * a.G, a.G, scale_of(T)), T);
    uint32_t flags;
    const bool live = beam_live(a, first + t, &flags);
    RowNorm x{0.0, 0.0f, 1.0f, 0};
    if (live) {
      x = y;
      flags = x.flags;
    }
    norm[t] = x;
    base[t] = static_cast<double>(score);
    state[t] = live ? (flags ? 0 : 1) : (flags == PR_FLAG_MASKED && score > -INFINITY ? 2 : 0);
    if (a.out.flags) a.out.flags[first + t] = flags;
  }
  if (t == 0) n_best = 0;
  __syncthreads();
  // The score key (0: none) of entry i of the request's lists, which reads `key`.
  auto score_of = [&](int i, uint64_t key) -> uint64_t {
    const int b = i / per;
    if (state[b] == 1) return key != 0 ? score_key(base[b] + norm[b].logprob(key_logit(key))) : 0;
    return state[b] == 2 && i == b * per ? score_key(base[b]) : 0;
  };
  uint64_t score[HELD];
  if constexpr (SMALL) {
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const int e = t + i * kBeamBlock;
      score[i] = e < N ? score_of(e, token[i]) : 0;
      if (e < N) held[e] = near_key(score[i]);
    }
    __syncthreads();
  }
  const int share = (a.k + lists - 1) / lists;
  // What the j-th candidates of the lists bound.
  auto bound_of = [&](int j) -> uint32_t {
    constexpr int PER = PR_MAX_BEAMS * kMaxSplit / kWave;
    const int m = (a.k + j - 1) / j, used = (lists + kWave - 1) / kWave;
    auto jth = [&](int l) -> uint32_t {
      if (l >= lists) return 0;
      const int e = l * a.k + j - 1;
      if constexpr (SMALL) return held[e];
      return near_key(score_of(e, mine[e]));
    };
    if (used == 1) {
      const uint32_t v[1] = {jth(lane)};
      return wave_nth(v, 1, m);
    }
    uint32_t v[PER];
#pragma unroll
    for (int u = 0; u < PER; ++u) v[u] = u < used ? jth(u * kWave + lane) : 0;
    return wave_nth(v, used, m);
  };
  {
    // j = share, 2 share, 4 share, .., k, dealt to the waves; of a small request's one
    // each, which leaves few enough.
    uint32_t at = 0;
    if constexpr (SMALL) {
      at = bound_of(wave == NW - 1 ? a.k : min(a.k, share << wave));
    } else {
#pragma unroll 1
      for (int i = wave; i == 0 || share << (i - 1) < a.k; i += NW) at = max(at, bound_of(min(a.k, share << i)));
    }
    if (lane == 0) bound[wave] = at;
  }
  __syncthreads();
  uint32_t floor = 0;
  for (int w = 0; w < NW; ++w) floor = max(floor, bound[w]);
  // fn(entry, score's key, beam, token) for each candidate from the floor on. The
  // lists are in order: a wave walks its own, `span` lanes a list and four entries a
  // lane at a time, for as long as one of them reaches the floor.
  auto walk = [&](auto fn) {
    const int own = (lists - wave + NW - 1) / NW;
    const int span = own >= kWave ? 1 : 1 << (31 - __builtin_clz(kWave / max(own, 1)));
    for (int l0 = 0; l0 < own; l0 += kWave / span) {
      const int l = (l0 + lane / span) * NW + wave;
      const bool mine_too = l0 + lane / span < own;
      const int b = mine_too ? l / a.G : 0;
      for (int j0 = lane % span;; j0 += 4 * span) {
        uint64_t key[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          key[i] = mine_too && j0 + i * span < a.k && state[b] == 1 ? mine[l * a.k + j0 + i * span] : 0;
        bool any = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int j = j0 + i * span, e = l * a.k + j;
          const uint64_t s = mine_too && j < a.k ? score_of(e, key[i]) : 0;
          if (s == 0 || near_key(s) < floor) continue;
          any = true;
          fn(e, s, b, key[i]);
        }
        if (!__any(any)) break;
      }
    }
  };
  bool in_list = false;
  if constexpr (!SMALL) {
    if (t == 0) {
      n_listed = most = 0;
      least = ~0u;
    }
    hist[t] = 0;
    __syncthreads();
    walk([&](int e, uint64_t s, int, uint64_t) {
      const uint32_t at = atomicAdd(&n_listed, 1u), key = near_key(s);
      atomicMax(&most, key);
      atomicMin(&least, key);
      if (at < static_cast<uint32_t>(kListed)) {
        listed[at] = key;
        entry[at] = e;
      }
    });
    __syncthreads();
    const int n = static_cast<int>(n_listed);
    in_list = n <= kListed;
    if (in_list && n > kCounted) {
      // Those from the k-th's of 256 bins on.
      constexpr int PER = kListed / kBeamBlock;
      const float low = key_float(least), width = (key_float(most) - low) * (1.0f / 255.0f);
      const float scale = width > 0x1p-120f && width < INFINITY ? 1.0f / width : 0.0f;
      uint32_t key[PER];
      int32_t e[PER], bin[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int at = t + i * kBeamBlock;
        bin[i] = -1;
        if (at >= n) continue;
        key[i] = listed[at];
        e[i] = entry[at];
        bin[i] = static_cast<int>(fminf(fmaxf((key_float(key[i]) - low) * scale, 0.0f), 255.0f));
        atomicAdd(&hist[bin[i]], 1u);
      }
      __syncthreads();
      const int from = cut_bin(hist, static_cast<uint32_t>(a.k));
      if (t == 0) n_listed = 0;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        if (bin[i] < from) continue;
        const uint32_t at = atomicAdd(&n_listed, 1u);
        listed[at] = key[i];
        entry[at] = e[i];
      }
      __syncthreads();
    }
  }
  // Each candidate of the thread from the floor on: its score's key, beam and token.
  auto candidates = [&](auto fn) {
    if constexpr (SMALL) {
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        if (score[i] != 0 && near_key(score[i]) >= floor) fn(score[i], (t + i * kBeamBlock) / per, token[i]);
    } else if (in_list) {
      for (int i = t; i < static_cast<int>(n_listed); i += kBeamBlock) {
        const int e = entry[i], b = e / per;
        const uint64_t key = state[b] == 1 ? mine[e] : 0;
        fn(score_of(e, key), b, key);
      }
    } else {
      walk([&](int, uint64_t s, int b, uint64_t key) { fn(s, b, key); });
    }
  };
  candidates([&](uint64_t s, int b, uint64_t key) {
    const uint32_t at = atomicAdd(&n_best, 1u);
    if (at < static_cast<uint32_t>(kCounted)) best[at] = Candidate{s, key, b};
  });
  __syncthreads();
  if (n_best > static_cast<uint32_t>(kCounted)) {
    const uint32_t k = static_cast<uint32_t>(a.k);
    const Cut by_score = find_cut<kBeamBlock>([&](auto fn) {
      candidates([&](uint64_t s, int, uint64_t) { fn(s); });
    }, k, cut_lds);
    Cut by_beam{0, 0, 0, false}, by_token{0, 0, 0, false};
    if (by_score.more) {  // equal scores: by beam, then by token
      by_beam = find_cut<kBeamBlock>([&](auto fn) {
        candidates([&](uint64_t s, int b, uint64_t) { fn(s == by_score.value ? static_cast<uint64_t>(255 - b) : 0); });
      }, by_score.need, cut_lds, 0x7fu);
      if (by_beam.more)
        by_token = find_cut<kBeamBlock>([&](auto fn) {
          candidates([&](uint64_t s, int b, uint64_t key) {
            fn(s == by_score.value && static_cast<uint64_t>(255 - b) == by_beam.value ? key : 0);
          });
        }, by_beam.need, cut_lds);
    }
    if (t == 0) n_best = 0;
    __syncthreads();
    candidates([&](uint64_t s, int b, uint64_t key) {
      bool take = by_score.takes(s);
      if (take && by_score.more && s == by_score.value) {
        const uint64_t kb = static_cast<uint64_t>(255 - b);
        take = by_beam.takes(kb) && (!by_beam.more || by_beam.above(kb) || by_token.takes(key));
      }
      if (take) best[atomicAdd(&n_best, 1u)] = Candidate{s, key, b};
    });
    __syncthreads();
  }
  const int n = static_cast<int>(n_best);
  for (int e = t; e < n + 4; e += kBeamBlock) near[e] = e < n ? near_key(best[e].score) : 0;
  __syncthreads();
  auto write = [&](int at, float s, int32_t parent, int32_t v, float lp) {
    const int64_t o = static_cast<int64_t>(blockIdx.x) * a.k + at;
    a.out.scores[o] = s;
    a.out.parent[o] = parent;
    a.out.token[o] = v;
    if (a.out.logprob) a.out.logprob[o] = lp;
  };
  for (int e = t; e < n; e += kBeamBlock) {
    const uint32_t my = near[e];
    int at = 0, same = 0;
    for (int i = 0; i < n; i += 4) {
      const vec4u q = *reinterpret_cast<const vec4u*>(near + i);
      at += (q.x > my ? 1 : 0) + (q.y > my ? 1 : 0) + (q.z > my ? 1 : 0) + (q.w > my ? 1 : 0);
      same += (q.x == my ? 1 : 0) + (q.y == my ? 1 : 0) + (q.z == my ? 1 : 0) + (q.w == my ? 1 : 0);
    }
    if (at >= a.k) continue;
    const Candidate c = best[e];
    if (same > 1)
      for (int i = 0; i < n; ++i) at += near[i] == my && best[i].before(c) ? 1 : 0;
    if (at >= a.k) continue;
    const bool itself = state[c.beam] == 2;
    const double l = itself ? 0.0 : norm[c.beam].logprob(key_logit(c.token));
    write(at, static_cast<float>(base[c.beam] + l), c.beam, itself ? a.done_token : key_index(c.token),
          static_cast<float>(l));
  }
  if (t >= n && t < a.k) write(t, -INFINITY, -1, -1, -INFINITY);
}

// Most workgroups of a launch: one that has 2^32 threads or more along x does not run.
constexpr int64_t most_groups(int block) { return (int64_t{1} << 31) / block; }
// fn(first, groups) for each of the launches that `groups` workgroups take.
template <typename Fn>
hipError_t in_launches(int64_t groups, int block, Fn&& fn) {
  for (int64_t at = 0; at < groups; at += most_groups(block)) {
    fn(at, dim3(static_cast<unsigned>(groups - at < most_groups(block) ? groups - at : most_groups(block))));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Workgroups along a row that is taken in parts: about 512 in all, each with at
// least 512 vectors. About 256 and 512 in all, k = 64: 128 rows of 262,144 float32
// logits 39.4 and 34.0, 16 rows 19.4 and 19.3. At least 256 and 512 vectors: 17
// rows of 50,257 bfloat16 logits, k = 256, 32.5 and 29.6.
constexpr int64_t kGroups = 512, kLeastVectors = 512;

int row_groups(int64_t n_rows, int64_t nvec) {
  const int64_t want = (kGroups + n_rows - 1) / n_rows, most = nvec / kLeastVectors;
  const int64_t G = want < most ? want : most;
  return static_cast<int>(G < 1 ? 1 : G > kMaxSplit ? kMaxSplit : G);
}

// Workgroups along a beam's row. Longer lists are whole rows', as the merge takes
// all lists of a request. In parts and whole, requests of 4 beams: of 151,936
// bfloat16 logits k = 4, 64 rows 19.4 and 24.8 us, 128 rows 23.2 and 25.4, 160
// rows 25.7 and 25.5, k = 16, 64 rows 23.9 and 28.4, k = 64, 44.5 and 40.1, k =
// 256, 141 and 105; of 32,000 float32 logits k = 4, 64 rows 14.9 and 17.4, k = 64,
// 28.7 and 20.3; of 262,144 float32 logits (65,536 vectors) k = 64, 16 rows 30.6
// and 37.9, 64 rows 36.9 and 39.6, k = 128, 47.9 and 45.9.
constexpr int64_t kWholeBeams = 160, kLongVectors = 32768;

int beam_split(int64_t n_rows, int32_t V, pr_dtype dtype, int32_t k) {
  const int64_t nvec = V / (dtype == PR_BF16 ? 8 : 4);
  if (n_rows <= 0 || n_rows >= kWholeBeams || k > (nvec < kLongVectors ? 32 : 64)) return 1;
  return row_groups(n_rows, nvec);
}

// And along a row of which no request's beams are merged: whole rows save a
// launch, which is more than parts save of a short row or of many. In parts and
// whole: 64 rows of 32,000 float32 logits (8,000 vectors), k = 8, 16.8 and 13.9;
// of 18,992 vectors, k = 16, 32 rows 18.2 and 20.1, 64 rows 19.6 and 20.6, 96 rows
// 22.7 and 20.9, k = 256, 16 rows 25.6 and 27.7, 64 rows 32.4 and 27.9; of 65,536
// vectors, k = 16, 96 rows 31.0 and 31.4, 160 rows 39.0 and 35.1, k = 256, 64 rows
// 32.5 and 43.3, 160 rows 48.9 and 43.9.
constexpr int64_t kWholeVectors = 12288, kWholeRows = 128;

int top_split(int64_t n_rows, int32_t V, pr_dtype dtype, int32_t k) {
  const int64_t nvec = V / (dtype == PR_BF16 ? 8 : 4);
  const int64_t most = (nvec / 256 < kWholeRows ? nvec / 256 : kWholeRows) / (k > 64 && nvec <= kLongVectors ? 2 : 1);
  return n_rows <= 0 || nvec <= kWholeVectors || n_rows >= most ? 1 : row_groups(n_rows, nvec);
}

// Whether whole rows are taken by 512 threads: up to a few hundred, which are a
// workgroup or two a compute unit, and lists of more than 64, which take more of
// a compute unit's shared memory. 256 and 512 threads, us: k = 8, 512 rows of
// 151,936 bfloat16 logits 33.5 and 31.8, 1,024 55.3 and 57.6, 2,048 101 and 108,
// 16,972 806 and 865 (k = 64); 512 rows of 32,000 float32 logits 17.1 and 17.3,
// 1,024 26.0 and 26.5. k = 200: 512 rows of 151,936 45.3 and 38.4, 2,048 130 and
// 125, of 32,000 float32 65 and 55.
bool wide_rows(int64_t n_rows) { return n_rows <= 512; }
template <int KMAX>
constexpr int kManyBlock = KMAX <= 64 ? kRowBlock : 2 * kRowBlock;  // of more rows

size_t lists_bytes(int64_t n_rows, int G, int32_t k) {
  return static_cast<size_t>(n_rows) * static_cast<size_t>(G) * (static_cast<size_t>(k) * sizeof(uint64_t) + sizeof(RowSum));
}

template <typename Tin, int KMAX>
hipError_t top(const TopArgs& a, hipStream_t stream) {
  if (a.G > 1) {
    uint64_t* list = static_cast<uint64_t*>(a.ws);
    RowSum* sums = reinterpret_cast<RowSum*>(list + a.n_rows * a.G * a.k);
    hipLaunchKernelGGL((top_parts_kernel<Tin, kRowBlock, KMAX>), dim3(static_cast<unsigned>(a.n_rows * a.G)),
                       dim3(kRowBlock), 0, stream, a, list, sums);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(top_merge_kernel, dim3(static_cast<unsigned>(a.n_rows)), dim3(kRowBlock), 0, stream, a, list, sums);
    return hipGetLastError();
  }
  constexpr int MANY = kManyBlock<KMAX>;
  const bool wide = wide_rows(a.n_rows);
  return in_launches(a.n_rows, wide ? 2 * kRowBlock : MANY, [&](int64_t at, dim3 grid) {
    if (wide)
      hipLaunchKernelGGL((top_kernel<Tin, 2 * kRowBlock, KMAX>), grid, dim3(2 * kRowBlock), 0, stream, a, at);
    else
      hipLaunchKernelGGL((top_kernel<Tin, MANY, KMAX>), grid, dim3(MANY), 0, stream, a, at);
  });
}

template <typename Tin, int KMAX>
hipError_t beam(const BeamArgs& a, hipStream_t stream) {
  const int64_t n = static_cast<int64_t>(a.n_req) * a.B * a.G;
  uint64_t* list = static_cast<uint64_t*>(a.ws);
  RowSum* sums = reinterpret_cast<RowSum*>(list + n * a.k);
  constexpr int MANY = kManyBlock<KMAX>;
  const bool wide = a.G == 1 && wide_rows(static_cast<int64_t>(a.n_req) * a.B);
  // (Rows in parts are few: one launch, so that `at` is a row wherever it is not 0.)
  const hipError_t e = in_launches(n, wide ? 2 * kRowBlock : MANY, [&](int64_t at, dim3 grid) {
    if (wide)
      hipLaunchKernelGGL((beam_rows_kernel<Tin, 2 * kRowBlock, KMAX>), grid, dim3(2 * kRowBlock), 0, stream, a, sums,
                         list, at);
    else
      hipLaunchKernelGGL((beam_rows_kernel<Tin, MANY, KMAX>), grid, dim3(MANY), 0, stream, a, sums, list, at);
  });
  if (e != hipSuccess) return e;
  const dim3 reqs(static_cast<unsigned>(a.n_req));
  if (a.B * a.G * a.k <= kHeld)
    hipLaunchKernelGGL(beam_merge_kernel<true>, reqs, dim3(kBeamBlock), 0, stream, a, sums, list);
  else
    hipLaunchKernelGGL(beam_merge_kernel<false>, reqs, dim3(kBeamBlock), 0, stream, a, sums, list);
  return hipGetLastError();
}

}  // namespace

size_t top_workspace_bytes(int64_t n_rows, int32_t V, pr_dtype dtype, int32_t k) {
  const int G = top_split(n_rows, V, dtype, k);
  return G > 1 ? lists_bytes(n_rows, G, k) : 0;
}

hipError_t launch_top(const TopArgs& a, pr_dtype dtype, hipStream_t stream) {
  TopArgs x = a;
  x.G = top_split(a.n_rows, a.V, dtype, a.k);
  if (x.k <= 64) return dtype == PR_BF16 ? top<uint16_t, 64>(x, stream) : top<float, 64>(x, stream);
  return dtype == PR_BF16 ? top<uint16_t, kMaxTop>(x, stream) : top<float, kMaxTop>(x, stream);
}

size_t beam_workspace_bytes(int64_t n_rows, int32_t V, pr_dtype dtype, int32_t k) {
  return n_rows < 1 ? 0 : lists_bytes(n_rows, beam_split(n_rows, V, dtype, k), k);
}

hipError_t launch_beam(const BeamArgs& a, pr_dtype dtype, hipStream_t stream) {
  BeamArgs x = a;
  x.G = beam_split(static_cast<int64_t>(a.n_req) * a.B, a.V, dtype, a.k);
  if (x.k <= 64) return dtype == PR_BF16 ? beam<uint16_t, 64>(x, stream) : beam<float, 64>(x, stream);
  return dtype == PR_BF16 ? beam<uint16_t, kMaxTop>(x, stream) : beam<float, kMaxTop>(x, stream);
}

}  // namespace pr
