// The loss of a student's logit rows against a teacher's largest log-probs, and
// its gradient in the logits.
//
// A row's entries are the teacher's tokens v_i with q_i = exp(their log-prob).
// With u = z / T, p = softmax(u), Q = sum q_i, P = sum p_{v_i}, r_p = 1 - P and
// r_q = max(0, 1 - Q) (0 unless the rest is a term, and where r_p = 0):
//   l = sum q_i (log q_i - log p_{v_i}) + r_q (log r_q - log r_p)
//   dl/du_v = (Q + r_q) p_v - q_i             v = v_i
//           = (Q r_p - r_q P) (p_v / r_p)     any other v
// (q_i and Q divided by Q where the entries are normalised.)
//
// The sum over the tokens that are no entry's is taken on its own, relative to
// its own largest logit: 1 - P would keep nothing of it where the student is
// sure of the teacher's tokens, and the two factors above are finite at any r_p.
// The vectors that hold entries' tokens are marked in a bit map, which the pass
// over the row leaves out; a thread for each takes those.
//
// Exponents are in base 2 and sums as in the other losses: float32 sums of
// positive terms, compensated per lane; what follows per row and over rows is
// in 64 bits. A gradient element is rounded to its type once.
#include <algorithm>

#include "distill.h"
#include "held_rows.h"

namespace pr {
namespace {

constexpr int kMaxTop = PR_MAX_TOP_LOGITS;
constexpr int kStatsBlock = 256;  // a thread for each of a row's entries
constexpr int kGradBlock = 512;
constexpr int kWindow = 1 << 16;  // vectors of a bit map
static_assert(kStatsBlock >= kMaxTop && kGradBlock >= kMaxTop, "a thread for each entry");

// What the gradient pass needs of a row: dz_v = k 2^fma(z_v, c, -A) outside the
// entries, in_k 2^fma(z_v, in_c, -in_A) - q_k q_i in them (either part relative to
// its own largest logit), the products in 64 bits: where student and teacher agree
// little is left of the two. All factors 0: the gradient is zero and the row is not
// read.
struct alignas(16) RowDistill {
  float A, k, c, in_A;
  double in_k, q_k;
  float in_c;

  __device__ __forceinline__ float in_entry(float z, double q) const {
    return static_cast<float>(in_k * static_cast<double>(fast_exp2(fmaf(z, in_c, -in_A))) - q_k * q);
  }
};

// A row's entries by token for the gradient pass: those of its workgroup p along
// the row are begin[p] .. begin[p + 1] - 1.
struct SortedEntry {
  int32_t id;
  double q;
};
struct SortedRows {
  SortedEntry* entry;  // [n_rows][k]
  int32_t* begin;      // [n_rows][parts + 1]
  int32_t parts;
};

// Sums over the entries. u is taken relative to the largest of their logits
// (entry_ref), so that what a row's logits have in common, however large, is no
// part of the loss's terms.
struct EntrySums {
  double Q, cross;  // sum q, sum q (log q - u)
};
__device__ __forceinline__ float entry_ref(const RowSum& in) { return in.m > -INFINITY ? in.m : 0.0f; }
// cross relative to `top`, the largest logit of the entries of all parts, from one
// part's. over_T: 1 / T.
__device__ __forceinline__ double cross_from(const EntrySums& e, const RowSum& in, float top, double over_T) {
  if (in.m == -INFINITY || in.m == top) return e.cross;
  return e.cross - e.Q * ((static_cast<double>(in.m) - static_cast<double>(top)) * over_T);
}

// What a row comes to: `in` are the tokens of the entries, `out` the others.
struct RowLoss {
  double loss, mass;
  uint32_t flags;
  RowDistill grad;
};

__device__ __forceinline__ uint32_t row_flags(const RowSum& in, const RowSum& out, uint32_t bad, float T) {
  uint32_t flags = bad;
  if (!temperature_ok(T)) flags |= PR_FLAG_BAD_TP;
  const float m = fmaxf(in.m, out.m);
  if (!(fabsf(in.S) < INFINITY) || !(fabsf(out.S) < INFINITY) || m == INFINITY || m == -INFINITY)
    flags |= PR_FLAG_NONFINITE;
  if (!flags && fabsf(m) > ldexpf(T, 100)) flags |= PR_FLAG_BAD_TP;
  return flags;
}

// Whether the rest is a term, and its q.
__device__ __forceinline__ double rest_q(const DistillArgs& a, const RowSum& out, double Q) {
  return a.tail == PR_TAIL_REST && out.S > 0.0f ? fmax(0.0, 1.0 - Q) : 0.0;
}

// The gradient's factors. The sums are S 2^A of each part, so P and r_p come
// from two exponentials and a division in float32, without a logarithm: the
// waves that hold a row wait for this.
__device__ __forceinline__ RowDistill row_factors(const DistillArgs& a, const RowSum& in, const RowSum& out, double Q,
                                                  uint32_t flags, float T, float c, float w) {
  const float nan = __uint_as_float(0x7fc00000u);
  if (flags) return RowDistill{0.0f, nan, 0.0f, 0.0f, nan, nan, 0.0f};
  RowDistill g;
  const RowRef ro = row_ref(out.S > 0.0f ? out.m : 0.0f, c), ri = row_ref(in.S > 0.0f ? in.m : 0.0f, c);
  g.c = ro.c;
  g.A = ro.A;
  g.in_c = ri.c;
  g.in_A = ri.A;
  const float top = fmaxf(in.m, out.m);
  // Of each part: its scale beside the larger, and its sum so scaled.
  const float si = in.S > 0.0f ? fast_exp2(ref_shift(in.m, top, c)) : 0.0f;
  const float so = out.S > 0.0f ? fast_exp2(ref_shift(out.m, top, c)) : 0.0f;
  const double pi = static_cast<double>(in.S) * static_cast<double>(si);
  const double po = static_cast<double>(out.S) * static_cast<double>(so), all = pi + po;
  const double rq = rest_q(a, out, Q), scale = a.tail == PR_TAIL_RENORM ? (Q > 0.0 ? 1.0 / Q : 0.0) : 1.0;
  const double q = a.tail == PR_TAIL_RENORM ? (Q > 0.0 ? 1.0 : 0.0) : Q;
  const double coef = a.grad_scale * static_cast<double>(w) / static_cast<double>(T), each = coef / all;
  g.k = out.S > 0.0f ? static_cast<float>(each * (q * po - rq * pi) / static_cast<double>(out.S)) : 0.0f;
  g.in_k = each * (q + rq) * static_cast<double>(si);
  g.q_k = coef * scale;
  return g;
}

// log of a sum of exps of u relative to the logit `from`, in 64 bits. S is relative
// to the reference's A, whose exact residual goes off its logarithm.
__device__ __forceinline__ double log_sum(const RowSum& p, float from, float T, float c) {
  if (!(p.S > 0.0f)) return -__longlong_as_double(0x7ff0000000000000ll);
  const RowRef ref = row_ref(p.m, c);
  const double delta = static_cast<double>(fmaf(p.m, ref.c, -ref.A));
  return (static_cast<double>(p.m) - static_cast<double>(from)) / static_cast<double>(T) + log(static_cast<double>(p.S)) -
         delta * 0.69314718055994530942;
}

// The loss and the student's probability of the entries' tokens.
__device__ __forceinline__ void row_terms(const DistillArgs& a, const RowSum& in, const RowSum& out, const EntrySums& e,
                                          float T, float c, RowLoss& x) {
  if (x.flags) {
    x.loss = x.mass = __longlong_as_double(0x7ff8000000000000ll);
    return;
  }
  const float from = entry_ref(in);
  const double li = log_sum(in, from, T, c), lo = log_sum(out, from, T, c);
  const double hi = fmax(li, lo), lse = hi + log1p(exp(fmin(li, lo) - hi)), rq = rest_q(a, out, e.Q);
  x.mass = exp(li - lse);
  x.loss = e.cross + e.Q * lse;
  if (a.tail == PR_TAIL_RENORM) x.loss = e.Q > 0.0 ? x.loss / e.Q - log(e.Q) : 0.0;
  if (rq > 0.0) x.loss += rq * (log(rq) - (lo - lse));
}

__device__ __forceinline__ RowLoss row_loss(const DistillArgs& a, const RowSum& in, const RowSum& out, const EntrySums& e,
                                            uint32_t bad, float T, float c, float w) {
  RowLoss x;
  x.flags = row_flags(in, out, bad, T);
  x.grad = row_factors(a, in, out, e.Q, x.flags, T, c, w);
  row_terms(a, in, out, e, T, c, x);
  return x;
}

__device__ __forceinline__ RowLoss masked_row() {
  return RowLoss{0.0, 0.0, PR_FLAG_MASKED, RowDistill{0.0f, 0.0f, 0.0f, 0.0f, 0.0, 0.0, 0.0f}};
}

__device__ __forceinline__ void write_row(const DistillArgs& a, int64_t r, const RowLoss& x) {
  if (a.out.token_loss) a.out.token_loss[r] = static_cast<float>(x.loss);
  if (a.out.mass) a.out.mass[r] = static_cast<float>(x.mass);
  if (a.out.flags) a.out.flags[r] = x.flags;
}

// Entry i of a row: its token (-1: none, or out of range), its log-prob and
// what is wrong with it.
struct Entry {
  int32_t id;
  float logq;
  uint32_t bad;
};

__device__ __forceinline__ Entry load_entry(const DistillArgs& a, int64_t r, int i) {
  Entry e{-1, -INFINITY, 0};
  if (i >= a.k) return e;
  const float lq = a.top_logprob[r * a.top_stride + i];
  const int32_t id = a.top_ids[r * a.top_stride + i];  // at once with it
  if (lq == -INFINITY) return e;
  if (!(lq < INFINITY)) e.bad |= PR_FLAG_NONFINITE;
  if (id < 0 || id >= a.rows.V) e.bad |= PR_FLAG_BAD_ID;
  if (!e.bad) {
    e.id = id;
    e.logq = lq;
  }
  return e;
}

// The stretch of up to VEC elements that a token belongs to: an aligned vector,
// or the elements before or after them all.
struct Group {
  int32_t base, len, vec;  // vec: -1 before the vectors, -2 after them
};

template <typename Tin>
__device__ __forceinline__ Group group_of(int32_t id, int32_t h, int32_t tail, int32_t V) {
  constexpr int VEC = Elem<Tin>::kVec;
  if (id < h) return Group{0, h, -1};
  if (id >= tail) return Group{tail, V - tail, -2};
  const int32_t j = (id - h) / VEC;
  return Group{h + j * VEC, VEC, j};
}

// Sums of two doubles over the workgroup; every thread gets them.
template <int BLOCK>
__device__ __forceinline__ EntrySums sum_entries(EntrySums e) {
  constexpr int NW = BLOCK / kWave;
  __shared__ EntrySums sh[NW];
  e.Q = wave_sum_d(e.Q);
  e.cross = wave_sum_d(e.cross);
  if (threadIdx.x % kWave == 0) sh[threadIdx.x / kWave] = e;
  __syncthreads();
  EntrySums t{0.0, 0.0};
  for (int w = 0; w < NW; ++w) {
    t.Q += sh[w].Q;
    t.cross += sh[w].cross;
  }
  return t;
}

// What a part of a row adds to its loss.
struct DistillPart {
  RowSum in, out;
  EntrySums entries;
  uint32_t bad, pad;
};

// A part of a row (workgroup g of G along it): its vectors' and their entries'
// sums; the first part also has the elements before the vectors, the last one
// those after them. Valid in thread 0. Every part looks at every entry.
// sorted: also writes the row's entries by token (G = 1).
template <typename Tin>
__device__ DistillPart row_part(const DistillArgs& a, int64_t r, int g, int G, float T, float c,
                                const SortedRows* sorted = nullptr) {
  constexpr int VEC = Elem<Tin>::kVec;
  __shared__ alignas(16) int32_t sh_id[kMaxTop + 4];  // the entries of this part, in no order
  __shared__ uint32_t marks[kWindow / 32];
  __shared__ int32_t by_id[kMaxTop];
  __shared__ uint32_t sh_bad, sh_ends, sh_n;
  const int t = threadIdx.x;
  const int32_t V = a.rows.V;
  const Tin* row = row_ptr<Tin>(a.rows, r);
  const int32_t h = static_cast<int32_t>(head_elems<Tin>(row, V)), nvec = (V - h) / VEC, tail = h + nvec * VEC;
  const int32_t vb = static_cast<int32_t>(static_cast<int64_t>(nvec) * g / G);
  const int32_t ve = static_cast<int32_t>(static_cast<int64_t>(nvec) * (g + 1) / G);
  const vec4u* vp = reinterpret_cast<const vec4u*>(row + h);
  vec4u v[4];
  const int32_t first_window = ve - vb < kWindow ? ve : vb + kWindow;
  scan::stretch_prefetch<Tin, kStatsBlock, 4>(row, h, vb, first_window, v);
  Entry e = load_entry(a, r, t);
  if (t == 0) sh_bad = sh_ends = sh_n = 0;
  for (int i = t; i < kWindow / 32; i += kStatsBlock) marks[i] = 0;
  __syncthreads();
  if (e.bad) atomicOr(&sh_bad, e.bad);
  const Group q = group_of<Tin>(e.id, h, tail, V);
  if (q.vec >= 0 ? q.vec < vb || q.vec >= ve : q.vec == -1 ? g != 0 : g != G - 1) e.id = -1;
  float z = -INFINITY;
  if (e.id >= 0) {
    z = Elem<Tin>::load1(row, e.id);
    sh_id[atomicAdd(&sh_n, 1u)] = e.id;
    if (q.vec >= 0 && q.vec < first_window) atomicOr(&marks[(q.vec - vb) / 32], 1u << (q.vec - vb) % 32);
    if (q.vec < 0) atomicOr(&sh_ends, q.vec == -1 ? 1u : 2u);
  }
  __syncthreads();
  const int n = static_cast<int>(sh_n);
  const uint32_t ends = sh_ends;
  if (t < 4) sh_id[n + t] = -1;
  LaneSum<true> in, out;
  out.add1(g == 0 && t < h && !(ends & 1u) ? Elem<Tin>::load1(row, t) : -INFINITY, c);
  out.add1(g == G - 1 && t < V - tail && !(ends & 2u) ? Elem<Tin>::load1(row, tail + t) : -INFINITY, c);
  for (int32_t w0 = vb; w0 < ve; w0 += kWindow) {
    const int32_t w1 = ve - w0 < kWindow ? ve : w0 + kWindow;
    if (w0 != vb) {
      for (int i = t; i < kWindow / 32; i += kStatsBlock) marks[i] = 0;
      __syncthreads();
      if (e.id >= 0 && q.vec >= w0 && q.vec < w1) atomicOr(&marks[(q.vec - w0) / 32], 1u << (q.vec - w0) % 32);
      __syncthreads();
      scan::stretch_prefetch<Tin, kStatsBlock, 4>(row, h, w0, w1, v);
    }
    // Without a branch: looking up which rounds have marks at all, and leaving
    // the others alone, took 209 to 227 us where this takes 192.
    scan::stream_stretch<Tin, kStatsBlock, 2, 4>(vp, w0, w1, v, [&](const vec4u* vv, int64_t j) {
      float x[2 * VEC];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        // Of the last rounds some vectors are past the window; they are -inf.
        const uint32_t at = static_cast<uint32_t>(static_cast<int32_t>(j) + u * kStatsBlock - w0) % kWindow;
        const bool marked = marks[at / 32] >> (at % 32) & 1u;
        Elem<Tin>::unpack(marked ? neg_inf_vec<Tin>() : vv[u], x + u * VEC);
      }
      out.add(x, c);
    });
    __syncthreads();
  }
  __syncthreads();
  in.add1(z, c);
  // The entry of a group's first token takes the group's other elements.
  {
    uint32_t mine = ~0u;
    if (e.id >= 0) {
      mine = 0;
      int same = 0, rank = 0;
      for (int i = 0; i < n; i += 4) {
        const vec4u o = *reinterpret_cast<const vec4u*>(sh_id + i);
        const uint32_t base = static_cast<uint32_t>(q.base), id = static_cast<uint32_t>(e.id);
        const uint32_t d[4] = {o.x - base, o.y - base, o.z - base, o.w - base};
#pragma unroll
        for (int u = 0; u < 4; ++u) mine |= d[u] < static_cast<uint32_t>(q.len) ? 1u << d[u] : 0u;
        same += (o.x == id ? 1 : 0) + (o.y == id ? 1 : 0) + (o.z == id ? 1 : 0) + (o.w == id ? 1 : 0);
        rank += (o.x < id ? 1 : 0) + (o.y < id ? 1 : 0) + (o.z < id ? 1 : 0) + (o.w < id ? 1 : 0);
      }
      if (sorted) {
        sorted->entry[r * a.k + rank] = SortedEntry{e.id, exp(static_cast<double>(e.logq))};
        by_id[rank] = e.id;
      }
      if (same > 1) atomicOr(&sh_bad, PR_FLAG_BAD_ID);
      if (mine & ((1u << (e.id - q.base)) - 1u)) mine = ~0u;
    }
    float other[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      other[i] = i < q.len && !(mine >> i & 1u) ? Elem<Tin>::load1(row, q.base + i) : -INFINITY;
    out.add(other, c);
  }
  DistillPart p;
  p.in = merge_block<kStatsBlock>(in, c);
  __syncthreads();
  // (An id that is there twice leaves gaps, in a row that is NaN.)
  if (sorted) {
    for (int32_t i = t; i <= sorted->parts; i += kStatsBlock) {
      const int64_t from = h + static_cast<int64_t>(i) * (kGradBlock * VEC);
      int lo = 0, len = i == 0 ? 0 : n;
      if (i == sorted->parts) lo = n, len = 0;
      while (len > 0) {  // the first entry not below `from`
        const int half = len / 2;
        const bool below = by_id[lo + half] < from;
        lo = below ? lo + half + 1 : lo;
        len = below ? len - half - 1 : half;
      }
      sorted->begin[r * (sorted->parts + 1) + i] = lo;
    }
  }
  p.out = merge_block<kStatsBlock>(out, c);
  // A probability of 0 adds nothing, whatever the student makes of its token.
  const double w = e.id >= 0 ? exp(static_cast<double>(e.logq)) : 0.0;
  EntrySums s{w, 0.0};
  if (w > 0.0)
    s.cross = w * (static_cast<double>(e.logq) -
                   (static_cast<double>(z) - static_cast<double>(entry_ref(p.in))) / static_cast<double>(T));
  p.entries = sum_entries<kStatsBlock>(s);
  p.bad = sh_bad;
  p.pad = 0;
  return p;
}

// One workgroup per row: its sums and everything but its gradient. The read
// bounds it where rows are long: 1,045 counting of 2,048 rows of 262,144 float32
// logits with 128 entries 209 us (5.3 TB/s); where they are short, their entries.
template <typename Tin>
__global__ __launch_bounds__(kStatsBlock) void distill_stats_kernel(DistillArgs a, double* term, RowDistill* rd,
                                                                   SortedRows sorted, int64_t first) {
  const int64_t r = first + blockIdx.x;
  const float w = a.rows.weight[r];
  RowLoss x = masked_row();
  if (w != 0.0f) {
    const float T = a.rows.temperature[r], c = scale_of(T);
    const DistillPart p = row_part<Tin>(a, r, 0, 1, T, c, sorted.entry ? &sorted : nullptr);
    if (threadIdx.x != 0) return;
    x = row_loss(a, p.in, p.out, p.entries, p.bad, T, c, w);
  } else if (threadIdx.x != 0) {
    return;
  }
  write_row(a, r, x);
  term[r] = w == 0.0f ? 0.0 : static_cast<double>(w) * x.loss;
  rd[r] = x.grad;
}

// The parts of a few rows, G of them a row: 17 rows of 50,257 bfloat16 logits with
// 256 entries 7.7 to 8.5 us, most of it a chain of barriers.
template <typename Tin>
__global__ __launch_bounds__(kStatsBlock) void distill_parts_kernel(DistillArgs a, DistillPart* part, int G) {
  const int64_t r = blockIdx.x / G;
  if (a.rows.weight[r] == 0.0f) return;
  const float T = a.rows.temperature[r];
  const DistillPart p = row_part<Tin>(a, r, blockIdx.x % G, G, T, scale_of(T));
  if (threadIdx.x == 0) part[blockIdx.x] = p;
}

// A row's loss from its parts, by one thread,
__device__ __forceinline__ RowLoss loss_from_parts(const DistillArgs& a, int64_t r, const DistillPart* part, int G) {
  const float w = a.rows.weight[r];
  if (w == 0.0f) return masked_row();
  const float T = a.rows.temperature[r], c = scale_of(T);
  const double over_T = 1.0 / static_cast<double>(T);
  RowSum in{-INFINITY, 0.0f}, out{-INFINITY, 0.0f};
#pragma unroll 4
  for (int g = 0; g < G; ++g) {
    in.m = fmaxf(in.m, part[r * G + g].in.m);
    out.m = fmaxf(out.m, part[r * G + g].out.m);
  }
  EntrySums e{0.0, 0.0};
  uint32_t bad = 0;
  auto add = [&](RowSum& s, const RowSum& p) {
    s.S += p.m == -INFINITY ? p.S : p.S * fast_exp2(ref_shift(p.m, s.m, c));
  };
#pragma unroll 4
  for (int g = 0; g < G; ++g) {
    const DistillPart p = part[r * G + g];
    add(in, p.in);
    add(out, p.out);
    e.Q += p.entries.Q;
    e.cross += cross_from(p.entries, p.in, in.m, over_T);
    bad |= p.bad;
  }
  return row_loss(a, in, out, e, bad, T, c, w);
}

// and by every wave of a workgroup, a lane a part.
__device__ __forceinline__ RowLoss loss_from_lanes(const DistillArgs& a, int64_t r, const DistillPart* part, int G) {
  const float w = a.rows.weight[r];
  if (w == 0.0f) return masked_row();
  const float T = a.rows.temperature[r], c = scale_of(T);
  const int lane = threadIdx.x % kWave;
  DistillPart p{{-INFINITY, 0.0f}, {-INFINITY, 0.0f}, {0.0, 0.0}, 0, 0};
  if (lane < G) p = part[r * G + lane];
  const uint32_t bad = (__any(p.bad & PR_FLAG_BAD_ID) ? PR_FLAG_BAD_ID : 0u) |
                       (__any(p.bad & PR_FLAG_NONFINITE) ? PR_FLAG_NONFINITE : 0u);
  const RowSum in = merge_lanes(p.in, c);
  const EntrySums s{wave_sum_d(p.entries.Q), wave_sum_d(cross_from(p.entries, p.in, in.m, 1.0 / static_cast<double>(T)))};
  return row_loss(a, in, merge_lanes(p.out, c), s, bad, T, c, w);
}

// All split rows' outputs, gradient factors (rd NULL: not wanted) and the loss,
// by one workgroup of kGradBlock threads.
__device__ __forceinline__ void finish_rows(const DistillArgs& a, const DistillPart* part, int G, RowDistill* rd) {
  __shared__ double sh[kGradBlock / kWave];
  double sum = 0.0;
  for (int64_t r = threadIdx.x; r < a.rows.n_rows; r += kGradBlock) {
    const RowLoss x = loss_from_parts(a, r, part, G);
    write_row(a, r, x);
    if (rd) rd[r] = x.grad;
    const float w = a.rows.weight[r];
    if (w != 0.0f) sum += static_cast<double>(w) * x.loss;
  }
  sum = wave_sum_d(sum);
  if (threadIdx.x % kWave == 0) sh[threadIdx.x / kWave] = sum;
  __syncthreads();
  if (threadIdx.x != 0) return;
  sum = 0.0;
  for (int w = 0; w < kGradBlock / kWave; ++w) sum += sh[w];
  a.loss[0] = static_cast<float>(sum);
}

__global__ __launch_bounds__(kGradBlock) void distill_finish_kernel(DistillArgs a, const DistillPart* part, int G,
                                                                   RowDistill* rd) {
  finish_rows(a, part, G, rd);
}

// The gradient of a stretch of a row, a vector per thread of workgroup `part`:
// short workgroups in memory order, past the caches. Each finds the entries
// among its own vectors.
template <typename Tin>
__device__ __forceinline__ void grad_stretch(const DistillArgs& a, int64_t r, int part, const RowDistill& q) {
  constexpr int VEC = Elem<Tin>::kVec;
  __shared__ uint32_t elements[(kGradBlock + 2 * 8) / 4];  // a byte a vector: its entries' elements; then the row's ends
  __shared__ double value[(kGradBlock + 2) * VEC];          // of those elements: q
  const int t = threadIdx.x;
  const int32_t V = a.rows.V;
  const Tin* row = row_ptr<Tin>(a.rows, r);
  Tin* out = static_cast<Tin*>(a.rows.grad) + r * a.rows.grad_stride;
  const int32_t h = static_cast<int32_t>(head_elems<Tin>(row, V)), nvec = (V - h) / VEC, tail = h + nvec * VEC;
  const int32_t j = part * kGradBlock + t;
  const bool ends = part == 0 && t < 16;
  const int32_t s = ends ? scalar_element(t, h, tail, V) : V;
  if (q.k == 0.0f && q.in_k == 0.0 && q.q_k == 0.0) {
    if (s < V) GradVec<Tin>::store1(out, s, 0.0f);
    if (j < nvec) stream_grad(out + h + static_cast<int64_t>(j) * VEC, vec4u{0, 0, 0, 0});
    return;
  }
  vec4u v = neg_inf_vec<Tin>();
  if (j < nvec) v = __builtin_nontemporal_load(reinterpret_cast<const vec4u*>(row + h) + j);
  const float zs = s < V ? Elem<Tin>::load1(row, s) : 0.0f;
  const Entry e = load_entry(a, r, t);
  if (t < static_cast<int>(sizeof(elements) / 4)) elements[t] = 0;
  __syncthreads();
  if (e.id >= 0) {
    const Group g = group_of<Tin>(e.id, h, tail, V);
    if (g.vec < 0 ? part == 0 : g.vec / kGradBlock == part) {
      const int slot = g.vec < 0 ? kGradBlock - 1 - g.vec : g.vec % kGradBlock, i = e.id - g.base;
      atomicOr(&elements[slot / 4], 1u << (slot % 4 * 8 + i));
      value[slot * VEC + i] = exp(static_cast<double>(e.logq));
    }
  }
  __syncthreads();
  const uint8_t* byte = reinterpret_cast<const uint8_t*>(elements);
  if (s < V) {
    const int slot = kGradBlock + t / 8, i = t % 8;
    GradVec<Tin>::store1(out, s, byte[slot] >> i & 1u
                                     ? q.in_entry(zs, value[slot * VEC + i])
                                     : q.k * fast_exp2(fmaf(zs, q.c, -q.A)));
  }
  if (j >= nvec) return;
  float z[VEC], g[VEC];
  Elem<Tin>::unpack(v, z);
#pragma unroll
  for (int i = 0; i < VEC; ++i) g[i] = q.k * fast_exp2(fmaf(z[i], q.c, -q.A));
  const uint32_t mine = byte[t];
  if (mine != 0) {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (mine >> i & 1u) g[i] = q.in_entry(z[i], value[t * VEC + i]);
  }
  stream_grad(out + h + static_cast<int64_t>(j) * VEC, GradVec<Tin>::pack(g));
}

// The gradients of the rows from `first` on (blockIdx.y), from factors that a
// kernel before has written; the first variant's entries are sorted. It moves the
// bytes of a copy: the 2,048 rows above 507 us (6.4 TB/s).
template <typename Tin>
__global__ __launch_bounds__(kGradBlock) void distill_sorted_grad_kernel(DistillArgs a, const RowDistill* rd,
                                                                        SortedRows sorted, int64_t first) {
  constexpr int VEC = Elem<Tin>::kVec;
  const int64_t r = first + blockIdx.y;
  const RowDistill q = rd[r];
  const int part = blockIdx.x, t = threadIdx.x;
  const int32_t V = a.rows.V;
  const Tin* row = row_ptr<Tin>(a.rows, r);
  Tin* out = static_cast<Tin*>(a.rows.grad) + r * a.rows.grad_stride;
  const int32_t h = static_cast<int32_t>(head_elems<Tin>(row, V)), nvec = (V - h) / VEC, tail = h + nvec * VEC;
  const int32_t j = part * kGradBlock + t;
  // The elements before the vectors go with the first part, those after them with the last.
  int32_t s = V;
  if (t < 8 && part == 0 && t < h) s = t;
  if (t >= 8 && t < 16 && part == sorted.parts - 1 && t - 8 < V - tail) s = tail + t - 8;
  if (q.k == 0.0f && q.in_k == 0.0 && q.q_k == 0.0) {
    if (s < V) GradVec<Tin>::store1(out, s, 0.0f);
    if (j < nvec) stream_grad(out + h + static_cast<int64_t>(j) * VEC, vec4u{0, 0, 0, 0});
    return;
  }
  const int32_t* begin = sorted.begin + r * (sorted.parts + 1) + part;
  const int32_t from = begin[0], to = begin[1];
  const SortedEntry* entry = sorted.entry + r * a.k;
  if (s < V) {
    const float z = Elem<Tin>::load1(row, s);
    float g = q.k * fast_exp2(fmaf(z, q.c, -q.A));
    for (int32_t i = from; i < to; ++i)
      if (entry[i].id == s) g = q.in_entry(z, entry[i].q);
    GradVec<Tin>::store1(out, s, g);
  }
  if (j >= nvec) return;
  float z[VEC], g[VEC];
  Elem<Tin>::unpack(__builtin_nontemporal_load(reinterpret_cast<const vec4u*>(row + h) + j), z);
#pragma unroll
  for (int i = 0; i < VEC; ++i) g[i] = q.k * fast_exp2(fmaf(z[i], q.c, -q.A));
  const int32_t base = h + j * VEC;
  for (int32_t i = from; i < to; ++i) {
    const int32_t d = entry[i].id - base;
    if (d < 0 || d >= VEC) continue;
    float zd = z[0];
#pragma unroll
    for (int u = 1; u < VEC; ++u) zd = u == d ? z[u] : zd;
    const float gd = q.in_entry(zd, entry[i].q);
#pragma unroll
    for (int u = 0; u < VEC; ++u) g[u] = u == d ? gd : g[u];
  }
  stream_grad(out + h + static_cast<int64_t>(j) * VEC, GradVec<Tin>::pack(g));
}

template <typename Tin>
__global__ __launch_bounds__(kGradBlock) void distill_grad_kernel(DistillArgs a, const RowDistill* rd) {
  grad_stretch<Tin>(a, blockIdx.y, blockIdx.x, rd[blockIdx.y]);
}

// The gradients of a few split rows: each workgroup works out its own row's
// factors instead of waiting for a kernel that does (the 17 rows above: 5.9 us).
// The first workgroup of the grid's last row finishes the rows.
template <typename Tin>
__global__ __launch_bounds__(kGradBlock) void distill_parts_grad_kernel(DistillArgs a, const DistillPart* part, int G) {
  if (blockIdx.y + 1 < gridDim.y)
    grad_stretch<Tin>(a, blockIdx.y, blockIdx.x, loss_from_lanes(a, blockIdx.y, part, G).grad);
  else if (blockIdx.x == 0)
    finish_rows(a, part, G, nullptr);
}

// The entries of a row as the wave that takes them holds them, KE a lane.
template <int KE>
struct Held {
  int32_t id[KE];
  float logq[KE];
  uint32_t mine[KE];  // which elements of its group are entries' tokens
  uint32_t ends;      // the same of the elements before (low byte) and after the vectors
  uint32_t bad;
};

__device__ __forceinline__ uint32_t group_slot(const Group& g, int32_t nvec) {
  return static_cast<uint32_t>(g.vec >= 0 ? g.vec : nvec + (g.vec == -1 ? 0 : 1));
}

// The loss of a row and its gradient in one read of the row, as the policy
// loss's kernel for such rows: the row's vectors stay in the registers of DW
// waves between their sum and their gradient, and one more wave takes what is
// scalar in a row. That wave also takes the entries: a bit map of the vectors
// that hold their tokens, made a row ahead, tells the others which vectors to
// leave to it, in the sum and in the gradient. There are three bit maps in turn:
// the one made while a row is summed was last read two rows before.
// Reads 2 and writes 2 bytes a bfloat16 logit, of which it reaches 5.0 TB/s:
// 16,972 rows of 151,936 logits with 64 entries, 15,193 of them counting, 1,950
// to 1,980 us; 512 rows of 32,000 float32 logits with 20 entries 24.7. With up to 64 entries
// the extra wave keeps pace with the others; with 65 to 256 a lane has up to 4
// and the row waits for them (4,096 rows of 151,936: 64 entries 534 us, 65 581,
// 256 706), the more so as 12 to 41 of its registers are spilled to scratch. Two of
// the smaller workgroups then share a compute unit only where the launch bound asks
// for it: 512 rows of 50,257 bfloat16 logits with 256 entries 34.6 us, without it
// 41.6.
template <typename Tin, int DW, int NR, int KE>
__global__ __launch_bounds__((DW + 1) * kWave, 4) void distill_row_kernel(DistillArgs a, double* term) {
  constexpr int VEC = Elem<Tin>::kVec, NT = DW * kWave, MOST = NR * NT;  // vectors
  __shared__ RowSum sh_sum[DW];
  __shared__ float sh_A, sh_c, sh_k;
  __shared__ int32_t rows_on[kListed], rows_off[kListed];
  __shared__ uint32_t sh_n[DW + 1];
  __shared__ uint64_t marks[3][MOST / 64 + 1];
  __shared__ alignas(16) uint32_t elements[(MOST + 16) / 4];  // a byte a vector: its entries' elements; then both ends
  static_assert(DW < kWave && NR <= kWave, "one wave merges the waves; a lane reads a bit map's word");
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
  const int32_t V = a.rows.V;
  const int64_t n = a.rows.n_rows, G = gridDim.x;
  const RowDeal deal = deal_rows<DW + 1>(a.rows.weight, n, G, rows_on, rows_off, sh_n);
  const bool listed = deal.listed;
  const int64_t turns = listed ? deal.n_on : n > blockIdx.x ? (n - blockIdx.x - 1) / G + 1 : 0;
  const int64_t turns_off = listed ? deal.n_off : turns;
  auto row_of = [&](const int32_t* list, int64_t k) -> int64_t {
    return listed ? static_cast<int64_t>(__builtin_amdgcn_readfirstlane(list[k])) : blockIdx.x + k * G;
  };
  // The first turn from k on whose row counts (without lists the others are passed over).
  auto next_turn = [&](int64_t k) {
    while (!listed && k < turns && a.rows.weight[row_of(rows_on, k)] == 0.0f) ++k;
    return k;
  };

  if (wave == DW) {
    auto load = [&](int64_t r, Held<KE>& e) {
      e.bad = 0;
#pragma unroll
      for (int i = 0; i < KE; ++i) {
        const Entry x = load_entry(a, r, lane + i * kWave);
        e.id[i] = x.id;
        e.logq[i] = x.logq;
        e.bad |= x.bad;
      }
    };
    auto mark = [&](int64_t r, Held<KE>& e, uint64_t* map) {
      const RowView<Tin> x(a.rows, r);
      const int32_t h = x.h, nvec = x.nvec, tail = x.tail();
      for (int32_t i = lane; i * 16 < nvec + 2; i += kWave) reinterpret_cast<vec4u*>(elements)[i] = vec4u{0, 0, 0, 0};
      for (int32_t i = lane; i * 64 < nvec; i += kWave) map[i] = 0;
      wave_lds_fence();
#pragma unroll
      for (int i = 0; i < KE; ++i) {
        if (e.id[i] < 0) continue;
        const Group g = group_of<Tin>(e.id[i], h, tail, V);
        const uint32_t slot = group_slot(g, nvec), bit = 1u << (slot % 4 * 8 + static_cast<uint32_t>(e.id[i] - g.base));
        if (atomicOr(&elements[slot / 4], bit) & bit) e.bad |= PR_FLAG_BAD_ID;
        if (g.vec >= 0) atomicOr(reinterpret_cast<uint32_t*>(map) + g.vec / 32, 1u << g.vec % 32);
      }
      wave_lds_fence();
      const uint8_t* byte = reinterpret_cast<const uint8_t*>(elements);
#pragma unroll
      for (int i = 0; i < KE; ++i)
        e.mine[i] = e.id[i] < 0 ? 0 : byte[group_slot(group_of<Tin>(e.id[i], h, tail, V), nvec)];
      e.ends = byte[nvec] | static_cast<uint32_t>(byte[nvec + 1]) << 8;
      wave_lds_fence();
    };
    Held<KE> e;
    int64_t k = next_turn(0);
    if (k < turns) {
      load(row_of(rows_on, k), e);
      mark(row_of(rows_on, k), e, marks[0]);
    }
    __syncthreads();
    for (int done = 0; k < turns; ++done) {
      const int64_t r = row_of(rows_on, k);
      const RowView<Tin> x(a.rows, r);
      const int32_t h = x.h, tail = x.tail();
      const float T = a.rows.temperature[r], c = scale_of(T), w = a.rows.weight[r];
      const int32_t s = scalar_element(lane, h, tail, V);
      const float zs = s < V ? Elem<Tin>::load1(x.row, s) : -INFINITY;
      const bool scalar = s < V && !(e.ends >> lane & 1u);  // no entry's
      float z[KE];
      vec4u v[KE];
#pragma unroll
      for (int i = 0; i < KE; ++i) {
        z[i] = -INFINITY;
        v[i] = neg_inf_vec<Tin>();
        if (e.id[i] < 0) continue;
        z[i] = Elem<Tin>::load1(x.row, e.id[i]);
        const Group g = group_of<Tin>(e.id[i], h, tail, V);
        // The entry of a group's first token takes the group's other elements.
        const uint32_t below = (1u << (e.id[i] - g.base)) - 1u;
        if (g.vec >= 0 && !(e.mine[i] & below)) v[i] = *x.in(g.vec, 0);
        else e.mine[i] = ~0u;
      }
      // The next row's entries, while this one is on its way.
      const int64_t k_next = next_turn(k + 1);
      Held<KE> e_next;
      if (k_next < turns) {
        load(row_of(rows_on, k_next), e_next);
        mark(row_of(rows_on, k_next), e_next, marks[(done + 1) % 3]);
      }
      LaneSum<false> in, out;
      out.add1(scalar ? zs : -INFINITY, c);
      EntrySums sums{0.0, 0.0};
      double q_of[KE];
#pragma unroll
      for (int i = 0; i < KE; ++i) {
        in.add1(z[i], c);
        float other[VEC];
        Elem<Tin>::unpack(v[i], other);
#pragma unroll
        for (int u = 0; u < VEC; ++u) other[u] = e.mine[i] >> u & 1u ? -INFINITY : other[u];
        out.add(other, c);
        // A probability of 0 adds nothing, whatever the student makes of its token.
        q_of[i] = e.id[i] >= 0 ? exp(static_cast<double>(e.logq[i])) : 0.0;
        sums.Q += q_of[i];
      }
      const float from = entry_ref(RowSum{in.mw, 0.0f});
#pragma unroll
      for (int i = 0; i < KE; ++i)
        if (q_of[i] > 0.0)
          sums.cross += q_of[i] * (static_cast<double>(e.logq[i]) -
                                   (static_cast<double>(z[i]) - static_cast<double>(from)) / static_cast<double>(T));
      sums.Q = wave_sum_d(sums.Q);
      sums.cross = wave_sum_d(sums.cross);
      const RowSum sum_in{in.mw, wave_sum(in.s)}, own{out.mw, wave_sum(out.s)};
      const uint32_t bad = (__any(e.bad & PR_FLAG_BAD_ID) ? PR_FLAG_BAD_ID : 0u) |
                           (__any(e.bad & PR_FLAG_NONFINITE) ? PR_FLAG_NONFINITE : 0u);
      __syncthreads();
      RowSum part{-INFINITY, 0.0f};
      if (lane < DW) part = sh_sum[lane];
      if (lane == DW) part = own;
      const RowSum sum_out = merge_lanes(part, c);
      RowLoss loss;
      loss.flags = row_flags(sum_in, sum_out, bad, T);
      const RowDistill q = row_factors(a, sum_in, sum_out, sums.Q, loss.flags, T, c, w);
      if (lane == 0) {
        sh_A = q.A;
        sh_c = q.c;
        sh_k = q.k;
      }
      __syncthreads();
      row_terms(a, sum_in, sum_out, sums, T, c, loss);
      if (lane == 0) {
        write_row(a, r, loss);
        term[r] = static_cast<double>(w) * loss.loss;
      }
      if (scalar) GradVec<Tin>::store1(x.out, s, q.k * fast_exp2(fmaf(zs, q.c, -q.A)));
#pragma unroll
      for (int i = 0; i < KE; ++i) {
        if (e.id[i] < 0) continue;
        GradVec<Tin>::store1(x.out, e.id[i], q.in_entry(z[i], q_of[i]));
        float other[VEC];
        Elem<Tin>::unpack(v[i], other);
        const int32_t base = group_of<Tin>(e.id[i], h, tail, V).base;
#pragma unroll
        for (int u = 0; u < VEC; ++u)
          if (!(e.mine[i] >> u & 1u))
            GradVec<Tin>::store1(x.out, base + u, q.k * fast_exp2(fmaf(other[u], q.c, -q.A)));
      }
      k = k_next;
      e = e_next;
    }
    for (int64_t i = 0; i < turns_off; ++i) {
      const int64_t r = row_of(rows_off, i);
      if (a.rows.weight[r] != 0.0f) continue;
      const RowView<Tin> x(a.rows, r);
      const int32_t s = scalar_element(lane, x.h, x.tail(), V);
      if (lane == 0) {
        write_row(a, r, masked_row());
        term[r] = 0.0;
      }
      if (s < V) GradVec<Tin>::store1(x.out, s, 0.0f);
    }
    return;
  }

  const int t = threadIdx.x;  // below NT
  int64_t k = next_turn(0);
  float T_next = k < turns ? a.rows.temperature[row_of(rows_on, k)] : 1.0f;
  __syncthreads();
  for (int done = 0; k < turns; ++done) {
    const int64_t r = row_of(rows_on, k);
    const float c = scale_of(T_next);
    const RowView<Tin> x(a.rows, r);
    // Every lane loads for every u, past the row's end a vector of the row
    // again, so that the loads in flight are always as many and a wave can
    // wait for one after the other. (Held rows have vectors.)
    auto place = [&](int u) {
      const int32_t at = u * NT < x.nvec ? u * NT : 0;
      return x.in(at, static_cast<uint32_t>(min(t, x.nvec - 1 - at)));
    };
    vec4u v[NR];
#pragma unroll
    for (int u = 0; u < NR; ++u) v[u] = *place(u);
    // Which of the wave's vectors u are the entries': a word of the bit map.
    const uint64_t words = lane < NR && (lane * DW + wave) * 64 < x.nvec ? marks[done % 3][lane * DW + wave] : 0;
    auto marked = [&](int u) {
      const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(words), u));
      const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(words >> 32), u));
      return static_cast<uint64_t>(hi) << 32 | lo;
    };
    LaneSum<false> L;
#pragma unroll
    for (int u = 0; u < NR; ++u)
      if (u * NT < x.nvec) {
        vec4u p = v[u];
        if ((u + 1) * NT > x.nvec && t >= x.nvec - u * NT) p = neg_inf_vec<Tin>();
        const uint64_t m = marked(u);
        if (m != 0 && m >> lane & 1u) p = neg_inf_vec<Tin>();
        float z[VEC];
        Elem<Tin>::unpack(p, z);
        L.add(z, c);
        __builtin_amdgcn_sched_barrier(0);
      }
    const float S = wave_sum(L.s);
    if (lane == 0) sh_sum[wave] = RowSum{L.mw, S};
    __syncthreads();
    k = next_turn(k + 1);
    __syncthreads();
    const float A = sh_A, cq = sh_c, kq = sh_k;
    if (k < turns) T_next = a.rows.temperature[row_of(rows_on, k)];
#pragma unroll
    for (int u = 0; u < NR; ++u) {
      forget(v[u]);
      const uint64_t m = marked(u);
      if (t < x.nvec - u * NT && !(m >> lane & 1u)) {
        float z[VEC];
        Elem<Tin>::unpack(v[u], z);
#pragma unroll
        for (int i = 0; i < VEC; ++i) z[i] = kq * fast_exp2(fmaf(z[i], cq, -A));
        store_grad(x.to(u * NT, t), GradVec<Tin>::pack(z));
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  for (int64_t i = 0; i < turns_off; ++i) {
    const int64_t r = row_of(rows_off, i);
    if (!listed && a.rows.weight[r] != 0.0f) continue;
    const RowView<Tin> x(a.rows, r);
    for (int32_t at = 0; at < x.nvec; at += NT)
      if (t < x.nvec - at) store_grad(x.to(at, t), vec4u{0, 0, 0, 0});
  }
}

template <typename Tin, int DW, int NR>
hipError_t launch_held(const DistillArgs& a, int64_t most, double* term, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(a.rows.n_rows < most ? a.rows.n_rows : most)), block((DW + 1) * kWave);
  if (a.k <= kWave)
    hipLaunchKernelGGL((distill_row_kernel<Tin, DW, NR, 1>), grid, block, 0, stream, a, term);
  else
    hipLaunchKernelGGL((distill_row_kernel<Tin, DW, NR, kMaxTop / kWave>), grid, block, 0, stream, a, term);
  return hipGetLastError();
}

// Shared memory that distill_stats_kernel asks for and does not use, so that no
// more than 5 of its workgroups share a compute unit: where many rows do not
// count, those that do are dealt out more evenly. 1,045 counting of 2,048 rows of
// 262,144 float32 logits: 205 us, without it 224.
constexpr unsigned kUnusedLds = 20000;

// Whether rows are held in a workgroup's registers. Shorter ones than for the
// policy loss are, as the pass that sums rows and puts their entries in order
// costs more here. 600 MB of rows, held and in two passes, with 20, 64 and 256
// entries (us, in brackets a row's vectors): bfloat16 4,096 logits a row (512)
// 1,098 and 999, 1,120 and 1,538, 2,437 and 4,540; 8,192 (1,024) 683 and 614,
// 713 and 871, 1,430 and 2,334; 12,000 (1,500) 510 and 516, 542 and 682, 1,062
// and 1,657; 16,384 (2,048) 397 and 435, 427 and 552, 829 and 1,256; 32,000 270
// and 370, 289 and 431, 508 and 764; float32 4,096 619 and 585, 648 and 836,
// 1,081 and 2,240; 16,000 255 and 354, 267 and 425, 405 and 758. 2,048 rows of
// 4,096 bfloat16 logits: 35 and 41, 34 and 58, 67 and 149.
constexpr int64_t kLeastHeld = 512, kLeastHeldFewEntries = 1500, kFewEntries = 32, kManyRows = 8192;
bool held(int64_t n_rows, int64_t nvec, int32_t k) {
  const bool short_rows = nvec < kLeastHeldFewEntries && k <= kFewEntries && n_rows >= kManyRows;
  return nvec >= kLeastHeld && nvec <= kRowVectors && !short_rows;
}

// Workgroups per row for a shape (0: rows are not split). Few rows that could be
// held are spread over the device as long as that is faster. Spread and held, 20
// and 256 entries (us): 16,384 bfloat16 logits (2,048 vectors) 48 rows 11.0 and
// 11.2, 12.5 and 17.1, 128 rows 14.8 and 11.7, 16.7 and 17.6; 50,257 of them
// (6,282) 8 rows 12.9 and 14.2, 13.7 and 19.0, 32 rows 15.0 and 14.7, 15.7 and
// 19.4; 32,000 float32 logits (8,000) 4 rows 12.6 and 12.6, 13.6 and 15.9, 32
// rows 16.2 and 13.2, 17.2 and 16.6; the larger size: 40,000 float32 logits
// (10,000) 24 rows 14.6 and 14.7, 15.3 and 18.4, 32 rows 17.7 and 14.9, 18.6 and
// 18.5; 151,936 bfloat16 logits (18,992) 48 rows 24.7 and 26.5, 26.8 and 31.2,
// 64 rows 29.3 and 27.4, 31.2 and 32.3.
int distill_split(int64_t n_rows, int32_t V, pr_dtype dtype, bool grad, int32_t k) {
  if (n_rows <= 0 || n_rows >= kSplitRows) return 0;
  const int64_t nvec = V / (dtype == PR_BF16 ? 8 : 4);
  const bool few = nvec <= kSmallRowVectors ? n_rows * nvec <= (k <= kWave ? 100000 : 250000)
                                            : n_rows <= nvec / 400;
  return grad && held(n_rows, nvec, k) && !few ? 0 : row_parts(n_rows, V, dtype);
}

constexpr int64_t kMostGroups = int64_t{1} << 23;  // a grid holds less than 2^32 threads

template <typename Tin>
int64_t grad_parts(int32_t V) {
  const int64_t nvec = V / Elem<Tin>::kVec;
  return nvec > 0 ? (nvec + kGradBlock - 1) / kGradBlock : 1;
}

// The workspace: the rows' gradient factors, then their terms of the loss and
// their sorted entries or, where they are split, their parts.
template <typename Tin>
hipError_t distill(const DistillArgs& a, hipStream_t stream) {
  const int64_t n = a.rows.n_rows;
  const pr_dtype dtype = sizeof(Tin) == 2 ? PR_BF16 : PR_F32;
  RowDistill* rd = static_cast<RowDistill*>(a.ws);
  double* term = reinterpret_cast<double*>(rd + n);
  const int64_t nvec = a.rows.V / Elem<Tin>::kVec, parts = grad_parts<Tin>(a.rows.V);
  const int G = distill_split(n, a.rows.V, dtype, a.rows.grad != nullptr, a.k);
  hipError_t e = hipSuccess;
  if (G > 0) {
    DistillPart* part = reinterpret_cast<DistillPart*>(rd + n);
    hipLaunchKernelGGL(distill_parts_kernel<Tin>, dim3(static_cast<unsigned>(n * G)), dim3(kStatsBlock), 0, stream, a,
                       part, G);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 grid(static_cast<unsigned>(parts), static_cast<unsigned>(n));
    if (a.rows.grad && n * parts <= kFewGroups) {
      hipLaunchKernelGGL(distill_parts_grad_kernel<Tin>, dim3(grid.x, grid.y + 1), dim3(kGradBlock), 0, stream, a,
                         part, G);
      return hipGetLastError();
    }
    hipLaunchKernelGGL(distill_finish_kernel, dim3(1), dim3(kGradBlock), 0, stream, a, part, G,
                       a.rows.grad ? rd : nullptr);
    e = hipGetLastError();
    if (e != hipSuccess || !a.rows.grad) return e;
    hipLaunchKernelGGL(distill_grad_kernel<Tin>, grid, dim3(kGradBlock), 0, stream, a, rd);
    return hipGetLastError();
  }
  if (n > 0 && a.rows.grad && held(n, nvec, a.k)) {
    e = nvec <= kSmallRowVectors ? launch_held<Tin, 7, 19>(a, 2 * kCUs, term, stream)
                                 : launch_held<Tin, 15, 20>(a, kCUs, term, stream);
  } else {
    SortedRows sorted{nullptr, nullptr, static_cast<int32_t>(parts)};
    if (a.rows.grad) {
      sorted.entry = reinterpret_cast<SortedEntry*>(term + n);
      sorted.begin = reinterpret_cast<int32_t*>(sorted.entry + n * a.k);
    }
    for (int64_t at = 0; at < n && e == hipSuccess; at += kMostGroups) {
      const int64_t rows = n - at < kMostGroups ? n - at : kMostGroups;
      hipLaunchKernelGGL(distill_stats_kernel<Tin>, dim3(static_cast<unsigned>(rows)), dim3(kStatsBlock), kUnusedLds,
                         stream, a, term, rd, sorted, at);
      e = hipGetLastError();
    }
    constexpr int64_t kMostY = 32768;
    for (int64_t at = 0; a.rows.grad && at < n && e == hipSuccess; at += kMostY) {
      const int64_t rows = n - at < kMostY ? n - at : kMostY;
      hipLaunchKernelGGL(distill_sorted_grad_kernel<Tin>,
                         dim3(static_cast<unsigned>(parts), static_cast<unsigned>(rows)), dim3(kGradBlock), 0, stream,
                         a, rd, sorted, at);
      e = hipGetLastError();
    }
  }
  return e == hipSuccess ? launch_loss_sum(term, n, 1.0, a.loss, stream) : e;
}

}  // namespace

size_t distill_workspace_bytes(int64_t n_rows, int32_t V, pr_dtype dtype, int32_t k) {
  const size_t n = n_rows < 0 ? 0 : static_cast<size_t>(n_rows), entries = k < 0 ? 0 : static_cast<size_t>(k);
  const size_t most = static_cast<size_t>(std::max(distill_split(n_rows, V, dtype, true, k),
                                                   distill_split(n_rows, V, dtype, false, k)));
  const size_t parts = static_cast<size_t>(dtype == PR_BF16 ? grad_parts<uint16_t>(V) : grad_parts<float>(V));
  size_t rows = n * sizeof(double);
  if (!held(n_rows, V / (dtype == PR_BF16 ? 8 : 4), k))
    rows += n * (entries * sizeof(SortedEntry) + (parts + 1) * sizeof(int32_t));
  return n * sizeof(RowDistill) + std::max(n * most * sizeof(DistillPart), rows);
}

hipError_t launch_distill(const DistillArgs& a, pr_dtype dtype, hipStream_t stream) {
  return dtype == PR_BF16 ? distill<uint16_t>(a, stream) : distill<float>(a, stream);
}

}  // namespace pr
