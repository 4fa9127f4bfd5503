// Losses over logit rows and their gradients in the logits: the clipped
// policy loss with a KL term and the preference loss over pairs of requests.
//
// With u = z / T, l = u_y - log sum exp(u), both losses are functions of the
// rows' l, and a row's gradient is
//   dloss/dz_v = (dloss/dl) / T * (delta_vy - softmax(u)_v),
// which takes a row's logits twice: for its sum of exps, then for its gradient.
//
// A policy row's dloss/dl is its own, so a workgroup that can hold the row
// reads it once (policy_row_kernel). A preference row's depends on every row
// of its pair, so its logits are read twice (preference_stats_kernel,
// preference_pair_kernel, grad_kernel), as are policy rows too short or too
// long to be held (policy_stats_kernel, grad_kernel). Few rows are spread over
// the device (parts_kernel and what follows it). All are bound by memory.
//
// Exponents are in base 2: with c = log2(e) / T and the row's reference
// A = round(m c), m its largest logit (row_ref, which gives c and A also where m
// is far from zero), x_v = fma(z_v, c, -A) and S = sum 2^x_v,
// softmax(u)_v = 2^x_v / S. A row's sums over the vocabulary
// are float32 per lane, all terms positive: at most 160 of them in a held row;
// elsewhere a lane takes V / (256 G) and compensates its sum. What follows per
// row (l, the loss's term, the coefficient) and the sums over rows are in 64
// bits; the ratio and 1 - p_y have the precision of float32
// exponentials of 64-bit arguments (in 64 bits they took registers that hold
// the row). A gradient element is rounded to its type once.
#include "loss.h"
#include "held_rows.h"

namespace pr {
namespace {

constexpr int kStatsBlock = 256;
constexpr int kGradBlock = 512;
constexpr int kSumBlock = 1024;

// What the gradient pass needs of a row: dz_v = k 2^fma(z_v, c, -A) for every
// v but y, whose element is gy. k = gy = 0: the row's gradient is zero.
struct alignas(16) RowGrad {
  float A, c, k, gy;
};

struct RowValue {
  double l;
  float A, c;      // of the row's reference
  uint32_t flags;  // 0 or the reasons why l is NaN
};

// l of a row from its sum of exps, in 64 bits. S is relative to A, the rounded
// product of m and the reference's c, whose exact residual goes off its logarithm.
__device__ __forceinline__ RowValue row_value(const RowSum& p, float T, float c, int32_t y, int32_t V, float zy) {
  RowValue v;
  const RowRef ref = row_ref(p.m, c);
  v.A = ref.A;
  v.c = ref.c;
  v.flags = 0;
  if (!temperature_ok(T)) v.flags |= PR_FLAG_BAD_TP;
  if (!(fabsf(p.S) < INFINITY) || p.m == INFINITY || p.m == -INFINITY) v.flags |= PR_FLAG_NONFINITE;
  if (!v.flags && fabsf(p.m) > ldexpf(T, 100)) v.flags |= PR_FLAG_BAD_TP;
  if (y < 0 || y >= V) v.flags |= PR_FLAG_BAD_ID;
  if (v.flags) {
    v.l = __longlong_as_double(0x7ff8000000000000ll);
    return v;
  }
  const double delta = static_cast<double>(fmaf(p.m, v.c, -v.A));
  const double lnS = log(static_cast<double>(p.S)) - delta * 0.69314718055994530942;
  v.l = (static_cast<double>(zy) - static_cast<double>(p.m)) / static_cast<double>(T) - lnS;
  return v;
}

// The gradient's factors of a row from coef = dloss/dl / T. 1 - p_y is
// -expm1(l), which keeps its precision when p_y is near 1.
__device__ __forceinline__ RowGrad row_grad(double coef, double l, float A, float c, float S) {
  if (coef == 0.0) return RowGrad{A, c, 0.0f, 0.0f};
  if (!(coef == coef)) {
    const float nan = __uint_as_float(0x7fc00000u);
    return RowGrad{0.0f, 0.0f, nan, nan};
  }
  return RowGrad{A, c, static_cast<float>(-coef / static_cast<double>(S)),
                 static_cast<float>(-coef) * expm1f(static_cast<float>(l))};
}

template <typename Tin>
__device__ __forceinline__ float token_logit(const LossRows& a, int64_t r, int32_t y) {
  return y >= 0 && y < a.V ? Elem<Tin>::load1(row_ptr<Tin>(a, r), y) : 0.0f;
}

// exp(x) with the range of 64 bits and the precision of 32, so that a ratio
// beyond float32 times an advantage of 0 is 0.
__device__ __forceinline__ double exp_wide(double x) {
  const double t = x * 1.4426950408889634, k = fmin(fmax(rint(t), -2000.0), 2000.0);
  return ldexp(static_cast<double>(exp2f(static_cast<float>(t - k))), static_cast<int>(k));
}

// What the policy loss makes of a row.
struct PolicyRow {
  double term;  // of the loss
  float logprob, ratio, kl;
  uint32_t flags;
  RowGrad grad;
};

__device__ __forceinline__ PolicyRow policy_row(const PolicyArgs& a, int64_t r, const RowValue& v, float T, float S,
                                                float w) {
  const double A = a.advantage[r], ratio = exp_wide(v.l - static_cast<double>(a.old_logprob[r]));
  const double free = ratio * A, held = fmin(fmax(ratio, a.clip_lo), a.clip_hi) * A;
  const bool clipped = free > held;
  double kl = 0.0, rise = 0.0;
  if (a.ref_logprob) {
    const double d = static_cast<double>(a.ref_logprob[r]) - v.l;
    rise = expm1(d);
    kl = d == INFINITY ? d : rise - d;  // a token of probability 0
  }
  const bool with_kl = a.kl_coef > 0.0;  // without, an infinite KL stands beside the loss alone
  const double gain = v.flags ? v.l : (clipped ? held : free);
  const double dl = static_cast<double>(w) * ((clipped ? 0.0 : -free) - (with_kl ? a.kl_coef * rise : 0.0));
  PolicyRow p;
  p.term = static_cast<double>(w) * ((with_kl ? a.kl_coef * kl : 0.0) - gain);
  p.logprob = static_cast<float>(v.l);
  p.ratio = static_cast<float>(ratio);
  p.kl = static_cast<float>(kl);
  p.flags = v.flags | (!v.flags && clipped ? PR_FLAG_CLIPPED : 0u);
  p.grad = row_grad(v.flags ? v.l : a.grad_scale * dl / static_cast<double>(T), v.l, v.A, v.c, S);
  return p;
}

__device__ __forceinline__ PolicyRow policy_masked() {
  return PolicyRow{0.0, 0.0f, 0.0f, 0.0f, PR_FLAG_MASKED, RowGrad{0.0f, 0.0f, 0.0f, 0.0f}};
}

__device__ __forceinline__ void policy_write(const PolicyArgs& a, int64_t r, const PolicyRow& p) {
  if (a.out.logprob) a.out.logprob[r] = p.logprob;
  if (a.out.ratio) a.out.ratio[r] = p.ratio;
  if (a.out.kl) a.out.kl[r] = p.kl;
  if (a.out.flags) a.out.flags[r] = p.flags;
}

// Sums by one workgroup, in a fixed order (valid in thread 0): of its
// threads' values, and of v[0..n).
__device__ __forceinline__ double block_total(double s) {
  __shared__ double sh[kSumBlock / kWave];
  s = wave_sum_d(s);
  if (threadIdx.x % kWave == 0) sh[threadIdx.x / kWave] = s;
  __syncthreads();
  double t = 0.0;
  if (threadIdx.x == 0)
    for (int w = 0; w < static_cast<int>(blockDim.x) / kWave; ++w) t += sh[w];
  return t;
}
__device__ __forceinline__ double block_sum(const double* v, int64_t n) {
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += blockDim.x) s += v[i];
  return block_total(s);
}

// loss = (sum of v) / over. One workgroup's chain of reads bounds it: 512
// values 3.9 us, 16,972 9.4.
__global__ __launch_bounds__(kSumBlock) void loss_sum_kernel(const double* v, int64_t n, double over, float* loss) {
  const double s = block_sum(v, n);
  if (threadIdx.x == 0) loss[0] = static_cast<float>(s / over);
}

// The sums of the rows' stretches, G of them a row, and each row's token's
// logit, for kernels that read it while the gradient takes the logits' place.
template <typename Tin>
__global__ __launch_bounds__(kStatsBlock) void parts_kernel(LossRows a, RowSum* part, float* zy, int32_t G) {
  const int64_t r = blockIdx.x / G;
  const int g = blockIdx.x % G;
  if (a.weight[r] == 0.0f) return;
  if (threadIdx.x == 0 && g == 0) zy[r] = token_logit<Tin>(a, r, a.ids[r]);
  const RowSum p = stretch_sum<Tin, kStatsBlock>(row_ptr<Tin>(a, r), a.V, g, G, scale_of(a.temperature[r]));
  if (threadIdx.x == 0) part[r * G + g] = p;
}

// Workgroups of a launch of kStatsBlock or kPairBlock threads: a grid holds
// less than 2^32 threads, so longer lists of rows or pairs take several.
constexpr int64_t kMostGroups = int64_t{1} << 23;

// One workgroup per row: its sum of exps, then everything but its gradient.
// The read bounds it: 912 counting of 2,048 rows of 262,144 float32 logits
// take 166 us (0.96 GB, 5.8 TB/s).
template <typename Tin>
__global__ __launch_bounds__(kStatsBlock) void policy_stats_kernel(PolicyArgs a, RowGrad* rg, int64_t first) {
  const int64_t r = first + blockIdx.x;
  const float w = a.rows.weight[r];
  PolicyRow p = policy_masked();
  if (w != 0.0f) {
    const float T = a.rows.temperature[r], c = scale_of(T);
    const int32_t y = a.rows.ids[r];
    const float zy = token_logit<Tin>(a.rows, r, y);
    const RowSum s = stretch_sum<Tin, kStatsBlock>(row_ptr<Tin>(a.rows, r), a.rows.V, 0, 1, c);
    if (threadIdx.x != 0) return;
    p = policy_row(a, r, row_value(s, T, c, y, a.rows.V, zy), T, s.S, w);
  } else if (threadIdx.x != 0) {
    return;
  }
  policy_write(a, r, p);
  a.row_loss[r] = p.term;
  rg[r] = p.grad;
}

__device__ __forceinline__ float grad_of(float z, const RowGrad& q) { return q.k * fast_exp2(fmaf(z, q.c, -q.A)); }

// The gradient of a stretch of a row, a vector per thread of workgroup `part`:
// short workgroups in memory order, past the caches, are what reads and
// writes fastest at once here. 13,260 of 16,972 rows of 151,936 bfloat16
// logits: 1,485 us (9.2 GB, 6.2 TB/s); 256 threads of eight vectors each took
// 1,785. Each element is read and written by one thread, so the gradient may take the
// logits' place.
template <typename Tin>
__device__ __forceinline__ void grad_stretch(const LossRows& a, int64_t r, int32_t part, const RowGrad& q) {
  constexpr int VEC = Elem<Tin>::kVec;
  const Tin* row = row_ptr<Tin>(a, r);
  Tin* out = static_cast<Tin*>(a.grad) + r * a.grad_stride;
  const int32_t h = static_cast<int32_t>(head_elems<Tin>(row, a.V)), nvec = (a.V - h) / VEC, tail = h + nvec * VEC;
  const int t = threadIdx.x;
  const int32_t y = a.ids[r];
  const bool zero = q.k == 0.0f && q.gy == 0.0f;
  if (part == 0 && t < 16) {
    const int32_t e = scalar_element(t, h, tail, a.V);
    if (e < a.V) GradVec<Tin>::store1(out, e, zero ? 0.0f : e == y ? q.gy : grad_of(Elem<Tin>::load1(row, e), q));
  }
  const int32_t j = part * kGradBlock + t;
  if (j >= nvec) return;
  vec4u g{0, 0, 0, 0};
  if (!zero) {
    float z[VEC];
    Elem<Tin>::unpack(__builtin_nontemporal_load(reinterpret_cast<const vec4u*>(row + h) + j), z);
#pragma unroll
    for (int k = 0; k < VEC; ++k) z[k] = grad_of(z[k], q);
    const int32_t at = y - (h + j * VEC);
    if (at >= 0 && at < VEC) {
#pragma unroll
      for (int k = 0; k < VEC; ++k) z[k] = k == at ? q.gy : z[k];
    }
    g = GradVec<Tin>::pack(z);
  }
  stream_grad(out + h + static_cast<int64_t>(j) * VEC, g);
}

// The gradients of the rows from `first` on (blockIdx.y). With n_sum > 0 the
// grid has a row more, whose first wave takes the loss that waits for the
// kernel before this one: the mean of `sum`'s values.
template <typename Tin>
__global__ __launch_bounds__(kGradBlock) void grad_kernel(LossRows a, const RowGrad* rg, int64_t first,
                                                          const double* sum, int32_t n_sum, float* loss) {
  const int64_t r = first + blockIdx.y;
  if (r == a.n_rows) {
    if (blockIdx.x > 0 || threadIdx.x >= kWave) return;
    double s = 0.0;
    for (int32_t i = threadIdx.x; i < n_sum; i += kWave) s += sum[i];
    s = wave_sum_d(s);
    if (threadIdx.x == 0) loss[0] = static_cast<float>(s / n_sum);
    return;
  }
  grad_stretch<Tin>(a, r, blockIdx.x, rg[r]);
}

// A split row's policy loss from its parts. The logits are not read: they
// may be giving way to the gradient.
__device__ __forceinline__ PolicyRow policy_from_parts(const PolicyArgs& a, int64_t r, const RowSum* part,
                                                       const float* zy) {
  const float w = a.rows.weight[r];
  if (w == 0.0f) return policy_masked();
  const float T = a.rows.temperature[r], c = scale_of(T), z = zy[r];
  const int32_t y = a.rows.ids[r];
  const RowSum s = merge_parts(part + r * a.G, a.G, c);
  return policy_row(a, r, row_value(s, T, c, y, a.rows.V, z), T, s.S, w);
}

// All split rows' outputs, gradient factors (rg NULL: not wanted) and the
// loss, by one workgroup.
__device__ __forceinline__ void policy_finish(const PolicyArgs& a, const RowSum* part, const float* zy, RowGrad* rg) {
  double sum = 0.0;
  for (int64_t r = threadIdx.x; r < a.rows.n_rows; r += kGradBlock) {
    const PolicyRow p = policy_from_parts(a, r, part, zy);
    policy_write(a, r, p);
    if (rg) rg[r] = p.grad;
    sum += p.term;
  }
  sum = block_total(sum);
  if (threadIdx.x == 0) a.loss[0] = static_cast<float>(sum);
}

__global__ __launch_bounds__(kGradBlock) void policy_finish_kernel(PolicyArgs a, const RowSum* part, const float* zy,
                                                                  RowGrad* rg) {
  policy_finish(a, part, zy, rg);
}

// The gradients of a few split rows: each workgroup works out its own row's
// factors instead of waiting for a kernel that does. The first workgroup of
// the grid's last row finishes the rows.
template <typename Tin>
__global__ __launch_bounds__(kGradBlock) void policy_parts_kernel(PolicyArgs a, const RowSum* part, const float* zy) {
  if (blockIdx.y + 1 < gridDim.y)
    grad_stretch<Tin>(a.rows, blockIdx.y, blockIdx.x, policy_from_parts(a, blockIdx.y, part, zy).grad);
  else if (blockIdx.x == 0)
    policy_finish(a, part, zy, nullptr);
}

// The policy loss of a row and its gradient in one read of the row.
//
// A workgroup keeps the row in registers between its sum and its gradient, NR
// vectors in each thread of its first DW waves, and adds each vector to its
// sums as it arrives. One more wave takes what is scalar in a row (its inputs,
// the elements outside the vectors, the loss in 64 bits): the registers for
// that are not taken from those that hold the row.
//
// The grid is the workgroups that run at once. Memory serves loads and stores
// best when they do not mix, and workgroups that start together and do the
// same stay together: so the rows that count are dealt out by their rank
// among those that do, and the zero gradients of the others are written last
// (written first: 1,818 us against 1,752). 13,260 of 16,972 rows of 151,936
// bfloat16 logits: 1,742 us (9.2 GB, 5.3 TB/s); a pass each for sums and
// gradients takes 616 + 1,485. Its reads and sums alone take 991: loads and
// stores of a compute unit take turns. Loads of the next row while a row is
// written made it 1,880 to 1,940. 512 rows of 32,000 float32 logits: 23 us.
template <typename Tin, int DW, int NR>
__global__ __launch_bounds__((DW + 1) * kWave) void policy_row_kernel(PolicyArgs a) {
  constexpr int VEC = Elem<Tin>::kVec, NT = DW * kWave;
  __shared__ RowSum sh_sum[DW];
  __shared__ RowGrad sh_q;
  __shared__ int32_t rows_on[kListed], rows_off[kListed];
  __shared__ uint32_t sh_n[DW + 1];
  static_assert(DW < kWave, "one wave merges the waves");
  const int lane = threadIdx.x % kWave;
  // As a scalar, so that what follows branches by wave and not by lane: both
  // branches pass the same barriers.
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
  const int32_t V = a.rows.V;
  const int64_t n = a.rows.n_rows, G = gridDim.x;

  const RowDeal deal = deal_rows<DW + 1>(a.rows.weight, n, G, rows_on, rows_off, sh_n);
  const bool listed = deal.listed;
  const uint32_t n_on = deal.n_on, n_off = deal.n_off;
  // A row for each workgroup, or too many to list: they are dealt out by row,
  // and the turn of a row that does not count is passed over.
  const int64_t turns = listed ? n_on : n > blockIdx.x ? (n - blockIdx.x - 1) / G + 1 : 0;
  const int64_t turns_off = listed ? n_off : turns;
  auto row_of = [&](const int32_t* list, int64_t k) -> int64_t {
    return listed ? static_cast<int64_t>(__builtin_amdgcn_readfirstlane(list[k])) : blockIdx.x + k * G;
  };

  if (wave == DW) {
    for (int64_t k = 0; k < turns; ++k) {
      const int64_t r = row_of(rows_on, k);
      const RowView<Tin> x(a.rows, r);
      const float w = a.rows.weight[r];
      if (w == 0.0f) continue;
      const int32_t e = scalar_element(lane, x.h, x.tail(), V);
      const float T = a.rows.temperature[r], c = scale_of(T);
      const int32_t y = a.rows.ids[r];
      const float zy = token_logit<Tin>(a.rows, r, y);
      const float z = e < V ? Elem<Tin>::load1(x.row, e) : -INFINITY;
      LaneSum<false> own;
      own.add1(z, c);
      const float S = wave_sum(own.s);
      __syncthreads();
      RowSum part{-INFINITY, 0.0f};
      if (lane < DW) part = sh_sum[lane];
      if (lane == DW) part = RowSum{own.mw, S};
      const RowSum sum = merge_lanes(part, c);
      const PolicyRow p = policy_row(a, r, row_value(sum, T, c, y, V, zy), T, sum.S, w);
      const RowGrad q = p.grad;
      if (lane == 0) sh_q = q;
      __syncthreads();
      if (lane == 0) {
        policy_write(a, r, p);
        a.row_loss[r] = p.term;
      }
      if (e < V) GradVec<Tin>::store1(x.out, e, e == y ? q.gy : grad_of(z, q));
    }
    for (int64_t k = 0; k < turns_off; ++k) {
      const int64_t r = row_of(rows_off, k);
      if (a.rows.weight[r] != 0.0f) continue;
      const RowView<Tin> x(a.rows, r);
      const int32_t e = scalar_element(lane, x.h, x.tail(), V);
      if (lane == 0) {
        policy_write(a, r, policy_masked());
        a.row_loss[r] = 0.0;
      }
      if (e < V) GradVec<Tin>::store1(x.out, e, 0.0f);
    }
    return;
  }

  const int t = threadIdx.x;  // below NT
  // A row's temperature and token are read a turn ahead: its loads return in
  // order, so what is read after the row's vectors arrives after them.
  int64_t r_next = turns > 0 ? row_of(rows_on, 0) : 0;
  float T_next = turns > 0 ? a.rows.temperature[r_next] : 1.0f;
  int32_t y_next = turns > 0 ? a.rows.ids[r_next] : 0;
  for (int64_t k = 0; k < turns; ++k) {
    const int64_t r = r_next;
    const float c = scale_of(T_next);
    const int32_t y = y_next;
    const bool more = k + 1 < turns;
    r_next = more ? row_of(rows_on, k + 1) : r;
    if (!listed && a.rows.weight[r] == 0.0f) {
      T_next = a.rows.temperature[r_next];
      y_next = a.rows.ids[r_next];
      continue;
    }
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
    // A lane's vector u, -inf past the row's end.
    auto within = [&](vec4u p, int u) {
      if ((u + 1) * NT > x.nvec && t >= x.nvec - u * NT) p = neg_inf_vec<Tin>();
      return p;
    };
    LaneSum<false> L;
    auto sum = [&](const vec4u& p) {
      float z[VEC];
      Elem<Tin>::unpack(p, z);
      L.add(z, c);
      __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int u = 0; u < NR; ++u)
      if (u * NT < x.nvec) sum(within(v[u], u));
    const float S = wave_sum(L.s);
    if (lane == 0) sh_sum[wave] = RowSum{L.mw, S};
    __syncthreads();
    __syncthreads();
    const RowGrad q = sh_q;
    T_next = a.rows.temperature[r_next];
    y_next = a.rows.ids[r_next];
    const int32_t jy = y >= x.h && y < x.tail() ? (y - x.h) / VEC : -1, ky = (y - x.h) % VEC;
    auto put = [&](const vec4u& p, int32_t at) {
      float z[VEC];
      Elem<Tin>::unpack(p, z);
#pragma unroll
      for (int i = 0; i < VEC; ++i) z[i] = grad_of(z[i], q);
      if (t == jy - at) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) z[i] = i == ky ? q.gy : z[i];
      }
      store_grad(x.to(at, t), GradVec<Tin>::pack(z));
      __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int u = 0; u < NR; ++u) {
      forget(v[u]);
      if (t < x.nvec - u * NT) put(v[u], u * NT);
    }
  }
  for (int64_t k = 0; k < turns_off; ++k) {
    const int64_t r = row_of(rows_off, k);
    if (!listed && a.rows.weight[r] != 0.0f) continue;
    const RowView<Tin> x(a.rows, r);
    for (int32_t at = 0; at < x.nvec; at += NT)
      if (t < x.nvec - at) store_grad(x.to(at, t), vec4u{0, 0, 0, 0});
  }
}

// Workgroups of the gradient pass along a row.
template <typename Tin>
int64_t grad_parts(int32_t V) {
  const int64_t nvec = V / Elem<Tin>::kVec;
  return nvec > 0 ? (nvec + kGradBlock - 1) / kGradBlock : 1;
}

template <typename Tin>
hipError_t launch_grad(const LossRows& a, const RowGrad* rg, hipStream_t stream, const double* sum = nullptr,
                       int32_t n_sum = 0, float* loss = nullptr) {
  constexpr int64_t kMostY = 32768;
  const int64_t parts = grad_parts<Tin>(a.V), total = a.n_rows + (n_sum > 0 ? 1 : 0);
  for (int64_t at = 0; at < total; at += kMostY) {
    const int64_t rows = total - at < kMostY ? total - at : kMostY;
    hipLaunchKernelGGL(grad_kernel<Tin>, dim3(static_cast<unsigned>(parts), static_cast<unsigned>(rows)),
                       dim3(kGradBlock), 0, stream, a, rg, at, sum, n_sum, loss);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// The preference loss of a row, first part: l and what its gradient needs.
__device__ __forceinline__ double preference_row(const PreferenceArgs& a, int64_t r, const RowSum& p, float T, float c,
                                                 int32_t y, float zy, double* l, RowGrad* rg) {
  const RowValue v = row_value(p, T, c, y, a.rows.V, zy);
  l[r] = v.l;
  rg[r] = RowGrad{v.A, v.c, p.S, T};
  if (a.out.logprob) a.out.logprob[r] = static_cast<float>(v.l);
  if (a.out.flags) a.out.flags[r] = v.flags;
  return v.l;
}

// A row's sum of exps, by G workgroups: 13,260 rows of 151,936 bfloat16 logits
// 616 us (4.0 GB, 6.5 TB/s).
template <typename Tin>
__global__ __launch_bounds__(kStatsBlock) void preference_stats_kernel(PreferenceArgs a, double* l, RowGrad* rg,
                                                                      RowSum* part, int64_t first) {
  const int64_t r = first + blockIdx.x / a.G;
  const int g = blockIdx.x % a.G;
  if (a.rows.weight[r] == 0.0f) {
    if (threadIdx.x == 0 && g == 0) {
      l[r] = 0.0;
      rg[r] = RowGrad{0.0f, 0.0f, 0.0f, 0.0f};
      if (a.out.logprob) a.out.logprob[r] = 0.0f;
      if (a.out.flags) a.out.flags[r] = PR_FLAG_MASKED;
    }
    return;
  }
  const float T = a.rows.temperature[r], c = scale_of(T);
  const int32_t y = a.rows.ids[r];
  const float zy = token_logit<Tin>(a.rows, r, y);
  const RowSum p = stretch_sum<Tin, kStatsBlock>(row_ptr<Tin>(a.rows, r), a.rows.V, g, a.G, c);
  if (threadIdx.x != 0) return;
  if (a.G > 1)
    part[r * a.G + g] = p;
  else
    preference_row(a, r, p, T, c, y, zy, l, rg);
}

// Most pairs whose mean one wave takes while the gradient is written. Beside it
// and in a launch of its own, two rows of 2,000 bfloat16 logits a pair: 32 pairs
// 10.7 and 12.5 us, 256 11.9 and 13.8, 512 15.7 and 16.4, 1,000 23.3 and 22.2,
// 4,096 67.9 and 57.5.
constexpr int32_t kPairsBeside = 512;

// One workgroup per pair: the sums over both requests, the pair's loss, and
// the gradient's factors of the pair's rows. Rows that were split finish here.
// A chain of a few dependent reads bounds it, 4 to 8 us.
constexpr int kPairBlock = 256;

__device__ __forceinline__ double softplus(double x) { return fmax(x, 0.0) + log1p(exp(-fabs(x))); }

template <typename Tin>
__global__ __launch_bounds__(kPairBlock) void preference_pair_kernel(PreferenceArgs a, double* l, RowGrad* rg,
                                                                    const RowSum* part, double* pair_loss,
                                                                    int32_t first) {
  __shared__ double sh[2][kPairBlock / kWave];
  const int64_t p = first + static_cast<int32_t>(blockIdx.x);
  int64_t off[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const int64_t o = a.offsets[2 * p + i];
    off[i] = o < 0 ? 0 : o > a.rows.n_rows ? a.rows.n_rows : o;
  }
  // The pair's rows, chosen request first.
  double q[2] = {0.0, 0.0};
  for (int64_t r = off[0] + threadIdx.x; r < off[2]; r += kPairBlock) {
    const float w = a.rows.weight[r];
    const float ref = a.ref_logprob ? a.ref_logprob[r] : 0.0f;
    double lr;
    if (a.G > 1) {
      if (w == 0.0f) continue;
      const int32_t y = a.rows.ids[r];
      const float T = a.rows.temperature[r], c = scale_of(T), zy = token_logit<Tin>(a.rows, r, y);
      const RowSum s = merge_parts(part + r * a.G, a.G, c);
      lr = preference_row(a, r, s, T, c, y, zy, l, rg);
    } else {
      lr = l[r];
    }
    if (w != 0.0f) q[r < off[1] ? 0 : 1] += static_cast<double>(w) * (lr - static_cast<double>(ref));
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    q[i] = wave_sum_d(q[i]);
    if (threadIdx.x % kWave == 0) sh[i][threadIdx.x / kWave] = q[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    q[i] = 0.0;
    for (int w = 0; w < kPairBlock / kWave; ++w) q[i] += sh[i][w];
  }
  const double h = a.beta * (q[0] - q[1]) - a.margin, s = a.label_smoothing;
  if (threadIdx.x == 0) {
    const double loss = (s < 1.0 ? (1.0 - s) * softplus(-h) : 0.0) + (s > 0.0 ? s * softplus(h) : 0.0);
    pair_loss[p] = loss;
    if (a.n_pairs == 1) a.loss[0] = static_cast<float>(loss);
    if (a.out.pair_loss) a.out.pair_loss[p] = static_cast<float>(loss);
    if (a.out.pair_logit) a.out.pair_logit[p] = static_cast<float>(h);
    if (a.out.seq_logratio) {
      a.out.seq_logratio[2 * p] = static_cast<float>(q[0]);
      a.out.seq_logratio[2 * p + 1] = static_cast<float>(q[1]);
    }
  }
  if (!a.rows.grad) return;
  // sigmoid(h) - 1 + s, without the cancellation of sigmoid(h) - 1.
  const double dh = s / (1.0 + exp(-h)) - (1.0 - s) / (1.0 + exp(h));
  const double dq = a.grad_scale * a.beta * dh / static_cast<double>(a.n_pairs);
  for (int64_t r = off[0] + threadIdx.x; r < off[2]; r += kPairBlock) {
    const float w = a.rows.weight[r];
    if (w == 0.0f) continue;
    const RowGrad e = rg[r];
    const double coef = (r < off[1] ? dq : -dq) * static_cast<double>(w) / static_cast<double>(e.gy);
    rg[r] = row_grad(coef, l[r], e.A, e.c, e.k);
  }
}

// Workgroups of the launch that starts at `at` of `total`.
unsigned groups_from(int64_t at, int64_t total) {
  return static_cast<unsigned>(total - at < kMostGroups ? total - at : kMostGroups);
}

size_t up16(size_t b) { return (b + 15) & ~size_t{15}; }

template <typename Tin>
hipError_t policy(const PolicyArgs& a, hipStream_t stream) {
  const int64_t n = a.rows.n_rows, nvec = a.rows.V / Elem<Tin>::kVec;
  hipError_t e = hipSuccess;
  if (a.G > 0) {
    RowGrad* rg = reinterpret_cast<RowGrad*>(a.row_loss);
    RowSum* part = reinterpret_cast<RowSum*>(rg + n);
    float* zy = reinterpret_cast<float*>(part + n * a.G);
    hipLaunchKernelGGL(parts_kernel<Tin>, dim3(static_cast<unsigned>(n * a.G)), dim3(kStatsBlock), 0, stream, a.rows,
                       part, zy, a.G);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t parts = grad_parts<Tin>(a.rows.V);
    if (a.rows.grad && n * parts <= kFewGroups) {
      hipLaunchKernelGGL(policy_parts_kernel<Tin>, dim3(static_cast<unsigned>(parts), static_cast<unsigned>(n + 1)),
                         dim3(kGradBlock), 0, stream, a, part, zy);
      return hipGetLastError();
    }
    hipLaunchKernelGGL(policy_finish_kernel, dim3(1), dim3(kGradBlock), 0, stream, a, part, zy,
                       a.rows.grad ? rg : nullptr);
    e = hipGetLastError();
    return e == hipSuccess && a.rows.grad ? launch_grad<Tin>(a.rows, rg, stream) : e;
  }
  if (n > 0 && a.rows.grad && held_row(nvec)) {
    const int64_t most = nvec <= kSmallRowVectors ? 2 * kCUs : kCUs;
    const dim3 grid(static_cast<unsigned>(n < most ? n : most));
    if (nvec <= kSmallRowVectors)
      hipLaunchKernelGGL((policy_row_kernel<Tin, 7, 19>), grid, dim3(512), 0, stream, a);
    else
      hipLaunchKernelGGL((policy_row_kernel<Tin, 15, 20>), grid, dim3(1024), 0, stream, a);
    e = hipGetLastError();
  } else if (n > 0) {
    RowGrad* rg = reinterpret_cast<RowGrad*>(reinterpret_cast<char*>(a.row_loss) +
                                             up16(static_cast<size_t>(n) * sizeof(double)));
    for (int64_t at = 0; at < n && e == hipSuccess; at += kMostGroups) {
      hipLaunchKernelGGL(policy_stats_kernel<Tin>, dim3(groups_from(at, n)), dim3(kStatsBlock), 0, stream, a, rg, at);
      e = hipGetLastError();
    }
    if (e == hipSuccess && a.rows.grad) e = launch_grad<Tin>(a.rows, rg, stream);
  }
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(kSumBlock), 0, stream, a.row_loss, n, 1.0, a.loss);
  return hipGetLastError();
}

template <typename Tin>
hipError_t preference(const PreferenceArgs& a, hipStream_t stream) {
  const size_t n = static_cast<size_t>(a.rows.n_rows);
  char* b = static_cast<char*>(a.ws);
  RowGrad* rg = reinterpret_cast<RowGrad*>(b);
  double* l = reinterpret_cast<double*>(b + n * sizeof(RowGrad));
  double* pair_loss = l + n;
  RowSum* part = reinterpret_cast<RowSum*>(pair_loss + a.n_pairs);
  hipError_t e = hipSuccess;
  // Only batches of few rows are split: with G > 1 one launch takes them all.
  for (int64_t at = 0; at < a.rows.n_rows && e == hipSuccess; at += kMostGroups) {
    hipLaunchKernelGGL(preference_stats_kernel<Tin>, dim3(groups_from(at, a.rows.n_rows) * static_cast<unsigned>(a.G)),
                       dim3(kStatsBlock), 0, stream, a, l, rg, part, at);
    e = hipGetLastError();
  }
  for (int64_t at = 0; at < a.n_pairs && e == hipSuccess; at += kMostGroups) {
    hipLaunchKernelGGL(preference_pair_kernel<Tin>, dim3(groups_from(at, a.n_pairs)), dim3(kPairBlock), 0, stream, a,
                       l, rg, part, pair_loss, static_cast<int32_t>(at));
    e = hipGetLastError();
  }
  // The mean over pairs: a single pair's own kernel writes it, that of a few
  // thousand goes beside their gradient.
  const bool beside = n > 0 && a.rows.grad && a.n_pairs > 1 && a.n_pairs <= kPairsBeside;
  if (e == hipSuccess && n > 0 && a.rows.grad)
    e = launch_grad<Tin>(a.rows, rg, stream, pair_loss, beside ? a.n_pairs : 0, a.loss);
  if (e != hipSuccess || beside || a.n_pairs == 1) return e;
  hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(kSumBlock), 0, stream, pair_loss,
                     static_cast<int64_t>(a.n_pairs), static_cast<double>(a.n_pairs), a.loss);
  return hipGetLastError();
}

}  // namespace

// Workgroups along a row for its sums: about 1,024 in all, each with at least
// 512 vectors. Preference loss, about 512, 1,024 and 2,048 in all: 128 rows of
// 151,936 bfloat16 logits 29.3, 30.8 and 33.1 us, 200 rows of as many float32
// logits 68.6, 66.5 and 67.9, 60 rows of 50,257 bfloat16 logits 13.8, 13.7 and
// 13.6. At least 256, 512 and 1,024 vectors: 17 rows of 50,257 11.7, 11.4 and
// 12.1 us, 60 rows 14.7, 13.7 and 15.0, 2 rows of 32,000 10.5, 10.2 and 10.5.
int row_parts(int64_t n_rows, int32_t V, pr_dtype dtype) {
  if (n_rows <= 0 || n_rows >= kSplitRows) return 1;
  const int64_t nvec = V / (dtype == PR_BF16 ? 8 : 4);
  const int64_t want = (1024 + n_rows - 1) / n_rows, most = nvec / 512;
  const int64_t G = want < most ? want : most;
  return static_cast<int>(G < 1 ? 1 : G > kMaxSplit ? kMaxSplit : G);
}

int policy_split(int64_t n_rows, int32_t V, pr_dtype dtype, bool grad) {
  if (n_rows <= 0 || n_rows >= kSplitRows) return 0;
  const int64_t nvec = V / (dtype == PR_BF16 ? 8 : 4);
  const int64_t few = nvec <= kSmallRowVectors ? kFewSmallRows : kFewRows;
  return grad && held_row(nvec) && n_rows > few ? 0 : row_parts(n_rows, V, dtype);
}

size_t policy_workspace_bytes(int64_t n_rows, int32_t V, pr_dtype dtype) {
  const size_t n = n_rows < 0 ? 0 : static_cast<size_t>(n_rows);
  const size_t terms = up16(n * sizeof(double));
  const size_t parts = static_cast<size_t>(row_parts(n_rows, V, dtype)) * sizeof(RowSum) + sizeof(float);
  return n * sizeof(RowGrad) + (n_rows < kSplitRows && n * parts > terms ? n * parts : terms);
}

hipError_t launch_loss_sum(const double* v, int64_t n, double over, float* loss, hipStream_t stream) {
  hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(kSumBlock), 0, stream, v, n, over, loss);
  return hipGetLastError();
}

hipError_t launch_policy(const PolicyArgs& a, pr_dtype dtype, hipStream_t stream) {
  return dtype == PR_BF16 ? policy<uint16_t>(a, stream) : policy<float>(a, stream);
}

int preference_split(int64_t n_rows, int32_t V, pr_dtype dtype) { return row_parts(n_rows, V, dtype); }

size_t preference_workspace_bytes(int64_t n_rows, int32_t n_pairs, int32_t G) {
  const size_t n = n_rows < 0 ? 0 : static_cast<size_t>(n_rows), P = n_pairs < 0 ? 0 : static_cast<size_t>(n_pairs);
  return n * sizeof(RowGrad) + (n + P) * sizeof(double) + (G > 1 ? n * static_cast<size_t>(G) * sizeof(RowSum) : 0);
}

hipError_t launch_preference(const PreferenceArgs& a, pr_dtype dtype, hipStream_t stream) {
  return dtype == PR_BF16 ? preference<uint16_t>(a, stream) : preference<float>(a, stream);
}

}  // namespace pr
