// Losses over logit rows and their gradients in the logits: the clipped
// policy loss with a KL term and the preference loss over pairs of requests.
//
// With u = z / T, l = u_y - log sum exp(u), both losses are functions of the
// rows' l, and a row's gradient is
//   dloss/dz_v = (dloss/dl) / T * (delta_vy - softmax(u)_v),
// so a row is read once for its sum of exps, then once more for its gradient.
//
// Exponents are in base 2: with c = log2(e) / T and the row's reference
// A = round(m c), m its largest logit, x_v = fma(z_v, c, -A) and
// S = sum 2^x_v, softmax(u)_v = 2^x_v / S. A row's sums over the vocabulary
// are float32 per lane (at most a few hundred terms each, all positive) and
// everything per row (l, ratio, coefficients) and over rows is in 64 bits.
#include "loss.h"
#include "row_scan.h"

namespace pr {
namespace {

using scan::head_elems;
using scan::neg_inf_vec;

constexpr int kStatsBlock = 256;
constexpr int kGradBlock = 256;
constexpr int kSumBlock = 1024;

// What the gradient pass needs of a row: dz_v = k 2^fma(z_v, c, -A) for every
// v but y, whose element is gy. k = gy = 0: the row's gradient is zero.
struct alignas(16) RowGrad {
  float A, c, k, gy;
};

// A row's sum of exps: its largest logit and, relative to round(m c), S.
struct RowSum {
  float m, S;
};

__device__ __forceinline__ float scale_of(float T) { return temperature_ok(T) ? kLog2e / T : kLog2e; }

// Running state of a lane: the wave's largest logit so far and the lane's sum
// relative to round(mw c). Every lane of the wave calls add() together.
struct LaneSum {
  float mw = -INFINITY, a = kNegSentinel, s = 0.0f;

  template <int N>
  __device__ __forceinline__ void add(const float (&z)[N], float c) {
    float top = z[0];
#pragma unroll
    for (int k = 1; k < N; ++k) top = fmaxf(top, z[k]);
    if (__any(top > mw)) {
      mw = fmaxf(mw, wave_max(top));
      // A mask of the type's lowest value may overflow here: it adds nothing
      // either way, and a row of nothing else is beyond the logits' bounds.
      const float now = fmaxf(mw * c, kNegSentinel);
      s *= fast_exp2(fmaxf(a - now, -kBig));
      a = now;
    }
    float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int k = 0; k < N; k += 2) {
      s0 += fast_exp2(fmaf(z[k], c, -a));
      if (k + 1 < N) s1 += fast_exp2(fmaf(z[k + 1 < N ? k + 1 : k], c, -a));
    }
    s += s0 + s1;
  }
  __device__ __forceinline__ void add1(float z, float c) {
    const float v[1] = {z};
    add(v, c);
  }
};

// Merge of the states held by the lanes of a wave (each relative to
// round(m c)); every lane gets the result. A state with m = -inf adds
// nothing but a NaN sum, which stays one.
__device__ __forceinline__ RowSum merge_lanes(RowSum e, float c) {
  RowSum r;
  r.m = wave_max(e.m);
  const float s = e.m == -INFINITY ? 0.0f : fast_exp2(fmaxf(e.m * c - r.m * c, -kBig));
  r.S = wave_sum(e.S * s);
  return r;
}

template <int BLOCK>
__device__ __forceinline__ RowSum merge_block(const LaneSum& L, float c) {
  constexpr int NW = BLOCK / kWave;
  __shared__ RowSum sh[NW];
  const RowSum w{L.mw, wave_sum(L.s)};
  const int lane = threadIdx.x % kWave;
  if (lane == 0) sh[threadIdx.x / kWave] = w;
  __syncthreads();
  return merge_lanes(lane < NW ? sh[lane] : RowSum{-INFINITY, 0.0f}, c);
}

struct RowValue {
  double l;
  float A;
  uint32_t flags;  // 0 or the reasons why l is NaN
};

// l of a row from its sum of exps. The exact residual of A = round(m c) moves
// S to the exact reference, so that the largest logit contributes exactly 1.
__device__ __forceinline__ RowValue row_value(const RowSum& p, float T, float c, int32_t y, int32_t V, float zy) {
  RowValue v;
  v.A = p.m * c;
  v.flags = 0;
  if (!temperature_ok(T)) v.flags |= PR_FLAG_BAD_TP;
  if (!(fabsf(p.S) < INFINITY) || p.m == INFINITY || p.m == -INFINITY) v.flags |= PR_FLAG_NONFINITE;
  if (!v.flags && fabsf(p.m) > ldexpf(T, 100)) v.flags |= PR_FLAG_BAD_TP;
  if (y < 0 || y >= V) v.flags |= PR_FLAG_BAD_ID;
  if (v.flags) {
    v.l = __longlong_as_double(0x7ff8000000000000ll);
    return v;
  }
  const double delta = static_cast<double>(fmaf(p.m, c, -v.A));
  const double lnS = ln_sum(static_cast<double>(p.S) * exp2(-delta));
  v.l = (static_cast<double>(zy) - static_cast<double>(p.m)) / static_cast<double>(T) - lnS;
  return v;
}

// The gradient's factors of a row from coef = dloss/dl / T. 1 - p_y is
// -expm1(l), which keeps its precision when p_y is near 1.
__device__ __forceinline__ RowGrad row_grad(double coef, double l, float A, float c, float S) {
  if (coef == 0.0) return RowGrad{0.0f, 0.0f, 0.0f, 0.0f};
  if (!(coef == coef)) {
    const float nan = __uint_as_float(0x7fc00000u);
    return RowGrad{0.0f, 0.0f, nan, nan};
  }
  return RowGrad{A, c, static_cast<float>(-coef / static_cast<double>(S)), static_cast<float>(-coef * expm1(l))};
}

template <typename Tin>
__device__ __forceinline__ const Tin* row_ptr(const LossRows& a, int64_t r) {
  return static_cast<const Tin*>(a.logits) + r * a.row_stride;
}

template <typename Tin>
__device__ __forceinline__ float token_logit(const LossRows& a, int64_t r, int32_t y) {
  return y >= 0 && y < a.V ? Elem<Tin>::load1(row_ptr<Tin>(a, r), y) : 0.0f;
}

// The policy loss of one row: outputs, its term of the loss and its gradient's factors.
__device__ __forceinline__ RowGrad policy_row(const PolicyArgs& a, int64_t r, const RowValue& v, float T, float c,
                                              float S, float w) {
  const double A = a.advantage[r], ratio = exp(v.l - static_cast<double>(a.old_logprob[r]));
  const double free = ratio * A, held = fmin(fmax(ratio, a.clip_lo), a.clip_hi) * A;
  const bool clipped = free > held;
  double kl = 0.0, rise = 0.0;
  if (a.ref_logprob) {
    const double d = static_cast<double>(a.ref_logprob[r]) - v.l;
    rise = expm1(d);
    kl = d == INFINITY ? d : rise - d;  // a token of probability 0
  }
  const double gain = v.flags ? v.l : (clipped ? held : free);
  a.row_loss[r] = static_cast<double>(w) * ((a.ref_logprob ? a.kl_coef * kl : 0.0) - gain);
  if (a.out.logprob) a.out.logprob[r] = static_cast<float>(v.l);
  if (a.out.ratio) a.out.ratio[r] = static_cast<float>(ratio);
  if (a.out.kl) a.out.kl[r] = static_cast<float>(kl);
  if (a.out.flags) a.out.flags[r] = v.flags | (!v.flags && clipped ? PR_FLAG_CLIPPED : 0u);
  const double dl = static_cast<double>(w) * ((clipped ? 0.0 : -free) - (a.ref_logprob ? a.kl_coef * rise : 0.0));
  return row_grad(v.flags ? v.l : a.grad_scale * dl / static_cast<double>(T), v.l, v.A, c, S);
}

__device__ __forceinline__ void policy_masked(const PolicyArgs& a, int64_t r) {
  a.row_loss[r] = 0.0;
  if (a.out.logprob) a.out.logprob[r] = 0.0f;
  if (a.out.ratio) a.out.ratio[r] = 0.0f;
  if (a.out.kl) a.out.kl[r] = 0.0f;
  if (a.out.flags) a.out.flags[r] = PR_FLAG_MASKED;
}

// Sum of v[0..n) by one workgroup, in a fixed order (valid in thread 0).
__device__ __forceinline__ double block_sum(const double* v, int64_t n) {
  __shared__ double sh[kSumBlock / kWave];
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += blockDim.x) s += v[i];
  s = wave_sum_d(s);
  if (threadIdx.x % kWave == 0) sh[threadIdx.x / kWave] = s;
  __syncthreads();
  double t = 0.0;
  if (threadIdx.x == 0)
    for (int w = 0; w < static_cast<int>(blockDim.x) / kWave; ++w) t += sh[w];
  return t;
}

__global__ __launch_bounds__(kSumBlock) void loss_sum_kernel(const double* v, int64_t n, double factor, float* loss) {
  const double s = block_sum(v, n);
  if (threadIdx.x == 0) loss[0] = static_cast<float>(s * factor);
}

// The sum of exps of a stretch of a row (the whole row when G = 1).
template <typename Tin, int BLOCK>
__device__ RowSum stretch_sum(const Tin* row, int32_t V, int g, int G, float c) {
  constexpr int VEC = Elem<Tin>::kVec;
  const int64_t h = head_elems<Tin>(row, V), nvec = (V - h) / VEC;
  const int64_t vb = nvec * g / G, ve = nvec * (g + 1) / G;
  const int t = threadIdx.x;
  LaneSum L;
  vec4u v[4];
  scan::stretch_prefetch<Tin, BLOCK, 4>(row, h, vb, ve, v);
  if (g == 0) L.add1(t < h ? Elem<Tin>::load1(row, t) : -INFINITY, c);
  if (g == G - 1) {
    const int64_t e = h + nvec * VEC + t;
    L.add1(e < V ? Elem<Tin>::load1(row, e) : -INFINITY, c);
  }
  const vec4u* vp = reinterpret_cast<const vec4u*>(row + h);
  scan::stream_stretch<Tin, BLOCK, 2, 4>(vp, vb, ve, v, [&](const vec4u* vv, int64_t) {
    float z[2 * VEC];
    Elem<Tin>::unpack(vv[0], z);
    Elem<Tin>::unpack(vv[1], z + VEC);
    L.add(z, c);
  });
  return merge_block<BLOCK>(L, c);
}

template <typename Tin>
__global__ __launch_bounds__(kStatsBlock) void policy_stats_kernel(PolicyArgs a, RowGrad* rg) {
  const int64_t r = blockIdx.x;
  const float w = a.rows.weight[r];
  if (w == 0.0f) {
    if (threadIdx.x == 0) {
      policy_masked(a, r);
      rg[r] = RowGrad{0.0f, 0.0f, 0.0f, 0.0f};
    }
    return;
  }
  const float T = a.rows.temperature[r], c = scale_of(T);
  const int32_t y = a.rows.ids[r];
  const float zy = token_logit<Tin>(a.rows, r, y);
  const RowSum p = stretch_sum<Tin, kStatsBlock>(row_ptr<Tin>(a.rows, r), a.rows.V, 0, 1, c);
  if (threadIdx.x == 0) {
    const RowValue v = row_value(p, T, c, y, a.rows.V, zy);
    rg[r] = policy_row(a, r, v, T, c, p.S, w);
  }
}

// A bfloat16 or float32 vector of gradients. The gradient's rows may sit
// otherwise than the logits' relative to 16 bytes, so its vectors are stored
// with the alignment of an element (global stores need no more).
template <typename Tin>
struct GradVec;
template <>
struct GradVec<float> {
  struct __attribute__((packed, aligned(4))) Store {
    vec4u v;
  };
  __device__ __forceinline__ static vec4u pack(const float (&g)[4]) {
    return vec4u{__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3])};
  }
  __device__ __forceinline__ static void store1(void* base, int64_t i, float g) { static_cast<float*>(base)[i] = g; }
};
typedef float float2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {  // round to nearest even
  const float2v f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

template <>
struct GradVec<uint16_t> {
  struct __attribute__((packed, aligned(2))) Store {
    vec4u v;
  };
  __device__ __forceinline__ static vec4u pack(const float (&g)[8]) {
    return vec4u{pack_bf16(g[0], g[1]), pack_bf16(g[2], g[3]), pack_bf16(g[4], g[5]), pack_bf16(g[6], g[7])};
  }
  __device__ __forceinline__ static void store1(void* base, int64_t i, float g) {
    static_cast<uint16_t*>(base)[i] = static_cast<uint16_t>(pack_bf16(g, 0.0f));
  }
};

template <typename Tin>
__device__ __forceinline__ void store_grad(Tin* at, const vec4u& v) {
  reinterpret_cast<typename GradVec<Tin>::Store*>(at)->v = v;
}

__device__ __forceinline__ float grad_of(float z, const RowGrad& q) { return q.k * fast_exp2(fmaf(z, q.c, -q.A)); }

// The gradient of a stretch of a row. Each element is read and written by one
// thread, so the gradient may take the logits' place.
template <typename Tin>
__global__ __launch_bounds__(kGradBlock) void grad_kernel(LossRows a, const RowGrad* rg, int32_t segs) {
  constexpr int VEC = Elem<Tin>::kVec;
  const int64_t r = blockIdx.x / segs;
  const int seg = blockIdx.x % segs;
  const RowGrad q = rg[r];
  const Tin* row = row_ptr<Tin>(a, r);
  Tin* out = static_cast<Tin*>(a.grad) + r * a.grad_stride;
  const int64_t h = head_elems<Tin>(row, a.V), nvec = (a.V - h) / VEC;
  const int64_t vb = nvec * seg / segs, ve = nvec * (seg + 1) / segs;
  const int t = threadIdx.x;
  const int32_t y = a.ids[r];
  const bool zero = q.k == 0.0f && q.gy == 0.0f;
  const int64_t tail = h + nvec * VEC;
  if (seg == 0 && t < h)
    GradVec<Tin>::store1(out, t, zero ? 0.0f : t == y ? q.gy : grad_of(Elem<Tin>::load1(row, t), q));
  if (seg == segs - 1 && tail + t < a.V)
    GradVec<Tin>::store1(out, tail + t,
                         zero ? 0.0f : tail + t == y ? q.gy : grad_of(Elem<Tin>::load1(row, tail + t), q));
  if (zero) {
    for (int64_t j = vb + t; j < ve; j += kGradBlock) store_grad(out + h + j * VEC, vec4u{0, 0, 0, 0});
    return;
  }
  const vec4u* vp = reinterpret_cast<const vec4u*>(row + h);
  for (int64_t j = vb + t; j < ve; j += kGradBlock) {
    float z[VEC];
    Elem<Tin>::unpack(vp[j], z);
#pragma unroll
    for (int k = 0; k < VEC; ++k) z[k] = grad_of(z[k], q);
    const int64_t at = y - (h + j * VEC);
    if (at >= 0 && at < VEC) {
#pragma unroll
      for (int k = 0; k < VEC; ++k) z[k] = k == at ? q.gy : z[k];
    }
    store_grad(out + h + j * VEC, GradVec<Tin>::pack(z));
  }
}

// Vectors of a row that one workgroup of the gradient pass takes.
constexpr int64_t kGradSegment = 8 * kGradBlock;

template <typename Tin>
hipError_t launch_grad(const LossRows& a, const RowGrad* rg, hipStream_t stream) {
  const int64_t nvec = a.V / Elem<Tin>::kVec;
  const int32_t segs = static_cast<int32_t>((nvec + kGradSegment - 1) / kGradSegment);
  const int32_t s = segs < 1 ? 1 : segs;
  // Lists of more than 2^31 workgroups take several launches.
  const int64_t most = (int64_t{1} << 30) / s;
  for (int64_t at = 0; at < a.n_rows; at += most) {
    LossRows b = a;
    b.n_rows = a.n_rows - at < most ? a.n_rows - at : most;
    b.logits = static_cast<const Tin*>(a.logits) + at * a.row_stride;
    b.grad = static_cast<Tin*>(a.grad) + at * a.grad_stride;
    b.ids = a.ids + at;
    hipLaunchKernelGGL(grad_kernel<Tin>, dim3(static_cast<unsigned>(b.n_rows * s)), dim3(kGradBlock), 0, stream, b,
                       rg + at, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// The preference loss of a row, first part: l and what its gradient needs.
__device__ __forceinline__ void preference_row(const PreferenceArgs& a, int64_t r, const RowSum& p, float T, float c,
                                               int32_t y, float zy, double* l, RowGrad* rg) {
  const RowValue v = row_value(p, T, c, y, a.rows.V, zy);
  l[r] = v.l;
  rg[r] = RowGrad{v.A, c, p.S, T};
  if (a.out.logprob) a.out.logprob[r] = static_cast<float>(v.l);
  if (a.out.flags) a.out.flags[r] = v.flags;
}

template <typename Tin>
__global__ __launch_bounds__(kStatsBlock) void preference_stats_kernel(PreferenceArgs a, double* l, RowGrad* rg,
                                                                      RowSum* part) {
  const int64_t r = blockIdx.x / a.G;
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

// One workgroup per pair: the sums over both requests, the pair's loss, and
// the gradient's factors of the pair's rows. Rows that were split finish here.
constexpr int kPairBlock = 256;

__device__ __forceinline__ double softplus(double x) { return fmax(x, 0.0) + log1p(exp(-fabs(x))); }

template <typename Tin>
__global__ __launch_bounds__(kPairBlock) void preference_pair_kernel(PreferenceArgs a, double* l, RowGrad* rg,
                                                                    const RowSum* part, double* pair_loss) {
  __shared__ double sh[2][kPairBlock / kWave];
  const int p = blockIdx.x;
  int64_t off[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const int64_t o = a.offsets[2 * p + i];
    off[i] = o < 0 ? 0 : o > a.rows.n_rows ? a.rows.n_rows : o;
  }
  double q[2] = {0.0, 0.0};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    for (int64_t r = off[i] + threadIdx.x; r < off[i + 1]; r += kPairBlock) {
      const float w = a.rows.weight[r];
      if (w == 0.0f) continue;
      if (a.G > 1) {
        const float T = a.rows.temperature[r], c = scale_of(T);
        RowSum s{-INFINITY, 0.0f};
        for (int g = 0; g < a.G; ++g) s.m = fmaxf(s.m, part[r * a.G + g].m);
        for (int g = 0; g < a.G; ++g) {
          const RowSum e = part[r * a.G + g];
          s.S += e.S * (e.m == -INFINITY ? 0.0f : fast_exp2(fmaxf(e.m * c - s.m * c, -kBig)));
        }
        const int32_t y = a.rows.ids[r];
        preference_row(a, r, s, T, c, y, token_logit<Tin>(a.rows, r, y), l, rg);
      }
      q[i] += static_cast<double>(w) * (l[r] - (a.ref_logprob ? static_cast<double>(a.ref_logprob[r]) : 0.0));
    }
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
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    for (int64_t r = off[i] + threadIdx.x; r < off[i + 1]; r += kPairBlock) {
      const float w = a.rows.weight[r];
      if (w == 0.0f) continue;
      const RowGrad e = rg[r];
      const double coef = (i == 0 ? dq : -dq) * static_cast<double>(w) / static_cast<double>(e.gy);
      rg[r] = row_grad(coef, l[r], e.A, e.c, e.k);
    }
  }
}

size_t up16(size_t b) { return (b + 15) & ~size_t{15}; }

template <typename Tin>
hipError_t policy(const PolicyArgs& a, hipStream_t stream) {
  RowGrad* rg = reinterpret_cast<RowGrad*>(reinterpret_cast<char*>(a.row_loss) +
                                           up16(static_cast<size_t>(a.rows.n_rows) * sizeof(double)));
  if (a.rows.n_rows > 0) {
    hipLaunchKernelGGL(policy_stats_kernel<Tin>, dim3(static_cast<unsigned>(a.rows.n_rows)), dim3(kStatsBlock), 0,
                       stream, a, rg);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.rows.grad) e = launch_grad<Tin>(a.rows, rg, stream);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(kSumBlock), 0, stream, a.row_loss, a.rows.n_rows, 1.0, a.loss);
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
  if (n > 0) {
    hipLaunchKernelGGL(preference_stats_kernel<Tin>, dim3(static_cast<unsigned>(n * static_cast<size_t>(a.G))),
                       dim3(kStatsBlock), 0, stream, a, l, rg, part);
    e = hipGetLastError();
  }
  if (e == hipSuccess && a.n_pairs > 0) {
    hipLaunchKernelGGL(preference_pair_kernel<Tin>, dim3(static_cast<unsigned>(a.n_pairs)), dim3(kPairBlock), 0,
                       stream, a, l, rg, part, pair_loss);
    e = hipGetLastError();
  }
  if (e == hipSuccess && n > 0 && a.rows.grad) e = launch_grad<Tin>(a.rows, rg, stream);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(kSumBlock), 0, stream, pair_loss,
                     static_cast<int64_t>(a.n_pairs), 1.0 / a.n_pairs, a.loss);
  return hipGetLastError();
}

}  // namespace

size_t policy_workspace_bytes(int64_t n_rows) {
  const size_t n = n_rows < 0 ? 0 : static_cast<size_t>(n_rows);
  return up16(n * sizeof(double)) + n * sizeof(RowGrad);
}

hipError_t launch_policy(const PolicyArgs& a, pr_dtype dtype, hipStream_t stream) {
  return dtype == PR_BF16 ? policy<uint16_t>(a, stream) : policy<float>(a, stream);
}

int preference_split(int64_t n_rows, int32_t V, pr_dtype dtype) {
  // Below 1,024 rows a row is spread over workgroups, at least 1,024 vectors each.
  const int64_t nvec = V / (dtype == PR_BF16 ? 8 : 4);
  if (n_rows <= 0 || n_rows >= 1024) return 1;
  const int64_t want = (2048 + n_rows - 1) / n_rows, most = nvec / 1024;
  const int64_t G = want < most ? want : most;
  return static_cast<int>(G < 1 ? 1 : G > 64 ? 64 : G);
}

size_t preference_workspace_bytes(int64_t n_rows, int32_t n_pairs, int32_t G) {
  const size_t n = n_rows < 0 ? 0 : static_cast<size_t>(n_rows), P = n_pairs < 0 ? 0 : static_cast<size_t>(n_pairs);
  return n * sizeof(RowGrad) + (n + P) * sizeof(double) + (G > 1 ? n * static_cast<size_t>(G) * sizeof(RowSum) : 0);
}

hipError_t launch_preference(const PreferenceArgs& a, pr_dtype dtype, hipStream_t stream) {
  return dtype == PR_BF16 ? preference<uint16_t>(a, stream) : preference<float>(a, stream);
}

}  // namespace pr
