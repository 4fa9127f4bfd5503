// A row's sum of exps, and what kernels that write a gradient beside the logits
// share (internal, device code only).
#pragma once

#include "row_scan.h"

namespace pr {

using scan::head_elems;
using scan::neg_inf_vec;

// A row's sum of exps: its largest logit and, relative to that one's reference, S.
struct RowSum {
  float m, S;
};

// A rejected temperature still gets a finite scale, so that what else is
// wrong with a row is seen.
__device__ __forceinline__ float scale_of(float T) { return temperature_ok(T) ? kLog2e / T : kLog2e; }

// Running state of a lane: the wave's largest logit so far, its reference (cw, a)
// and the lane's sum relative to that. Every lane of the wave calls add() together. LONG:
// for rows of any length, the sum's roundings so far are held beside it
// (Kahan's sum); without, a row of 4 million logits was off by 5.5e-6 of its
// sum, and the error grows with the row.
template <bool LONG>
struct LaneSum {
  float mw = -INFINITY, a = kNegSentinel, cw = 1.0f, s = 0.0f, over = 0.0f;

  template <int N>
  __device__ __forceinline__ void add(const float (&z)[N], float c) {
    float top = z[0];
#pragma unroll
    for (int k = 1; k < N; ++k) top = fmaxf(top, z[k]);
    add_top(z, top, c);
  }
  // top: the largest of z.
  template <int N>
  __device__ __forceinline__ void add_top(const float (&z)[N], float top, float c) {
    if (__any(top > mw)) {
      mw = fmaxf(mw, wave_max(top));
      const RowRef now = row_ref(mw, c);
      const float f = now.far ? 0.0f : fast_exp2(fmaxf(a - now.A, -kBig));
      s *= f;
      if (LONG) over *= f;
      a = now.A;
      cw = now.c;
    }
    float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int k = 0; k < N; k += 2) {
      s0 += fast_exp2(fmaf(z[k], cw, -a));
      if (k + 1 < N) s1 += fast_exp2(fmaf(z[k + 1 < N ? k + 1 : k], cw, -a));
    }
    if (LONG) {
      const float x = (s0 + s1) - over, t = s + x;
      over = (t - s) - x;
      s = t;
    } else {
      s += s0 + s1;
    }
  }
  __device__ __forceinline__ void add1(float z, float c) {
    const float v[1] = {z};
    add(v, c);
  }
};

// Merge of the states held by the lanes of a wave (each relative to its own
// largest logit's reference); every lane gets the result. A state with m = -inf adds
// nothing but a NaN sum, which stays one.
__device__ __forceinline__ RowSum merge_lanes(RowSum e, float c) {
  RowSum r;
  r.m = wave_max(e.m);
  const float s = e.m == -INFINITY ? 0.0f : fast_exp2(ref_shift(e.m, r.m, c));
  r.S = wave_sum(e.S * s);
  return r;
}

template <int BLOCK>
__device__ __forceinline__ RowSum merge_block(const LaneSum<true>& L, float c) {
  constexpr int NW = BLOCK / kWave;
  __shared__ RowSum sh[NW];
  const RowSum w{L.mw, wave_sum(L.s)};
  const int lane = threadIdx.x % kWave;
  if (lane == 0) sh[threadIdx.x / kWave] = w;
  __syncthreads();
  return merge_lanes(lane < NW ? sh[lane] : RowSum{-INFINITY, 0.0f}, c);
}

// The sum of exps of a stretch of a row (the whole row when G = 1).
template <typename Tin, int BLOCK>
__device__ RowSum stretch_sum(const Tin* row, int32_t V, int g, int G, float c) {
  constexpr int VEC = Elem<Tin>::kVec;
  const int64_t h = head_elems<Tin>(row, V), nvec = (V - h) / VEC;
  const int64_t vb = nvec * g / G, ve = nvec * (g + 1) / G;
  const int t = threadIdx.x;
  LaneSum<true> L;
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

// The state of a row from its G parts, all of them read at once.
constexpr int kMaxSplit = 16;

__device__ __forceinline__ RowSum merge_parts(const RowSum* part, int G, float c) {
  RowSum e[kMaxSplit];
  RowSum s{-INFINITY, 0.0f};
#pragma unroll
  for (int g = 0; g < kMaxSplit; ++g) e[g] = g < G ? part[g] : RowSum{-INFINITY, 0.0f};
#pragma unroll
  for (int g = 0; g < kMaxSplit; ++g) s.m = fmaxf(s.m, e[g].m);
  const float A = s.m * c;
  if (fabsf(A) < kFar) {
#pragma unroll
    for (int g = 0; g < kMaxSplit; ++g)
      s.S += e[g].S * (e[g].m == -INFINITY ? 0.0f : fast_exp2(fmaxf(e[g].m * c - A, -kBig)));
  } else {  // as ref_shift: equal ones count alike
#pragma unroll
    for (int g = 0; g < kMaxSplit; ++g) s.S += e[g].m == s.m || e[g].S != e[g].S ? e[g].S : 0.0f;
  }
  return s;
}

// A bfloat16 or float32 vector of gradients. The gradient's rows may sit
// otherwise than the logits' relative to 16 bytes, so its vectors are stored
// with the alignment of an element (global stores need no more).
template <typename Tin>
struct GradVec;
template <>
struct GradVec<float> {
  typedef uint32_t Store __attribute__((ext_vector_type(4), aligned(4)));
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
  typedef uint32_t Store __attribute__((ext_vector_type(4), aligned(2)));
  __device__ __forceinline__ static vec4u pack(const float (&g)[8]) {
    return vec4u{pack_bf16(g[0], g[1]), pack_bf16(g[2], g[3]), pack_bf16(g[4], g[5]), pack_bf16(g[6], g[7])};
  }
  __device__ __forceinline__ static void store1(void* base, int64_t i, float g) {
    static_cast<uint16_t*>(base)[i] = static_cast<uint16_t>(pack_bf16(g, 0.0f));
  }
};

template <typename Tin>
__device__ __forceinline__ void store_grad(Tin* at, const vec4u& v) {
  *reinterpret_cast<typename GradVec<Tin>::Store*>(at) = v;
}
// The same past the caches.
template <typename Tin>
__device__ __forceinline__ void stream_grad(Tin* at, const vec4u& v) {
  typedef typename GradVec<Tin>::Store Store;
  __builtin_nontemporal_store(static_cast<Store>(v), reinterpret_cast<Store*>(at));
}

// The element outside a row's vectors that thread t takes: the first 8
// threads those before the vectors, the next 8 those after them (V: none).
__device__ __forceinline__ int32_t scalar_element(int t, int32_t h, int32_t tail, int32_t V) {
  if (t < 8) return t < h ? t : V;
  return t - 8 < V - tail ? tail + t - 8 : V;
}

}  // namespace pr
