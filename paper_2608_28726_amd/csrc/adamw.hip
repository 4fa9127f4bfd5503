// An AdamW step over many tensors in one launch, states in 32 or 8 bits.
//
// m' = b1 m + (1 - b1) g, v' = b2 v + (1 - b2) g^2,
// p' = p (1 - lr wd) - lr c1 m' / (c2 sqrt(v') + eps), elementwise in float32.
// The step does a few dozen operations per 14 to 30 bytes: memory bounds it.
#include "adamw.h"

namespace pr {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 4;  // consecutive elements of a lane: a wave takes one block of 256
static_assert(kPer * kWave == kAdamBlock, "a wave takes a block");

// 32 random bits of a counter: two rounds of multiply and xor-shift by odd
// constants (the golden ratio and the square root of 2 in 32 bits).
__device__ __forceinline__ uint32_t mix(uint32_t x) {
  x *= 0x9E3779B9u;
  x ^= x >> 15;
  x *= 0x6A09E667u;
  return x ^ (x >> 13);
}

// Elements i .. i+3 of a tensor of n, as float32 (0 past the end). Tensors
// may start at any element, so vectors are read with an element's alignment.
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Unaligned {
  T v[N];
};

template <typename T>
__device__ __forceinline__ void load4(const T* p, int64_t i, int64_t n, T (&x)[4]) {
  if (i + 4 <= n) {
    const Unaligned<T, 4> u = *reinterpret_cast<const Unaligned<T, 4>*>(p + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = u.v[k];
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = i + k < n ? p[i + k] : T(0);
  }
}
template <typename T>
__device__ __forceinline__ void store4(T* p, int64_t i, int64_t n, const T (&x)[4]) {
  if (i + 4 <= n) {
    Unaligned<T, 4> u;
#pragma unroll
    for (int k = 0; k < 4; ++k) u.v[k] = x[k];
    *reinterpret_cast<Unaligned<T, 4>*>(p + i) = u;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < n) p[i + k] = x[k];
  }
}

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float(static_cast<uint32_t>(x) << 16); }

__device__ __forceinline__ uint16_t bf16_nearest(float x) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x)); }

// Value of an 8-bit state: k under block exponent E (top = 15 for m, 31 for v).
template <int TOP>
__device__ __forceinline__ float decode(uint32_t k, uint32_t E) {
  const float x = k ? __uint_as_float((k + 8u * (E - TOP)) << 20) : 0.0f;
  return E == 255u ? __uint_as_float(0x7fc00000u) : x;
}

// Exponent of a block from its largest magnitude (as bits).
template <int TOP>
__device__ __forceinline__ uint32_t block_exponent(uint32_t largest) {
  const uint32_t E = (largest + 0xfffffu) >> 23;
  return E > TOP ? (E < 255u ? E : 255u) : TOP + 1;
}

// Code of a magnitude (as bits) with 20 random bits.
template <int TOP, int LEAST>
__device__ __forceinline__ uint32_t encode(uint32_t bits, uint32_t random, uint32_t E) {
  const int k = static_cast<int>((bits + random) >> 20) - 8 * (static_cast<int>(E) - TOP);
  return bits == 0u ? 0u : static_cast<uint32_t>(max(k, LEAST)) & (8u * (TOP + 1) - 1);
}

template <typename Tp, typename Tg, bool EIGHT, bool GIVEN>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const AdamTensor* tensors, const AdamChunk* chunks,
                                                         AdamScalars s, AdamGrads grads, int32_t first) {
  const AdamChunk ch = chunks[blockIdx.x];
  const AdamTensor& t = tensors[ch.tensor];
  const Tg* grad = static_cast<const Tg*>(GIVEN ? grads.p[ch.tensor - first] : t.grad);
  if (!grad) return;
  const int64_t n = t.n;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  Tp* param = static_cast<Tp*>(t.param);
  const uint32_t key = mix(static_cast<uint32_t>(ch.tensor) + 1u + s.key);
  const int64_t base = static_cast<int64_t>(ch.chunk) * kAdamChunk;
  for (int64_t b = base + wave * kAdamBlock; b < base + kAdamChunk && b < n; b += kThreads / kWave * kAdamBlock) {
    const int64_t i = b + lane * kPer;
    Tp pr_[4];
    Tg gr[4];
    float m[4], v[4];
    load4(param, i, n, pr_);
    load4(grad, i, n, gr);
    if constexpr (EIGHT) {
      uint8_t mk[4], vk[4];
      load4(static_cast<const uint8_t*>(t.m), i, n, mk);
      load4(static_cast<const uint8_t*>(t.v), i, n, vk);
      const uint32_t me = t.m_exp[b / kAdamBlock], ve = t.v_exp[b / kAdamBlock];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float a = decode<15>(mk[k] & 127u, me);
        m[k] = mk[k] & 128u ? -a : a;
        v[k] = decode<31>(vk[k], ve);
      }
    } else {
      load4(static_cast<const float*>(t.m), i, n, m);
      load4(static_cast<const float*>(t.v), i, n, v);
    }
    float p[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float g = widen(gr[k]) * s.grad_scale;
      m[k] = m[k] * s.beta1 + g * s.one_minus_beta1;
      v[k] = v[k] * s.beta2 + (g * g) * s.one_minus_beta2;
      p[k] = widen(pr_[k]) * s.decay - s.rate * m[k] / (s.c2 * sqrtf(v[k]) + s.eps);
    }
    uint32_t rnd[4] = {0, 0, 0, 0};
    if constexpr (EIGHT || sizeof(Tp) == 2) {
#pragma unroll
      for (int k = 0; k < 4; ++k) rnd[k] = mix(static_cast<uint32_t>(i) + k + key);
    }
    if constexpr (sizeof(Tp) == 2) {
      uint16_t o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t bits = __float_as_uint(p[k]);
        // A NaN or an infinity keeps its bits: a carry would make it something else.
        const uint32_t up = (bits & 0x7f800000u) == 0x7f800000u ? bits | ((bits & 0x7fffffu) ? 0x400000u : 0u)
                                                                 : bits + (rnd[k] & 0xffffu);
        o[k] = static_cast<uint16_t>(up >> 16);
      }
      store4(param, i, n, o);
    } else {
      store4(param, i, n, p);
      if (t.copy) {
        uint16_t o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = bf16_nearest(p[k]);
        store4(t.copy, i, n, o);
      }
    }
    if constexpr (EIGHT) {
      uint32_t mb[4], vb[4], mt = 0, vt = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        mb[k] = i + k < n ? __float_as_uint(m[k]) & 0x7fffffffu : 0u;
        vb[k] = i + k < n ? __float_as_uint(v[k]) & 0x7fffffffu : 0u;
        mt = max(mt, mb[k]);
        vt = max(vt, vb[k]);
      }
      const uint32_t me = block_exponent<15>(wave_max_u(mt)), ve = block_exponent<31>(wave_max_u(vt));
      uint8_t mk[4], vk[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        mk[k] = static_cast<uint8_t>(encode<15, 0>(mb[k], rnd[k] & 0xfffffu, me) | (m[k] < 0.0f ? 128u : 0u));
        vk[k] = static_cast<uint8_t>(encode<31, 1>(vb[k], rnd[k] >> 12, ve));
      }
      store4(static_cast<uint8_t*>(t.m), i, n, mk);
      store4(static_cast<uint8_t*>(t.v), i, n, vk);
      if (lane == 0) {
        t.m_exp[b / kAdamBlock] = static_cast<uint8_t>(me);
        t.v_exp[b / kAdamBlock] = static_cast<uint8_t>(ve);
      }
    } else {
      store4(static_cast<float*>(t.m), i, n, m);
      store4(static_cast<float*>(t.v), i, n, v);
    }
  }
}

__global__ __launch_bounds__(kThreads) void adamw_moments_kernel(const AdamTensor* tensors, const AdamChunk* chunks,
                                                                 uint16_t* m_out, uint16_t* v_out) {
  const AdamChunk ch = chunks[blockIdx.x];
  const AdamTensor& t = tensors[ch.tensor];
  const int64_t n = t.n, at = t.first_block * kAdamBlock;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t base = static_cast<int64_t>(ch.chunk) * kAdamChunk;
  for (int64_t b = base + wave * kAdamBlock; b < base + kAdamChunk && b < n; b += kThreads / kWave * kAdamBlock) {
    const int64_t i = b + lane * kPer;
    uint8_t mk[4], vk[4];
    load4(static_cast<const uint8_t*>(t.m), i, n, mk);
    load4(static_cast<const uint8_t*>(t.v), i, n, vk);
    const uint32_t me = t.m_exp[b / kAdamBlock], ve = t.v_exp[b / kAdamBlock];
    uint16_t mo[4], vo[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      // At most 4 significant bits: the upper half of the float32 holds the value.
      const uint32_t a = __float_as_uint(decode<15>(mk[k] & 127u, me)) >> 16;
      mo[k] = static_cast<uint16_t>(a | (mk[k] & 128u ? 0x8000u : 0u));
      vo[k] = static_cast<uint16_t>(__float_as_uint(decode<31>(vk[k], ve)) >> 16);
    }
    store4(m_out, at + i, at + n, mo);
    store4(v_out, at + i, at + n, vo);
  }
}

template <typename Tp, typename Tg, bool EIGHT>
void launch(const AdamPlan& plan, int64_t begin, int64_t end, const AdamScalars& s, const AdamGrads* grads,
            int32_t first, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(end - begin)), block(kThreads);
  if (grads)
    hipLaunchKernelGGL((adamw_kernel<Tp, Tg, EIGHT, true>), grid, block, 0, stream, plan.tensors, plan.chunks + begin,
                       s, *grads, first);
  else
    hipLaunchKernelGGL((adamw_kernel<Tp, Tg, EIGHT, false>), grid, block, 0, stream, plan.tensors, plan.chunks + begin,
                       s, AdamGrads{}, 0);
}

template <typename Tp, typename Tg>
void launch_bits(const AdamPlan& plan, int64_t begin, int64_t end, const AdamScalars& s, const AdamGrads* grads,
                 int32_t first, hipStream_t stream) {
  if (plan.state_bits == 8)
    launch<Tp, Tg, true>(plan, begin, end, s, grads, first, stream);
  else
    launch<Tp, Tg, false>(plan, begin, end, s, grads, first, stream);
}

}  // namespace

hipError_t launch_adamw(const AdamPlan& plan, int64_t begin, int64_t end, const AdamScalars& s, const AdamGrads* grads,
                        int32_t first, hipStream_t stream) {
  constexpr int64_t kMost = int64_t{1} << 30;  // workgroups of a launch
  for (int64_t at = begin; at < end; at += kMost) {
    const int64_t to = end - at < kMost ? end : at + kMost;
    const bool p16 = plan.param_dtype == PR_BF16, g16 = plan.grad_dtype == PR_BF16;
    if (p16 && g16)
      launch_bits<uint16_t, uint16_t>(plan, at, to, s, grads, first, stream);
    else if (p16)
      launch_bits<uint16_t, float>(plan, at, to, s, grads, first, stream);
    else if (g16)
      launch_bits<float, uint16_t>(plan, at, to, s, grads, first, stream);
    else
      launch_bits<float, float>(plan, at, to, s, grads, first, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_adamw_moments(const AdamPlan& plan, int64_t n_chunks, uint16_t* m, uint16_t* v, hipStream_t stream) {
  constexpr int64_t kMost = int64_t{1} << 30;
  for (int64_t at = 0; at < n_chunks; at += kMost) {
    const int64_t k = n_chunks - at < kMost ? n_chunks - at : kMost;
    hipLaunchKernelGGL(adamw_moments_kernel, dim3(static_cast<unsigned>(k)), dim3(kThreads), 0, stream, plan.tensors,
                       plan.chunks + at, m, v);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace pr
