// An AdamW step over many tensors in one launch, states in 32 or 8 bits.
//
// m' = b1 m + (1 - b1) g, v' = b2 v + (1 - b2) g^2,
// p' = p - (lr wd p + lr c1 m' / (c2 sqrt(v') + eps)), elementwise in float32.
// The step moves 10 to 30 bytes an element for 30 to 80 operations: memory
// bounds it. 216 million float32 parameters with bfloat16 gradients and copies:
// 32-bit states 1,092 us (6.1 GB, 5.6 TB/s), 8-bit states 629 us (3.5 GB, 5.5
// TB/s), their values 266 us (1.3 GB, 4.9 TB/s) under a trace, 1,076 and 854 us
// (both) without; a copy reaches 6.5 TB/s. Short
// workgroups in memory order suit it: of 512 threads and 2,048 elements the
// 8-bit step took 599 us, of 256 and 1,024 617, of 256 and 2,048 674.
#include "adamw.h"

namespace pr {
namespace {

constexpr int kThreads = 512;
constexpr int kPer = 4;  // consecutive elements of a lane: a wave takes one block of 256
static_assert(kPer * kWave == kAdamBlock, "a wave takes a block");
constexpr int kTurns = kAdamChunk / (kThreads * kPer);
static_assert(kTurns * kThreads * kPer == kAdamChunk, "a chunk is whole blocks for every wave");

// Two rounds of multiply and xor-shift by odd constants (the golden ratio and
// the square root of 2 in 32 bits) turn a counter into 32 random bits. The
// first product of consecutive counters is one product and sums.
constexpr uint32_t kMix1 = 0x9E3779B9u, kMix2 = 0x6A09E667u;
__device__ __forceinline__ uint32_t mix_product(uint32_t x) {  // x: the counter times kMix1
  x ^= x >> 15;
  x *= kMix2;
  return x ^ (x >> 13);
}

// The tensors' memory is reached through pointers read from the plan: said to
// be global memory, or every access would be a generic one.
template <typename T>
using Global = __attribute__((address_space(1))) T;
template <typename T>
__device__ __forceinline__ Global<T>* global(T* p) {
  return (Global<T>*)p;
}

// Four elements, with the alignment of one: tensors may start anywhere.
typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t ushort4u __attribute__((ext_vector_type(4), aligned(2)));
typedef uint8_t byte4u __attribute__((ext_vector_type(4), aligned(1)));
template <typename T>
struct FourOf;
template <>
struct FourOf<float> {
  typedef float4u type;
};
template <>
struct FourOf<uint16_t> {
  typedef ushort4u type;
};
template <>
struct FourOf<uint8_t> {
  typedef byte4u type;
};
template <typename T>
using Four = typename FourOf<T>::type;

// Elements i .. i + 3 of n (0 past the end). FULL: all four are there.
// STREAM: past the caches.
template <bool FULL, bool STREAM, typename T>
__device__ __forceinline__ void load4(const T* base, int32_t i, int32_t n, T (&x)[4]) {
  const Global<const T>* p = global(base);
  if (FULL || i + 4 <= n) {
    const auto* q = (const Global<const Four<T>>*)(p + i);
    const Four<T> u = STREAM ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = u[k];
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = i + k < n ? p[i + k] : T(0);
  }
}
template <bool FULL, bool STREAM, typename T>
__device__ __forceinline__ void store4(T* base, int32_t i, int32_t n, const T (&x)[4]) {
  Global<T>* p = global(base);
  if (FULL || i + 4 <= n) {
    Four<T> u;
#pragma unroll
    for (int k = 0; k < 4; ++k) u[k] = x[k];
    auto* q = (Global<Four<T>>*)(p + i);
    if (STREAM)
      __builtin_nontemporal_store(u, q);
    else
      *q = u;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < n) p[i + k] = x[k];
  }
}
// Four bytes as a word, byte k element i + k.
template <bool FULL, bool STREAM>
__device__ __forceinline__ uint32_t load_codes(const uint8_t* base, int32_t i, int32_t n) {
  uint8_t x[4];
  load4<FULL, STREAM>(base, i, n, x);
  return static_cast<uint32_t>(x[0]) | static_cast<uint32_t>(x[1]) << 8 | static_cast<uint32_t>(x[2]) << 16 |
         static_cast<uint32_t>(x[3]) << 24;
}
template <bool FULL, bool STREAM>
__device__ __forceinline__ void store_codes(uint8_t* base, int32_t i, int32_t n, uint32_t w) {
  const uint8_t x[4] = {static_cast<uint8_t>(w), static_cast<uint8_t>(w >> 8), static_cast<uint8_t>(w >> 16),
                        static_cast<uint8_t>(w >> 24)};
  store4<FULL, STREAM>(base, i, n, x);
}

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float(static_cast<uint32_t>(x) << 16); }

typedef float float2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void bf16_nearest(const float (&p)[4], uint16_t (&o)[4]) {
  const uint32_t a = __builtin_bit_cast(uint32_t, __builtin_convertvector((float2v{p[0], p[1]}), bf16x2));
  const uint32_t b = __builtin_bit_cast(uint32_t, __builtin_convertvector((float2v{p[2], p[3]}), bf16x2));
  o[0] = static_cast<uint16_t>(a);
  o[1] = static_cast<uint16_t>(a >> 16);
  o[2] = static_cast<uint16_t>(b);
  o[3] = static_cast<uint16_t>(b >> 16);
}

constexpr uint32_t kNanBits = 0x7fc00000u;

// Bits of the value of code k > 0 are (k + base) << 20, with base = 8 (E - TOP)
// of the block's exponent E (TOP = 15 for m, 31 for v).
template <int TOP>
__device__ __forceinline__ uint32_t code_base(uint32_t E) { return 8u * (E - TOP); }

__device__ __forceinline__ float decode_m(uint32_t word, int k, uint32_t base) {
  const uint32_t c = (word >> (8 * k)) & 127u;
  const uint32_t bits = c ? (c + base) << 20 : 0u;
  return __uint_as_float(bits | ((word << (24 - 8 * k)) & 0x80000000u));
}
__device__ __forceinline__ float decode_v(uint32_t word, int k, uint32_t base) {
  const uint32_t c = (word >> (8 * k)) & 255u;
  return __uint_as_float(c ? (c + base) << 20 : 0u);
}

// Exponent of a block from its largest magnitude (as bits).
template <int TOP>
__device__ __forceinline__ uint32_t block_exponent(uint32_t largest) {
  return min(max((largest + 0xfffffu) >> 23, static_cast<uint32_t>(TOP + 1)), 255u);
}

// The parameter after its decay and update. The decay joins the update before
// either meets p: 1 - lr wd in float32 is a multiple of 2^-24, which at rates
// of post-training is off by tens of percent of lr wd, for all elements alike.
// An infinite parameter stays infinite.
__device__ __forceinline__ float moved(float p, const AdamScalars& s, float update) {
  const float q = p - fmaf(s.decay, p, update);
  return fabsf(p) == INFINITY ? p * s.keep - update : q;
}

template <typename Tp, typename Tg, bool EIGHT, bool STREAM, bool FULL>
__device__ __forceinline__ void step_block(const AdamChunk& ch, const Tg* grad, const AdamScalars& s, int32_t b) {
  const int32_t n = ch.n, i = b + static_cast<int32_t>(threadIdx.x % kWave) * kPer;
  Tp pr_[4];
  Tg gr[4];
  float m[4], v[4];
  Tp* param = static_cast<Tp*>(ch.param);
  load4<FULL, STREAM>(param, i, n, pr_);
  load4<FULL, STREAM>(grad, i, n, gr);
  if constexpr (EIGHT) {
    const uint32_t mw = load_codes<FULL, STREAM>(static_cast<const uint8_t*>(ch.m), i, n);
    const uint32_t vw = load_codes<FULL, STREAM>(static_cast<const uint8_t*>(ch.v), i, n);
    const uint32_t me = global(ch.m_exp)[b / kAdamBlock], ve = global(ch.v_exp)[b / kAdamBlock];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m[k] = decode_m(mw, k, code_base<15>(me));
      v[k] = decode_v(vw, k, code_base<31>(ve));
    }
    if (me == 255u || ve == 255u) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (me == 255u) m[k] = __uint_as_float(kNanBits);
        if (ve == 255u) v[k] = __uint_as_float(kNanBits);
      }
    }
  } else {
    load4<FULL, STREAM>(static_cast<const float*>(ch.m), i, n, m);
    load4<FULL, STREAM>(static_cast<const float*>(ch.v), i, n, v);
  }
  float p[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float g = widen(gr[k]) * s.grad_scale;
    m[k] = m[k] * s.beta1 + g * s.one_minus_beta1;
    v[k] = v[k] * s.beta2 + (g * g) * s.one_minus_beta2;
  }
  // The update is off by at most four roundings with the hardware's square
  // root and reciprocal (1 ulp each), a part in 10^7 of a step that is itself
  // a small part of p. The square root takes values below 2^-126 for 0.
  if (s.tiny_eps) {
#pragma unroll
    for (int k = 0; k < 4; ++k) p[k] = moved(widen(pr_[k]), s, s.rate * m[k] / (s.c2 * sqrtf(v[k]) + s.eps));
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      p[k] = moved(widen(pr_[k]), s,
                   s.rate * m[k] * __builtin_amdgcn_rcpf(s.c2 * __builtin_amdgcn_sqrtf(v[k]) + s.eps));
  }
  uint32_t rnd[4];
  if constexpr (EIGHT || sizeof(Tp) == 2) {
    const uint32_t key = mix_product((static_cast<uint32_t>(ch.tensor) + 1u + s.key) * kMix1);
    const uint32_t x = (static_cast<uint32_t>(ch.first) + static_cast<uint32_t>(i) + key) * kMix1;
#pragma unroll
    for (int k = 0; k < 4; ++k) rnd[k] = mix_product(x + static_cast<uint32_t>(k) * kMix1);
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
    store4<FULL, STREAM>(param, i, n, o);
  } else {
    store4<FULL, STREAM>(param, i, n, p);
    if (ch.copy) {
      uint16_t o[4];
      bf16_nearest(p, o);
      store4<FULL, STREAM>(ch.copy, i, n, o);
    }
  }
  if constexpr (EIGHT) {
    uint32_t mb[4], vb[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      mb[k] = FULL || i + k < n ? __float_as_uint(m[k]) & 0x7fffffffu : 0u;
      vb[k] = FULL || i + k < n ? __float_as_uint(v[k]) & 0x7fffffffu : 0u;
    }
    const uint32_t me = block_exponent<15>(wave_max_u(max(max(mb[0], mb[1]), max(mb[2], mb[3]))));
    const uint32_t ve = block_exponent<31>(wave_max_u(max(max(vb[0], vb[1]), max(vb[2], vb[3]))));
    const int32_t m0 = static_cast<int32_t>(code_base<15>(me)), v0 = static_cast<int32_t>(code_base<31>(ve));
    uint32_t mw = 0, vw = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      // 20 random bits round up with the probability of what they stand for.
      // A zero's code falls below 0 with the base (at least 8) and is 0 again.
      const int32_t mk = max(static_cast<int32_t>((mb[k] + (rnd[k] & 0xfffffu)) >> 20) - m0, 0);
      const int32_t vk = max(static_cast<int32_t>((vb[k] + (rnd[k] >> 12)) >> 20) - v0, 1);
      const uint32_t sign = m[k] < 0.0f ? 128u : 0u;
      mw |= ((static_cast<uint32_t>(mk) & 127u) | sign) << (8 * k);
      vw |= (vb[k] ? static_cast<uint32_t>(vk) & 255u : 0u) << (8 * k);
    }
    store_codes<FULL, STREAM>(static_cast<uint8_t*>(ch.m), i, n, mw);
    store_codes<FULL, STREAM>(static_cast<uint8_t*>(ch.v), i, n, vw);
    if (threadIdx.x % kWave == 0) {
      global(ch.m_exp)[b / kAdamBlock] = static_cast<uint8_t>(me);
      global(ch.v_exp)[b / kAdamBlock] = static_cast<uint8_t>(ve);
    }
  } else {
    store4<FULL, STREAM>(static_cast<float*>(ch.m), i, n, m);
    store4<FULL, STREAM>(static_cast<float*>(ch.v), i, n, v);
  }
}

// First element of the calling wave's block in turn k, as a scalar.
__device__ __forceinline__ int32_t wave_block(int k) {
  return (__builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave) + k * (kThreads / kWave)) * kAdamBlock;
}

struct NoGrads {};

template <typename Tp, typename Tg, bool EIGHT, bool STREAM, typename Grads>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const AdamChunk* chunks, AdamScalars s, Grads grads) {
  const AdamChunk& ch = chunks[blockIdx.x];
  const Tg* grad;
  if constexpr (sizeof(Grads) > sizeof(NoGrads)) {
    const void* g = grads.p[ch.tensor - grads.first];
    grad = g ? static_cast<const Tg*>(g) + ch.first : nullptr;
  } else {
    grad = static_cast<const Tg*>(ch.grad);
  }
  if (!grad) return;
#pragma unroll
  for (int k = 0; k < kTurns; ++k) {
    const int32_t b = wave_block(k);
    if (b + kAdamBlock <= ch.n)
      step_block<Tp, Tg, EIGHT, STREAM, true>(ch, grad, s, b);
    else if (b < ch.n)
      step_block<Tp, Tg, EIGHT, STREAM, false>(ch, grad, s, b);
  }
}

template <bool STREAM, bool FULL>
__device__ __forceinline__ void moments_block(const AdamChunk& ch, int32_t b, uint16_t* m_out, uint16_t* v_out) {
  const int32_t n = ch.n, i = b + static_cast<int32_t>(threadIdx.x % kWave) * kPer;
  const uint32_t mw = load_codes<FULL, STREAM>(static_cast<const uint8_t*>(ch.m), i, n);
  const uint32_t vw = load_codes<FULL, STREAM>(static_cast<const uint8_t*>(ch.v), i, n);
  const uint32_t me = global(ch.m_exp)[b / kAdamBlock], ve = global(ch.v_exp)[b / kAdamBlock];
  uint16_t mo[4], vo[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    // At most 4 significant bits: the upper half of the float32 holds the value.
    mo[k] = static_cast<uint16_t>((me == 255u ? kNanBits : __float_as_uint(decode_m(mw, k, code_base<15>(me)))) >> 16);
    vo[k] = static_cast<uint16_t>((ve == 255u ? kNanBits : __float_as_uint(decode_v(vw, k, code_base<31>(ve)))) >> 16);
  }
  store4<FULL, STREAM>(m_out + ch.block * kAdamBlock, i, n, mo);
  store4<FULL, STREAM>(v_out + ch.block * kAdamBlock, i, n, vo);
}

template <bool STREAM>
__global__ __launch_bounds__(kThreads) void adamw_moments_kernel(const AdamChunk* chunks, uint16_t* m_out,
                                                                 uint16_t* v_out) {
  const AdamChunk& ch = chunks[blockIdx.x];
#pragma unroll
  for (int k = 0; k < kTurns; ++k) {
    const int32_t b = wave_block(k);
    if (b + kAdamBlock <= ch.n)
      moments_block<STREAM, true>(ch, b, m_out, v_out);
    else if (b < ch.n)
      moments_block<STREAM, false>(ch, b, m_out, v_out);
  }
}

template <typename Tp, typename Tg, bool EIGHT, bool STREAM>
void launch(const AdamChunk* chunks, int64_t count, const AdamScalars& s, const AdamGrads* grads, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(count)), block(kThreads);
  if (grads)
    hipLaunchKernelGGL((adamw_kernel<Tp, Tg, EIGHT, STREAM, AdamGrads>), grid, block, 0, stream, chunks, s, *grads);
  else
    hipLaunchKernelGGL((adamw_kernel<Tp, Tg, EIGHT, STREAM, NoGrads>), grid, block, 0, stream, chunks, s, NoGrads{});
}

template <typename Tp, typename Tg>
void launch_kind(const AdamPlan& plan, int64_t at, int64_t count, const AdamScalars& s, const AdamGrads* grads,
                 hipStream_t stream) {
  const AdamChunk* c = plan.chunks + at;
  if (plan.state_bits == 8)
    plan.streamed ? launch<Tp, Tg, true, true>(c, count, s, grads, stream)
                  : launch<Tp, Tg, true, false>(c, count, s, grads, stream);
  else
    plan.streamed ? launch<Tp, Tg, false, true>(c, count, s, grads, stream)
                  : launch<Tp, Tg, false, false>(c, count, s, grads, stream);
}

// Workgroups of a launch: a grid holds less than 2^32 threads, so a plan of
// more than 8.6e9 elements takes several.
constexpr int64_t kMostGroups = (int64_t{1} << 31) / kThreads;

}  // namespace

hipError_t launch_adamw(const AdamPlan& plan, int64_t begin, int64_t end, const AdamScalars& s, const AdamGrads* grads,
                        hipStream_t stream) {
  for (int64_t at = begin; at < end; at += kMostGroups) {
    const int64_t k = end - at < kMostGroups ? end - at : kMostGroups;
    const bool p16 = plan.param_dtype == PR_BF16, g16 = plan.grad_dtype == PR_BF16;
    if (p16 && g16)
      launch_kind<uint16_t, uint16_t>(plan, at, k, s, grads, stream);
    else if (p16)
      launch_kind<uint16_t, float>(plan, at, k, s, grads, stream);
    else if (g16)
      launch_kind<float, uint16_t>(plan, at, k, s, grads, stream);
    else
      launch_kind<float, float>(plan, at, k, s, grads, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_adamw_moments(const AdamPlan& plan, int64_t n_chunks, uint16_t* m, uint16_t* v, hipStream_t stream) {
  for (int64_t at = 0; at < n_chunks; at += kMostGroups) {
    const int64_t k = n_chunks - at < kMostGroups ? n_chunks - at : kMostGroups;
    if (plan.streamed)
      hipLaunchKernelGGL(adamw_moments_kernel<true>, dim3(static_cast<unsigned>(k)), dim3(kThreads), 0, stream,
                         plan.chunks + at, m, v);
    else
      hipLaunchKernelGGL(adamw_moments_kernel<false>, dim3(static_cast<unsigned>(k)), dim3(kThreads), 0, stream,
                         plan.chunks + at, m, v);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace pr
