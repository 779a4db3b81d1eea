// Activations, their slopes and the 8-bit form of saved activations, as the linear layers' kernels use them
// (include/smat.h defines both).
#pragma once

#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "smat.h"

namespace smat {
namespace lin {

constexpr int kGroup = SMAT_PACK8_GROUP;

// Activations of bf16 calls go by the hardware's 2^x and 1 / x, 2 ulp and 1 ulp, results below 2^-126 flushed to 0: one
// instruction each, where expf and a division are 6 to 10. A product's epilogue makes a value per sum, and its instructions
// bound it; a result's rounding to bf16 hides their error. Those of fp32 calls, whose results would show it, are right to a
// few units in the last place. Memory bounds those mostly: 8191 x 4096 read back through none 27.3 us, silu 28.5, GELU 33.3 (with
// the forms for bf16 28.1 and 29.9), with rows off every boundary 8191 x 1100 14.7, 18.2 and 20.9 (16.4 and 19.4).
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_fast(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

constexpr float kLog2e = 1.4426950408889634f;

// sigmoid(c x) with its limits at infinities. The exponent is one fp32 number: relative error (1.5 |c x| + 4) 2^-23, 5e-7 near
// 0 and 5e-6 at -20, down to 2^-126 (c x = -87), below which it is 0. The activations with a sigmoid form use it, the tanh form
// of GELU too (1 + tanh u = 2 sigmoid(2u)), so that small values far out on the negative side keep their digits.
__device__ __forceinline__ float sigmoid_fast(float x, float c) { return rcp_fast(1.0f + exp2_fast(-c * kLog2e * x)); }

// sigmoid(x) and sigmoid(x) sigmoid(-x), by e = exp(-|x|), which never overflows: 8 2^-24 relative and 5 more, of an x that is
// exact, down to where e is below 2^-126
struct Sigmoid {
  float s, slope;
};
__device__ __forceinline__ Sigmoid sigmoid_full(float x) {
  const float e = expf(-fabsf(x)), r = rcp_fast(1.0f + e);
  return {x < 0.0f ? e * r : r, e * r * r};
}

// Phi(h) = exp(-h^2 / 2) t Q(t), t = 1 / (1 + 0.35 |h|), taken from the side where it is small; Q and its error, 5 2^-24
// relative with its roundings, by fit_normal_cdf.py. With the reciprocal (2) and the exponential (4, and 1.5 h^2 for the
// roundings of its argument, which expf would have nearly all too) (13 + 1.5 h^2) 2^-24, down to 2^-126; `g` = exp(-h^2 / 2).
// CUDA's normcdff takes 71 us to read 8191 x 4096 back through GELU, with expf here it was 41.
__device__ __forceinline__ float normal_cdf(float h, float& g) {
  const float t = rcp_fast(fmaf(0.35f, fabsf(h), 1.0f));
  g = exp2_fast(h * h * (-0.5f * kLog2e));
  float s = fmaf(t, -0.0291206744f, 0.143846497f);
  s = fmaf(s, t, -0.255450249f);
  s = fmaf(s, t, 0.158865809f);
  s = fmaf(s, t, -0.0228923205f);
  s = fmaf(s, t, 0.105413429f);
  s = fmaf(s, t, 0.119857527f);
  s = fmaf(s, t, 0.13985835f);
  s = fmaf(s, t, 0.139621615f);
  s = s * t * g;
  return h > 0.0f ? 1.0f - s : s;
}

// Phi(h) by Abramowitz and Stegun 7.1.26 (erfc(z) = t (a1 + t (a2 + ...)) exp(-z^2), t = 1 / (1 + p z), z = |h| /
// sqrt2; off by 1.5e-7 at most, so Phi by 0.75e-7), taken from the side where it is small; `g` = exp(-h^2 / 2). In the tail
// that is 0.16% of Phi at -5, 1% at -8 and 3.7% at -13: fewer digits than a bf16 result has from -6.2 on.
__device__ __forceinline__ float normal_cdf_fast(float h, float& g) {
  const float t = rcp_fast(fmaf(0.3275911f * 0.70710678f, fabsf(h), 1.0f));
  g = exp2_fast(h * h * (-0.5f * kLog2e));
  float s = fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
  s = fmaf(s, t, 0.5f * 1.421413741f);
  s = fmaf(s, t, 0.5f * -0.284496736f);
  s = fmaf(s, t, 0.5f * 0.254829592f);
  s = s * t * g;
  return h > 0.0f ? 1.0f - s : s;
}

constexpr float kTanhGain = 1.5957691216057308f;  // 2 sqrt(2 / pi)
constexpr float kTanhCube = 0.044715f;

// T: the call's type
template <int ACT, class T>
__device__ __forceinline__ float act_value(float h) {
  constexpr bool kFull = sizeof(T) == 4;
  if (ACT == SMAT_ACT_RELU) return h > 0.0f || h != h ? h : 0.0f;
  if (ACT == SMAT_ACT_GELU) {
    float g;
    return h * (kFull ? normal_cdf(h, g) : normal_cdf_fast(h, g));
  }
  if (ACT == SMAT_ACT_GELU_TANH) {
    const float x = h * fmaf(kTanhCube, h * h, 1.0f);
    return h * (kFull ? sigmoid_full(kTanhGain * x).s : sigmoid_fast(x, kTanhGain));
  }
  if (ACT == SMAT_ACT_QUICK_GELU) return h * (kFull ? sigmoid_full(1.702f * h).s : sigmoid_fast(h, 1.702f));
  if (ACT == SMAT_ACT_SILU) return h * (kFull ? sigmoid_full(h).s : sigmoid_fast(h, 1.0f));
  return h;
}

// act'. Beyond +-200 every slope here is 0 or 1 in fp32; h is held there, so that an infinity or a huge h gives
// the limit and not inf * 0. NaN stays NaN.
template <int ACT, class T>
__device__ __forceinline__ float act_slope(float h) {
  constexpr bool kFull = sizeof(T) == 4;
  if (ACT == SMAT_ACT_RELU) return h > 0.0f ? 1.0f : (h != h ? h : 0.0f);
  if (ACT == SMAT_ACT_NONE) return 1.0f;
  asm("min.NaN.f32 %0, %0, 0f43480000;\nmax.NaN.f32 %0, %0, 0fC3480000;" : "+f"(h));
  if (ACT == SMAT_ACT_GELU) {
    float g;
    const float c = kFull ? normal_cdf(h, g) : normal_cdf_fast(h, g);
    return fmaf(h * 0.39894228040143268f, g, c);
  }
  if (ACT == SMAT_ACT_GELU_TANH) {
    const float u = h * h, x = h * fmaf(kTanhCube, u, 1.0f), by = h * fmaf(3.0f * kTanhCube * kTanhGain, u, kTanhGain);
    if (kFull) {
      const Sigmoid t = sigmoid_full(kTanhGain * x);
      return fmaf(by, t.slope, t.s);
    }
    const float s = sigmoid_fast(x, kTanhGain);
    return fmaf(by, fmaf(-s, s, s), s);
  }
  const float c = ACT == SMAT_ACT_QUICK_GELU ? 1.702f : 1.0f;
  if (kFull) {
    const Sigmoid t = sigmoid_full(c * h);
    return fmaf(c * h, t.slope, t.s);
  }
  const float s = sigmoid_fast(h, c);
  return fmaf(c * h, fmaf(-s, s, s), s);
}

// Runs the statement with ACT one of the six activations: the branch is taken once per block of elements.
#define SMAT_WITH_ACT(act, ...)                                                                  \
  switch (act) {                                                                                 \
    case SMAT_ACT_RELU: { constexpr int ACT = SMAT_ACT_RELU; __VA_ARGS__; } break;               \
    case SMAT_ACT_GELU: { constexpr int ACT = SMAT_ACT_GELU; __VA_ARGS__; } break;               \
    case SMAT_ACT_GELU_TANH: { constexpr int ACT = SMAT_ACT_GELU_TANH; __VA_ARGS__; } break;     \
    case SMAT_ACT_QUICK_GELU: { constexpr int ACT = SMAT_ACT_QUICK_GELU; __VA_ARGS__; } break;   \
    case SMAT_ACT_SILU: { constexpr int ACT = SMAT_ACT_SILU; __VA_ARGS__; } break;               \
    default: { constexpr int ACT = SMAT_ACT_NONE; __VA_ARGS__; } break;                          \
  }

// The 8-bit form's byte e of a group whose largest magnitude has the bits `top` (sign bit clear): the largest
// value's exponent less 6, and one more where it would round to 128 (its significand is at least 127.5 / 64, the
// bits 0x7F0000: the addition carries into the exponent from there on); at least 1; 255 for infinities and NaN.
__device__ __forceinline__ uint32_t pack_exponent(uint32_t top) {
  const int e = (int)((top + 0x10000u) >> 23) - 6;
  return top >= 0x7F800000u ? 255u : (uint32_t)(e < 1 ? 1 : e);
}

// q of a value in the low byte (the others hold something else), the factor being 2^(127 - e): the product is exact,
// or far below 1/2, and its rounding to a whole number, ties to even, is
// that of an addition to 1.5 * 2^23, whose last place is 1. In a group of e = 255 it is not q: see pack_poisoned.
__device__ __forceinline__ uint32_t pack_value(float x, float factor) {
  return __float_as_uint(fmaf(x, factor, 12582912.0f));
}

// q in a group that holds an infinity or NaN: +-127 for infinities, 0 for the rest
__device__ __forceinline__ uint32_t pack_poisoned(float x) {
  return fabsf(x) == __int_as_float(0x7F800000) ? (x > 0.0f ? 127u : 129u) : 0u;
}

// the low bytes of four words
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

// 4 * WORDS values' q
template <int WORDS>
__device__ __forceinline__ void pack_words(const float* v, uint32_t e, uint32_t* w) {
  if (e == 255u) {
#pragma unroll
    for (int i = 0; i < WORDS; ++i, v += 4)
      w[i] = low_bytes(pack_poisoned(v[0]), pack_poisoned(v[1]), pack_poisoned(v[2]), pack_poisoned(v[3]));
    return;
  }
  const float f = __uint_as_float((254u - e) << 23);
#pragma unroll
  for (int i = 0; i < WORDS; ++i, v += 4)
    w[i] = low_bytes(pack_value(v[0], f), pack_value(v[1], f), pack_value(v[2], f), pack_value(v[3], f));
}
__device__ __forceinline__ uint32_t pack_one(float x, uint32_t e) {
  return e == 255u ? pack_poisoned(x) : pack_value(x, __uint_as_float((254u - e) << 23));
}

// The larger magnitude; NaN if one is (as bits: larger than infinity's).
__device__ __forceinline__ float larger(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(fabsf(a)), "f"(fabsf(b)));
  return y;
}

// 2^(e - 127); infinity for e = 255 (q = 0 then reads as NaN, +-127 as +-infinity).
__device__ __forceinline__ float unpack_scale(uint32_t e) { return __uint_as_float(e << 23); }

// The values of 4 * WORDS q. 2^23 + 128 + q is a float whose last place is 1: a byte of q + 128 put into 2^23's bits;
// what is left is one multiply-add, exact like the product (a conversion from an integer runs at an eighth of its
// rate). Where 2^23 times the scale could overflow, from e = 230 on, and for e = 255, the product it is.
template <int WORDS>
__device__ __forceinline__ void unpack_words8(const uint32_t* w, uint32_t e, float* v) {
  const float by = unpack_scale(e);
  if (e >= 230u) {
#pragma unroll
    for (int i = 0; i < 4 * WORDS; ++i) v[i] = (float)(int8_t)(w[i / 4] >> (8 * (i % 4))) * by;
    return;
  }
  const float less = -8388736.0f * by;
#pragma unroll
  for (int i = 0; i < 4 * WORDS; ++i)
    v[i] = fmaf(__uint_as_float(__byte_perm(w[i / 4] ^ 0x80808080u, 0x4B000000u, 0x7540 | (i % 4))), by, less);
}

// Thread-block cluster: a barrier of all its threads (with release and acquire of shared memory), and a float of
// the shared memory of its CTA `rank`, at the place that `p` has here.
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The barrier alone: for an end at which nobody reads what others wrote (a release would wait for every store to memory).
__device__ __forceinline__ void cluster_meet() {
  asm volatile("barrier.cluster.arrive.relaxed.aligned;\nbarrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_address(const void* p, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ float cluster_load(const float* p, uint32_t rank) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_address(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ float4 cluster_load4(uint32_t address) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(address)
               : "memory");
  return v;
}

template <class T>
__device__ __forceinline__ float to_float(T v);
template <>
__device__ __forceinline__ float to_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

}  // namespace lin
}  // namespace smat
