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

// sigmoid by the hardware's exponential (2 ulp) and reciprocal: 1e-6 relative over the whole range, and its
// limits at infinities. Every activation below that has a sigmoid form uses it, the tanh form of GELU too
// (1 + tanh u = 2 sigmoid(2u)), so that small values far out on the negative side keep their digits.
__device__ __forceinline__ float sigmoid(float x) { return __fdividef(1.0f, 1.0f + __expf(-x)); }

constexpr float kTanhGain = 1.5957691216057308f;  // 2 sqrt(2 / pi)
constexpr float kTanhCube = 0.044715f;

template <int ACT>
__device__ __forceinline__ float act_value(float h) {
  if (ACT == SMAT_ACT_RELU) return h > 0.0f || h != h ? h : 0.0f;
  if (ACT == SMAT_ACT_GELU) return 0.5f * h * erfcf(-0.70710678118654752f * h);
  if (ACT == SMAT_ACT_GELU_TANH) return h * sigmoid(kTanhGain * h * fmaf(kTanhCube, h * h, 1.0f));
  if (ACT == SMAT_ACT_QUICK_GELU) return h * sigmoid(1.702f * h);
  if (ACT == SMAT_ACT_SILU) return h * sigmoid(h);
  return h;
}

// act'. Beyond +-100 every slope here is 0 or 1 in fp32; h is held there, so that an infinity or a huge h gives
// the limit and not inf * 0. NaN stays NaN.
template <int ACT>
__device__ __forceinline__ float act_slope(float h) {
  if (ACT == SMAT_ACT_RELU) return h > 0.0f ? 1.0f : (h != h ? h : 0.0f);
  if (ACT == SMAT_ACT_NONE) return 1.0f;
  h = h > 100.0f ? 100.0f : (h < -100.0f ? -100.0f : h);
  if (ACT == SMAT_ACT_GELU)
    return fmaf(h * 0.39894228040143268f, __expf(-0.5f * h * h), 0.5f * erfcf(-0.70710678118654752f * h));
  if (ACT == SMAT_ACT_GELU_TANH) {
    const float s = sigmoid(kTanhGain * h * fmaf(kTanhCube, h * h, 1.0f));
    return fmaf(h * kTanhGain * fmaf(3.0f * kTanhCube, h * h, 1.0f), s * (1.0f - s), s);
  }
  const float c = ACT == SMAT_ACT_QUICK_GELU ? 1.702f : 1.0f;
  const float s = sigmoid(c * h);
  return fmaf(c * h, s * (1.0f - s), s);
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

// 2^(127 - e), by which a value is multiplied before it is rounded. The products are exact (or far below 1/2).
// For e = 255 the factor is 0: 0 for finite values, NaN for infinities and NaN, which pack_value sorts out.
__device__ __forceinline__ float pack_factor(uint32_t e) {
  return e == 255u ? 0.0f : __uint_as_float((254u - e) << 23);
}

// q of one value, in the low byte.
__device__ __forceinline__ uint32_t pack_value(float x, float factor) {
  if (factor == 0.0f) return fabsf(x) == __int_as_float(0x7F800000) ? (x > 0.0f ? 127u : 129u) : 0u;
  return (uint32_t)__float2int_rn(x * factor) & 0xFFu;
}

// 2^(e - 127); infinity for e = 255 (q = 0 then reads as NaN, +-127 as +-infinity).
__device__ __forceinline__ float unpack_scale(uint32_t e) { return __uint_as_float(e << 23); }

__device__ __forceinline__ float unpack_value(uint32_t word, int byte, float scale) {
  return (float)(int8_t)(word >> (8 * byte)) * scale;
}

// Thread-block cluster: a barrier of all its threads (with release and acquire of shared memory), and a float of
// the shared memory of its CTA `rank`, at the place that `p` has here.
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
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
__device__ __forceinline__ float4 cluster_load4(const float* p, uint32_t rank) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(cluster_address(p, rank))
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
