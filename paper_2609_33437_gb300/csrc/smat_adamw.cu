// One AdamW step over a list of tensors, moments in 32 bits or in 8 (include/smat.h, "AdamW").
//
// A warp takes a group of 256 neighbours at a time, 8 a lane, so that the largest magnitudes of a group in 8 bits are one
// reduction over the warp. Every CTA walks through a stretch of the list's groups; the tensors' addresses come with the launch
// (no table on the device, nothing to copy), and a warp looks for its tensor once and then goes on from it.

#include "smat_adamw.h"

#include <type_traits>

#include "smat_linear.cuh"

namespace smat {
namespace adamw {
namespace {

using bf16 = __nv_bfloat16;
using lin::from_float;
using lin::to_float;

constexpr int kWarps = 8, kEach = kGroup / 32;
static_assert(kEach == 8, "a lane's elements");

template <int N>
struct Launch {
  Call c;
  Entry entries[N];
};

// 8 neighbours
template <class T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  } else {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
template <class T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// A code of PLACES binary places is a small float: its upper bits an exponent, 0 for multiples of the unit. At the places of an
// fp32 number's exponent and fraction it is its value times 2^-(126 + PLACES) (a subnormal number where the exponent is 0), so
// two exact products make the value: by 2^127, and by 2^(PLACES - 1) and the unit. e = 255 stands for NaN: 0 by infinity.
template <int PLACES>
__device__ __forceinline__ float unit_of(uint32_t e) {
  return __uint_as_float(min(e + PLACES - 1, 255u) << 23);
}
template <int PLACES>
__device__ __forceinline__ float value_of(uint32_t code, float unit) {
  return __fmul_rn(__fmul_rn(__uint_as_float(code << (23 - PLACES)), 0x1p127f), unit);
}
// The code of v >= 0, `inverse` being 1 / unit: the neighbour below, or the one above if the place between the two plus the
// 16 bits of `part` reaches 1.
template <int PLACES>
__device__ __forceinline__ uint32_t code_of(float v, float inverse, uint32_t part) {
  const float f = __fmul_rn(v, inverse);
  const int at = max((int)(__float_as_uint(f) >> 23) - 127 - PLACES, 0);
  const float by = __uint_as_float((uint32_t)(127 - at) << 23);
  const float u = __uint_as_float(0x3F800000u | part << 7) - (1.0f - 0x1p-17f);  // (part + 1/2) 2^-16, exactly
  // its whole part: the low bits of a sum with 2^23, rounded down
  const uint32_t whole = __float_as_uint(__fadd_rd(__fadd_rn(__fmul_rn(f, by), u), 8388608.0f)) & 0xFFu;
  return ((uint32_t)at << PLACES) + whole;
}
// e of a group whose largest magnitude has the bits `top`
__device__ __forceinline__ uint32_t exponent_of(uint32_t top, int less) {
  return top >= 0x7F800000u ? 255u : (uint32_t)max((int)(top >> 23) - less, 1);
}

// m1, m2 and the parameter, each operation rounded (as smat_grad_map_adamw_multi does it).
__device__ __forceinline__ void moments(const Constants& c, float g, float& m1, float& m2) {
  m1 = __fadd_rn(__fmul_rn(c.b1, m1), __fmul_rn(c.omb1, g));
  m2 = __fadd_rn(__fmul_rn(c.b2, m2), __fmul_rn(c.omb2, __fmul_rn(g, g)));
}
__device__ __forceinline__ float updated(const Constants& c, float p, float m1, float r) {
  const float d = __fadd_rn(__fdiv_rn(r, c.bc2), c.eps);
  return __fsub_rn(__fmul_rn(p, c.decay), __fmul_rn(c.step, __fdiv_rn(m1, d)));
}

template <int BITS, class P, class G, int N>
__global__ void __launch_bounds__(32 * kWarps) step_kernel(const __grid_constant__ Launch<N> a) {
  __shared__ Constants shared_c;
  __shared__ uint32_t shared_key;
  Constants c = a.c.c;
  uint32_t key = a.c.key;
  if (a.c.step_at || a.c.lr_at) {  // what the device knows
    if (threadIdx.x == 0) {
      const double lr = a.c.lr_at ? (double)*a.c.lr_at : a.c.lr;
      if (a.c.step_at) {
        const double t = (double)*a.c.step_at;
        c.step = (float)(lr / -expm1(t * a.c.log_b1));
        c.bc2 = (float)sqrt(-expm1(t * a.c.log_b2));
        key = mix(mix(a.c.seed_key ^ (uint32_t)*a.c.step_at));
      } else {
        c.step = (float)(lr / a.c.bc1);
      }
      c.decay = (float)(1.0 - lr * a.c.weight_decay);
      shared_c = c, shared_key = key;
    }
    __syncthreads();
    c = shared_c, key = shared_key;
  }
  const float scale = a.c.scale_at ? *a.c.scale_at : a.c.scale;
  const int lane = threadIdx.x % 32;
  const uint32_t begin = (uint32_t)((uint64_t)a.c.groups * blockIdx.x / gridDim.x);
  const uint32_t end = (uint32_t)((uint64_t)a.c.groups * (blockIdx.x + 1) / gridDim.x);
  uint32_t group = begin + threadIdx.x / 32;
  if (group >= end) return;
  int at = 0;
  for (int high = a.c.n; high - at > 1;) {  // entries[at].first <= group < entries[high].first
    const int mid = (at + high) / 2;
    if (a.entries[mid].first <= group)
      at = mid;
    else
      high = mid;
  }
  for (; group < end; group += kWarps) {
    while (at + 1 < a.c.n && a.entries[at + 1].first <= group) ++at;
    const Entry& e = a.entries[at];
    const uint32_t after = at + 1 < a.c.n ? a.entries[at + 1].first : a.c.groups;
    const int count = kGroup - (group + 1 == after ? e.lacks : 0);  // of this group's elements
    const int64_t in = (int64_t)(group - e.first) * kGroup + lane * kEach, place = (int64_t)group * kGroup + lane * kEach;
    P* pp = (P*)e.p + in;
    const G* gp = (const G*)e.g + in;
    const int mine = min(max(count - lane * kEach, 0), kEach);
    const bool fast = e.whole && mine == kEach;
    float p[8], g[8], m1[8], m2[8];
    uint2 q1, q2;
    uint32_t x1, x2;
    if constexpr (BITS == 8) {
      q1 = *reinterpret_cast<const uint2*>((const uint8_t*)a.c.m1 + place);
      q2 = *reinterpret_cast<const uint2*>((const uint8_t*)a.c.m2 + place);
      x1 = a.c.e1[group];
      x2 = a.c.e2[group];
    } else {
      load8((const float*)a.c.m1 + place, m1);
      load8((const float*)a.c.m2 + place, m2);
    }
    if (fast) {
      load8(pp, p);
      load8(gp, g);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = i < mine ? to_float(pp[i]) : 0.0f;
        g[i] = i < mine ? to_float(gp[i]) : 0.0f;
      }
    }
    if constexpr (BITS == 8) {
      const float u1 = unit_of<3>(x1), u2 = unit_of<4>(x2);
      uint32_t top1 = 0, top2 = 0;
      float r[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t b1 = (i < 4 ? q1.x : q1.y) >> 8 * (i % 4), b2 = (i < 4 ? q2.x : q2.y) >> 8 * (i % 4);
        m1[i] = __uint_as_float(__float_as_uint(value_of<3>(b1 & 127u, u1)) | (b1 & 128u) << 24);
        r[i] = value_of<4>(b2 & 255u, u2);
        m2[i] = __fmul_rn(r[i], r[i]);
        moments(c, __fmul_rn(g[i], scale), m1[i], m2[i]);
        if (i >= mine) m1[i] = m2[i] = 0.0f;
        r[i] = __fsqrt_rn(m2[i]);
        top1 = max(top1, __float_as_uint(m1[i]) & 0x7FFFFFFFu);
        top2 = max(top2, __float_as_uint(r[i]) & 0x7FFFFFFFu);
        p[i] = updated(c, p[i], m1[i], r[i]);
      }
      top1 = __reduce_max_sync(0xFFFFFFFFu, top1);
      top2 = __reduce_max_sync(0xFFFFFFFFu, top2);
      x1 = exponent_of(top1, 16), x2 = exponent_of(top2, 17);
      uint32_t w1[2] = {0, 0}, w2[2] = {0, 0};
      const float v1 = __uint_as_float((254u - min(x1, 253u)) << 23), v2 = __uint_as_float((254u - min(x2, 253u)) << 23);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t d = mix((uint32_t)(a.c.place + place + i) ^ key);
        const uint32_t c1 = code_of<3>(fabsf(m1[i]), v1, d & 0xFFFFu) | (m1[i] < 0.0f ? 128u : 0u);
        const uint32_t c2 = code_of<4>(r[i], v2, d >> 16);
        w1[i / 4] |= (x1 == 255u ? 0u : c1) << 8 * (i % 4);
        w2[i / 4] |= (x2 == 255u ? 0u : c2) << 8 * (i % 4);
      }
      *reinterpret_cast<uint2*>((uint8_t*)a.c.m1 + place) = make_uint2(w1[0], w1[1]);
      *reinterpret_cast<uint2*>((uint8_t*)a.c.m2 + place) = make_uint2(w2[0], w2[1]);
      if (lane == 0) a.c.e1[group] = (uint8_t)x1, a.c.e2[group] = (uint8_t)x2;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        moments(c, __fmul_rn(g[i], scale), m1[i], m2[i]);
        p[i] = updated(c, p[i], m1[i], __fsqrt_rn(m2[i]));
      }
      if (mine == kEach) {
        store8((float*)a.c.m1 + place, m1);
        store8((float*)a.c.m2 + place, m2);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < mine) ((float*)a.c.m1)[place + i] = m1[i], ((float*)a.c.m2)[place + i] = m2[i];
      }
    }
    if (fast) {
      store8(pp, p);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < mine) pp[i] = from_float<P>(p[i]);
    }
  }
}

// What 8 bits stand for, in bf16, which holds it exactly.
__global__ void __launch_bounds__(256) values_kernel(const uint8_t* q1, const uint8_t* e1, const uint8_t* q2, const uint8_t* e2,
                                                     bf16* m1, bf16* r, int64_t places) {
  for (int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8; at < places; at += (int64_t)gridDim.x * 256 * 8) {
    const uint2 a = *reinterpret_cast<const uint2*>(q1 + at), b = *reinterpret_cast<const uint2*>(q2 + at);
    const float u1 = unit_of<3>(e1[at / kGroup]), u2 = unit_of<4>(e2[at / kGroup]);
    float v[8], w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t b1 = (i < 4 ? a.x : a.y) >> 8 * (i % 4), b2 = (i < 4 ? b.x : b.y) >> 8 * (i % 4);
      v[i] = __uint_as_float(__float_as_uint(value_of<3>(b1 & 127u, u1)) | (b1 & 128u) << 24);
      w[i] = value_of<4>(b2 & 255u, u2);
    }
    store8(m1 + at, v);
    store8(r + at, w);
  }
}

template <int BITS, class P, class G, int N>
cudaError_t launch_of(const Call& c, const Entry* entries, int sms, cudaStream_t s) {
  Launch<N> a;
  a.c = c;
  for (int i = 0; i < c.n; ++i) a.entries[i] = entries[i];
  const int64_t sets = ((int64_t)c.groups + kWarps - 1) / kWarps, room = (int64_t)sms * 4;
  step_kernel<BITS, P, G, N><<<(unsigned)(sets < room ? sets : room), 32 * kWarps, 0, s>>>(a);
  return cudaGetLastError();
}
template <int BITS, class P, class G>
cudaError_t launch_sized(const Call& c, const Entry* entries, int sms, cudaStream_t s) {
  if (c.n <= 32) return launch_of<BITS, P, G, 32>(c, entries, sms, s);
  if (c.n <= 320) return launch_of<BITS, P, G, 320>(c, entries, sms, s);
  return launch_of<BITS, P, G, kMaxEntries>(c, entries, sms, s);
}
template <int BITS>
cudaError_t launch_typed(const Call& c, const Entry* entries, int dtype, int grad_dtype, int sms, cudaStream_t s) {
  if (dtype == SMAT_F32 && grad_dtype == SMAT_F32) return launch_sized<BITS, float, float>(c, entries, sms, s);
  if (dtype == SMAT_F32) return launch_sized<BITS, float, bf16>(c, entries, sms, s);
  if (grad_dtype == SMAT_F32) return launch_sized<BITS, bf16, float>(c, entries, sms, s);
  return launch_sized<BITS, bf16, bf16>(c, entries, sms, s);
}

}  // namespace

cudaError_t launch_step(const Call& c, const Entry* entries, int dtype, int grad_dtype, int bits, int sms, cudaStream_t s) {
  return bits == 8 ? launch_typed<8>(c, entries, dtype, grad_dtype, sms, s)
                   : launch_typed<32>(c, entries, dtype, grad_dtype, sms, s);
}

cudaError_t launch_values(const uint8_t* q1, const uint8_t* e1, const uint8_t* q2, const uint8_t* e2, void* m1, void* r,
                          int64_t places, int sms, cudaStream_t s) {
  const int64_t sets = (places + 2047) / 2048, room = (int64_t)sms * 8;
  values_kernel<<<(unsigned)(sets < room ? sets : room), 256, 0, s>>>(q1, e1, q2, e2, (bf16*)m1, (bf16*)r, places);
  return cudaGetLastError();
}

}  // namespace adamw
}  // namespace smat
