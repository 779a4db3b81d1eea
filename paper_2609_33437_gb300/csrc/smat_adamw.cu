// One AdamW step over a list of tensors, moments in 32 bits or in 8 (include/smat.h, "AdamW").
//
// A warp takes a group of 256 neighbours at a time, 8 a lane, so that the largest magnitudes of a group in 8 bits are one
// reduction over the warp. All CTAs walk through the list side by side, 8 groups each at a time (a stretch of its own for each:
// 1,500 us for 315e6 elements in fp32, 5.9 TB/s; like this 1,360 us, 6.5 TB/s, which is memory's rate); the tensors' addresses
// come with the launch (no table on the device, nothing to copy), and a warp looks for its tensor once and then goes on from it.
//
// With moments in 8 bits memory is not what bounds it: 147e6 elements of bf16 370 us (4.0 TB/s; the issue slots are 75% busy, 76
// instructions an element). Codes by exponents and shifts of every value took 480 us, with divisions too 580; five CTAs per SM
// instead of four (48 registers) 375.

#include "smat_adamw.h"

#include <type_traits>

#include "smat_linear.cuh"

namespace smat {
namespace adamw {
namespace {

using bf16 = __nv_bfloat16;
using lin::from_float;
using lin::to_float;

constexpr int kWarps = 8, kCtas = 4, kEach = kGroup / 32;
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
    asm volatile("ld.global.L1::no_allocate.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
                 : "l"(p)
                 : "memory");
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
    asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
                 "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
                 : "memory");
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

// Two fp32 numbers, which one instruction multiplies. (Not for sums that have to be rounded by themselves: the compiler makes one
// instruction of a product and a sum of pairs, whatever rounding they name.)
struct Two {
  uint64_t u;
  __device__ __forceinline__ Two() {}
  __device__ __forceinline__ Two(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(u) : "f"(a), "f"(b)); }
  __device__ __forceinline__ explicit Two(float a) : Two(a, a) {}
  __device__ __forceinline__ void apart(float& a, float& b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(u)); }
};
__device__ __forceinline__ Two operator*(Two a, Two b) {
  Two y;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(y.u) : "l"(a.u), "l"(b.u));
  return y;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
  Two y;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y.u) : "l"(a.u), "l"(b.u), "l"(c.u));
  return y;
}

// A code of PLACES binary places is a small float: its upper bits an exponent, 0 for multiples of the unit. At the places of an
// fp32 number's exponent and fraction it is its value times 2^-(126 + PLACES) (a subnormal number where the exponent is 0), so an
// exact product makes the value: by 2^(126 + PLACES) times the unit, 2^(e + PLACES - 1). For large units that is no fp32 number
// and takes two factors (`far`); e = 255 stands for NaN: 0 by infinity.
__device__ __forceinline__ float float_of(uint32_t bits) { return __uint_as_float(bits); }
template <int PLACES>
struct Unit {
  float by, more;
  __device__ __forceinline__ Unit(uint32_t e, bool far)
      : by(far ? 0x1p127f : float_of((e + PLACES + 126u) << 23)), more(float_of(min(e + PLACES - 1, 255u) << 23)) {}
  __device__ __forceinline__ void operator()(float a, float b, bool far, float& x, float& y) const {
    Two v = Two(a, b) * Two(by);
    if (far) v = v * Two(more);
    v.apart(x, y);
  }
};
__device__ __forceinline__ bool far_units(uint32_t e1, uint32_t e2) { return max(e1, e2) > 120u; }
// Byte i of four as such a float: m1's has a sign before 7 bits, r's 8 bits.
__device__ __forceinline__ float signed_code(uint32_t w, int i) {
  return __int_as_float((int)__byte_perm(w, 0, i << 12 | 0x0444) >> 4 & (int)0x87F00000u);
}
__device__ __forceinline__ float plain_code(uint32_t w, int i) { return __uint_as_float(__byte_perm(w, 0, i << 12 | 0x0444) >> 5); }

// A code is the upper bits of an fp32 number: of v >= 0 itself from the first full-precision code on (B = 2^(e + PLACES - 127)), of
// v + B less an exponent's step below; the larger of the two numbers (as bits) is the right one on either side of B. v + B is
// rounded down, and what is below the code's last place is a fraction of 23 - PLACES bits to which the 16 bits of `part`, and a
// half of their last one, are added: a carry is the neighbour above. The result's upper byte is the code. part: the 16 bits in
// the middle of a word.
template <int PLACES>
struct Coder {
  float first;
  uint32_t off;
  __device__ __forceinline__ explicit Coder(uint32_t e)
      : first(float_of((e + PLACES) << 23)), off(128u - ((e + PLACES - 1) << 23 << (PLACES + 1))) {}
  __device__ __forceinline__ uint32_t operator()(float v, uint32_t part) const {
    const uint32_t low = __float_as_uint(__fadd_rd(v, first)) - (1u << 23);
    return max(low, __float_as_uint(v)) * (2u << PLACES) + (part + off);
  }
};
// The upper bytes of four words
__device__ __forceinline__ uint32_t upper_bytes(const uint32_t* w) {
  return __byte_perm(__byte_perm(w[0], w[1], 0x0073), __byte_perm(w[2], w[3], 0x0073), 0x5410);
}
// The largest magnitude; NaN if one is.
__device__ __forceinline__ float larger_of(float a, float b, float c) {
  float y;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(fabsf(b)), "f"(fabsf(c)));
  return y;
}
// e of a group whose largest magnitude has the bits `top`
__device__ __forceinline__ uint32_t exponent_of(uint32_t top, int less) {
  return top >= 0x7F800000u ? 255u : (uint32_t)max((int)(top >> 23) - less, 1);
}

// m1 and m2, each operation rounded (as smat_grad_map_adamw_multi does it).
__device__ __forceinline__ void moments(const Constants& c, float g, float& m1, float& m2) {
  m1 = __fadd_rn(__fmul_rn(c.b1, m1), __fmul_rn(c.omb1, g));
  m2 = __fadd_rn(__fmul_rn(c.b2, m2), __fmul_rn(c.omb2, __fmul_rn(g, g)));
}
// The parameter, with moments in 32 bits, rounded like them.
__device__ __forceinline__ float updated(const Constants& c, float p, float m1, float r) {
  const float d = __fadd_rn(__fdiv_rn(r, c.bc2), c.eps);
  return __fsub_rn(__fmul_rn(p, c.decay), __fmul_rn(c.step, __fdiv_rn(m1, d)));
}

template <int BITS, class P, class G, int N>
__global__ void __launch_bounds__(32 * kWarps, kCtas) step_kernel(const __grid_constant__ Launch<N> a) {
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
        const double root = sqrt(-expm1(t * a.c.log_b2));
        c.bc2 = (float)root, c.inv_bc2 = (float)(1.0 / root);
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
  const uint32_t first_place = (uint32_t)a.c.place;
  int64_t group = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32;
  if (group >= a.c.groups) return;
  int at = 0;
  for (int high = a.c.n; high - at > 1;) {  // entries[at].first <= group < entries[high].first
    const int mid = (at + high) / 2;
    if (a.entries[mid].first <= group)
      at = mid;
    else
      high = mid;
  }
  for (; group < a.c.groups; group += (int64_t)gridDim.x * kWarps) {
    while (at + 1 < a.c.n && a.entries[at + 1].first <= group) ++at;
    const Entry& e = a.entries[at];
    const uint32_t after = at + 1 < a.c.n ? a.entries[at + 1].first : a.c.groups;
    const int count = kGroup - (group + 1 == after ? e.lacks : 0);  // of this group's elements
    const int64_t in = (group - e.first) * kGroup + lane * kEach, place = group * kGroup + lane * kEach;
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
      const uint32_t w1[2] = {q1.x, q1.y}, w2[2] = {q2.x, q2.y};
      float r[8];
      auto read = [&](auto is_far) {
        constexpr bool kFar = decltype(is_far)::value;
        const Unit<3> u1(x1, kFar);
        const Unit<4> u2(x2, kFar);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          u1(signed_code(w1[i / 4], i % 4), signed_code(w1[i / 4], i % 4 + 1), kFar, m1[i], m1[i + 1]);
          u2(plain_code(w2[i / 4], i % 4), plain_code(w2[i / 4], i % 4 + 1), kFar, r[i], r[i + 1]);
        }
      };
      if (far_units(x1, x2))
        read(std::true_type());
      else
        read(std::false_type());
      // two at a time: with moments in 8 bits the instructions bound the step
      const Two by(scale);
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const Two old(r[i], r[i + 1]);
        (old * old).apart(m2[i], m2[i + 1]);
        (Two(g[i], g[i + 1]) * by).apart(g[i], g[i + 1]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) moments(c, g[i], m1[i], m2[i]);
      if (mine < kEach) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i >= mine) m1[i] = m2[i] = 0.0f;
      }
      float top1 = 0.0f, top2 = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = 2 * i, f = e + 1;
        r[e] = __fsqrt_rn(m2[e]), r[f] = __fsqrt_rn(m2[f]);
        top1 = larger_of(top1, m1[e], m1[f]), top2 = larger_of(top2, r[e], r[f]);
        // the parameter, whose change the moments' steps of 1/16 make coarse anyway, by the hardware's reciprocal: what is
        // subtracted is off by 3 units in its last place (1 of the reciprocal, half a unit each of 1 / bc2, the sum, the product)
        float d0, d1;
        fma2(Two(r[e], r[f]), Two(c.inv_bc2), Two(c.eps)).apart(d0, d1);
        const Two x = Two(m1[e], m1[f]) * Two(lin::rcp_fast(d0), lin::rcp_fast(d1));
        fma2(Two(-c.step), x, Two(p[e], p[f]) * Two(c.decay)).apart(p[e], p[f]);
      }
      x1 = exponent_of(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top1)), 16);
      x2 = exponent_of(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top2)), 17);
      const Coder<3> code1(x1);
      const Coder<4> code2(x2);
      // a lane's places differ in the last three bits, which the first step of their mixing leaves where they are
      uint32_t mixed = (first_place + (uint32_t)place) ^ key;
      mixed ^= mixed >> 16;
      uint32_t c1[8], c2[8], sign[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t d = (mixed ^ i) * kMix1;
        d = (d ^ d >> 13) * kMix2;  // the last step, d ^ d >> 16, leaves the upper half as it is
        const uint32_t upper = __byte_perm(d, 0, 0x4324), lower = __byte_perm(d, 0, 0x4104) ^ upper;
        c1[i] = code1(fabsf(m1[i]), lower);
        c2[i] = code2(r[i], upper);
        sign[i] = __float_as_uint(m1[i]);
      }
      uint2 s1 = make_uint2(upper_bytes(c1) | (upper_bytes(sign) & 0x80808080u),
                            upper_bytes(c1 + 4) | (upper_bytes(sign + 4) & 0x80808080u));
      uint2 s2 = make_uint2(upper_bytes(c2), upper_bytes(c2 + 4));
      if (x1 == 255u) s1 = make_uint2(0, 0);
      if (x2 == 255u) s2 = make_uint2(0, 0);
      *reinterpret_cast<uint2*>((uint8_t*)a.c.m1 + place) = s1;
      *reinterpret_cast<uint2*>((uint8_t*)a.c.m2 + place) = s2;
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
    const uint32_t x1 = e1[at / kGroup], x2 = e2[at / kGroup];
    const bool far = far_units(x1, x2);
    const Unit<3> u1(x1, far);
    const Unit<4> u2(x2, far);
    float v[8], w[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const uint32_t x = i < 4 ? a.x : a.y, y = i < 4 ? b.x : b.y;
      u1(signed_code(x, i % 4), signed_code(x, i % 4 + 1), far, v[i], v[i + 1]);
      u2(plain_code(y, i % 4), plain_code(y, i % 4 + 1), far, w[i], w[i + 1]);
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
  const int64_t sets = ((int64_t)c.groups + kWarps - 1) / kWarps, room = (int64_t)sms * kCtas;
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
