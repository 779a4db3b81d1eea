// Weight gradients over few rows: dW(n, k) = sum over 1 to 16 rows m of dy(m, n) x^(m, k), db(n) = sum of dy(m, n) (smat_linear.h).
//
// The result is by far the most that is moved, so the kernel is one pass that writes it: a thread holds C columns of every
// row of x^ in registers (read back from 8 bits where they are saved so) and makes those columns of one row of dW after
// another, whose factors dy(m, n) lie in shared memory; a CTA has up to 256 rows of 32 * C columns. fp32 products and sums. Columns
// of a thread are neighbours where rows start on 16 bytes, 32 apart else, so that a warp writes whole stretches either way.

#include "smat_linear.cuh"
#include "smat_linear.h"

namespace smat {
namespace lin {
namespace {

constexpr int kThreads = 256, kMostRows = 256;  // of dW, per CTA

template <class T>
__device__ __forceinline__ float stored(float v) {  // what x^ is rounded to before it is multiplied
  return to_float(from_float<T>(v));
}

template <class T, int L, int C, bool VEC>
__global__ void __launch_bounds__(kThreads) outer_kernel(const Outer a, int per) {
  __shared__ float factor[kMostRows][L];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t n0 = (int64_t)blockIdx.y * per, k0 = (int64_t)blockIdx.x * (32 * C);
  const T* dy = (const T*)a.dy;
  for (int n = threadIdx.x; n < per; n += kThreads)
#pragma unroll
    for (int m = 0; m < L; ++m) factor[n][m] = m < a.rows && n0 + n < a.n ? to_float(dy[m * a.lddy + n0 + n]) : 0.0f;
  // this thread's columns: place(c)
  auto place = [&](int c) { return k0 + (VEC ? lane * C + c : 32 * c + lane); };
  // all loads first; rows past the last one read it again and count as 0
  float x[L][C];
  const int last = (int)a.rows - 1;
  if (a.q) {
#pragma unroll
    for (int m = 0; m < L; ++m)
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int64_t k = place(c) < a.k ? place(c) : a.k - 1, row = m < last ? m : last;
        x[m][c] = (float)a.q[row * a.ldq + k] * unpack_scale(a.e[row * a.lde + k / kGroup]);
      }
  } else {
#pragma unroll
    for (int m = 0; m < L; ++m)
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int64_t k = place(c) < a.k ? place(c) : a.k - 1, row = m < last ? m : last;
        x[m][c] = to_float(((const T*)a.x)[row * a.ldx + k]);
      }
  }
  SMAT_WITH_ACT(a.act, _Pragma("unroll") for (int m = 0; m < L; ++m) _Pragma("unroll") for (int c = 0; c < C; ++c)
                    x[m][c] = m <= last ? stored<T>(act_value<ACT, T>(x[m][c])) : 0.0f)
  __syncthreads();
  if (a.db && blockIdx.x == 0 && threadIdx.x < per && n0 + threadIdx.x < a.n) {
    T* db = (T*)a.db + n0 + threadIdx.x;
    float t = a.add_db ? to_float(*db) : 0.0f;
#pragma unroll
    for (int m = 0; m < L; ++m) t += factor[threadIdx.x][m];
    *db = from_float<T>(t);
  }
#pragma unroll 2
  for (int r = warp; r < per; r += kThreads / 32) {
    const int64_t n = n0 + r;
    if (n >= a.n) break;
    T* out = (T*)a.dw + n * a.lddw;
    float v[C];
#pragma unroll
    for (int c = 0; c < C; ++c) v[c] = 0.0f;
    if (a.add_dw) {
      if (VEC && place(0) + C <= a.k) {
        constexpr int kWords = C * (int)sizeof(T) / 4;
        uint32_t w[kWords];
#pragma unroll
        for (int h = 0; h < kWords; h += 4) {
          if constexpr (kWords >= 4) {
            const uint4 u = *reinterpret_cast<const uint4*>(out + place(0) + h * 4 / (int)sizeof(T));
            w[h] = u.x, w[h + 1] = u.y, w[h + 2] = u.z, w[h + 3] = u.w;
          } else {
            const uint2 u = *reinterpret_cast<const uint2*>(out + place(0));
            w[0] = u.x, w[1] = u.y;
          }
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
          v[c] = sizeof(T) == 4 ? __uint_as_float(w[c % kWords])
                                : __uint_as_float(c % 2 ? w[c / 2 % kWords] & 0xFFFF0000u : w[c / 2 % kWords] << 16);
      } else {
#pragma unroll
        for (int c = 0; c < C; ++c)
          if (place(c) < a.k) v[c] = to_float(out[place(c)]);
      }
    }
#pragma unroll
    for (int m = 0; m < L; ++m) {
      const float f = factor[r][m];
#pragma unroll
      for (int c = 0; c < C; ++c) v[c] = fmaf(f, x[m][c], v[c]);
    }
    if (VEC && place(0) + C <= a.k) {
      if constexpr (sizeof(T) == 2) {
        uint32_t w[C / 2];
#pragma unroll
        for (int c = 0; c < C / 2; ++c) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * c], v[2 * c + 1]);
          w[c] = *reinterpret_cast<const uint32_t*>(&b);
        }
        if constexpr (C == 8)
          *reinterpret_cast<uint4*>(out + place(0)) = make_uint4(w[0], w[1], w[2], w[3]);
        else
          *reinterpret_cast<uint2*>(out + place(0)) = make_uint2(w[0], w[1]);
      } else {
#pragma unroll
        for (int c = 0; c < C; c += 4)
          *reinterpret_cast<float4*>(out + place(c)) = make_float4(v[c], v[c + 1], v[c + 2], v[c + 3]);
      }
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (place(c) < a.k) out[place(c)] = from_float<T>(v[c]);
    }
  }
}

template <class T, int L, int C>
cudaError_t launch_as(const Outer& a, int sms, cudaStream_t s) {
  const int64_t across = (a.k + 32 * C - 1) / (32 * C);
  // rows per CTA: as many as leave two CTAs for each SM, since reading x^ costs each CTA as much as writing some rows
  int per = kMostRows;
  while (per > 16 && across * ((a.n + per - 1) / per) < 2 * sms) per /= 2;
  const dim3 grid((unsigned)across, (unsigned)((a.n + per - 1) / per));
  if ((uintptr_t)a.dw % 16 == 0 && a.lddw * sizeof(T) % 16 == 0)
    outer_kernel<T, L, C, true><<<grid, kThreads, 0, s>>>(a, per);
  else
    outer_kernel<T, L, C, false><<<grid, kThreads, 0, s>>>(a, per);
  return cudaGetLastError();
}
template <class T>
cudaError_t launch_type(const Outer& a, int sms, cudaStream_t s) {
  // 16 bytes of a row per thread; 8 where the rows of x^ would take all registers
  constexpr int C = sizeof(T) == 2 ? 8 : 4;
  if (a.rows <= 1) return launch_as<T, 1, C>(a, sms, s);
  if (a.rows <= 4) return launch_as<T, 4, C>(a, sms, s);
  if constexpr (sizeof(T) == 4)
    if (a.rows > 8) return launch_as<T, 16, 4>(a, sms, s);
  return launch_as<T, 8, 4>(a, sms, s);
}

}  // namespace

cudaError_t launch_outer(const Outer& a, int dtype, int sms, cudaStream_t s) {
  return dtype == SMAT_BF16 ? launch_type<__nv_bfloat16>(a, sms, s) : launch_type<float>(a, sms, s);
}

}  // namespace lin
}  // namespace smat
