// The linear layers' products on the fp32 units: fp32 sums of fp32 products, for any type, size, stride and
// alignment (smat_linear.h, Product; include/smat.h).
//
// A CTA of 256 threads makes a tile of BM x 128 sums, BM / 16 x 8 of them in each thread's registers as packed
// pairs (one instruction multiplies and adds two). Slices of 16 along l go through shared memory, the next one
// loaded to registers while one is multiplied. Where the tiles are fewer than the SMs, l is cut among the CTAs of a
// cluster; each leaves its sums in its own shared memory and then adds up and finishes its share of the rows, in
// the cluster's order: no workspace, no atomics, the same result every time.

#include "smat_linear.cuh"
#include "smat_linear.h"

namespace smat {
namespace lin {
namespace {

constexpr int kThreads = 256, kBN = 128, kBK = 16, kPad = 4;

struct Args {
  Product p;
  bool va, vb;    // operands whose rows may be read 16 (fp32) or 8 (bf16) bytes at a time
  bool vr, vo;    // residual, out: four elements at a time
  int l_share;    // l per CTA of a cluster, a multiple of kBK
};

// four values of a row, `count` of them there
template <class T>
__device__ __forceinline__ float4 load4(const T* p, int64_t count, bool vec) {
  if (vec && count >= 4) {
    if constexpr (sizeof(T) == 4) {
      return __ldg(reinterpret_cast<const float4*>(p));
    } else {
      const uint2 u = __ldg(reinterpret_cast<const uint2*>(p));
      return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16),
                         __uint_as_float(u.y & 0xFFFF0000u));
    }
  }
  float4 v;
  v.x = count > 0 ? to_float(p[0]) : 0.0f;
  v.y = count > 1 ? to_float(p[1]) : 0.0f;
  v.z = count > 2 ? to_float(p[2]) : 0.0f;
  v.w = count > 3 ? to_float(p[3]) : 0.0f;
  return v;
}

// One operand's slice [R][kBK] into registers, then into shared memory as [kBK][R + kPad].
template <class T, int R, bool MN>
struct Slice {
  static constexpr int kSteps = (R * kBK / 4 + kThreads - 1) / kThreads;
  float4 v[kSteps];

  __device__ __forceinline__ void load(const T* p, int64_t ld, int64_t first, int64_t end, int64_t l, int64_t l_end,
                                       bool vec) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int at = threadIdx.x + s * kThreads;
      v[s] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (R * kBK / 4 % kThreads && at >= R * kBK / 4) continue;
      if (MN) {
        const int64_t k = l + at / (R / 4), i = first + at % (R / 4) * 4;
        if (k < l_end) v[s] = load4(p + k * ld + i, end - i, vec);
      } else {
        const int64_t i = first + at / (kBK / 4), k = l + at % (kBK / 4) * 4;
        if (i < end) v[s] = load4(p + i * ld + k, l_end - k, vec);
      }
    }
  }

  __device__ __forceinline__ void store(float (*to)[R + kPad]) const {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int at = threadIdx.x + s * kThreads;
      if (R * kBK / 4 % kThreads && at >= R * kBK / 4) continue;
      if (MN) {
        *reinterpret_cast<float4*>(&to[at / (R / 4)][at % (R / 4) * 4]) = v[s];
      } else {
        const int i = at / (kBK / 4), k = at % (kBK / 4) * 4;
        to[k][i] = v[s].x, to[k + 1][i] = v[s].y, to[k + 2][i] = v[s].z, to[k + 3][i] = v[s].w;
      }
    }
  }
};

__device__ __forceinline__ uint64_t pair_of(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ void fma_pair(uint64_t& acc, uint64_t a, uint64_t b) {
  asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(acc) : "l"(a), "l"(b));
}

template <class T>
__device__ __forceinline__ void store4(T* p, int64_t count, bool vec, const float (&v)[4]) {
  if (vec && count >= 4) {
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
      const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
      *reinterpret_cast<uint2*>(p) =
          make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < count) p[i] = from_float<T>(v[i]);
}

// Four sums (i, j .. j + 3) to what the call returns. The 8 lanes that share a group of 32 columns call it together.
template <class T>
__device__ __forceinline__ void finish4(const Args& a, int64_t i, int64_t j, float (&v)[4]) {
  const Product& p = a.p;
  const int64_t count = i < p.I ? p.J - j : 0;
  T* out = (T*)p.out + i * p.ldo + j;
  if (p.mode == kForward) {
    if (p.bias && count > 0) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (t < count) v[t] += to_float(((const T*)p.bias)[j + t]);
    }
    if (p.q) {
      float big = 0.0f;
#pragma unroll
      for (int t = 0; t < 4; ++t) big = t < count ? larger(big, v[t]) : big;
      uint32_t top = __float_as_uint(big);
#pragma unroll
      for (int d = 1; d < 8; d *= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
      const uint32_t ex = pack_exponent(top);
      uint32_t w;
      pack_words<1>(v, ex, &w);
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (t < count) p.q[i * p.ldq + j + t] = (int8_t)(w >> (8 * t));
      if (count > 0 && j % kGroup == 0) p.e[i * p.lde + j / kGroup] = (uint8_t)ex;
    }
    if (count <= 0) return;
    SMAT_WITH_ACT(p.act, _Pragma("unroll") for (int t = 0; t < 4; ++t) v[t] = act_value<ACT>(v[t]))
    if (p.residual) {
      const float4 r = load4((const T*)p.residual + i * p.ldr + j, count, a.vr);
      v[0] += r.x, v[1] += r.y, v[2] += r.z, v[3] += r.w;
    }
  } else {
    if (count <= 0) return;
    if (p.mode == kGradInput && p.act != SMAT_ACT_NONE) {
      const float scale = unpack_scale(p.e[i * p.lde + j / kGroup]);
      SMAT_WITH_ACT(p.act, _Pragma("unroll") for (int t = 0; t < 4; ++t) if (t < count) v[t] *=
                    act_slope<ACT>((float)p.q[i * p.ldq + j + t] * scale))
    }
    if (p.accumulate) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (t < count) v[t] += to_float(out[t]);
    }
  }
  store4(out, count, a.vo, v);
}

template <class T, int BM, bool A_MN, bool B_MN>
__global__ void __launch_bounds__(kThreads, BM == 128 ? 2 : 3) simt_kernel(const Args a) {
  constexpr int TM = BM / 16;  // consecutive rows per thread
  extern __shared__ __align__(16) float shared[];
  static_assert(TM == 8 || TM == 2, "");
  float (*sa)[kBK][BM + kPad] = reinterpret_cast<float (*)[kBK][BM + kPad]>(shared);
  float (*sb)[kBK][kBN + kPad] = reinterpret_cast<float (*)[kBK][kBN + kPad]>(shared + 2 * kBK * (BM + kPad));
  float (*sums)[kBN] = reinterpret_cast<float (*)[kBN]>(shared);  // afterwards

  const Product& p = a.p;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  const int64_t i0 = (int64_t)blockIdx.x * BM, j0 = (int64_t)blockIdx.y * kBN;
  const int64_t l0 = (int64_t)blockIdx.z * a.l_share;
  const int64_t l1 = l0 + a.l_share < p.L ? l0 + a.l_share : p.L;

  uint64_t acc[TM][4];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0;

  Slice<T, BM, A_MN> na;
  Slice<T, kBN, B_MN> nb;
  const T *pa = (const T*)p.a, *pb = (const T*)p.b;
  if (l0 < l1) {
    na.load(pa, p.lda, i0, p.I, l0, l1, a.va);
    nb.load(pb, p.ldb, j0, p.J, l0, l1, a.vb);
    na.store(sa[0]);
    nb.store(sb[0]);
  }
  __syncthreads();
  int at = 0;
  for (int64_t l = l0; l < l1; l += kBK, at ^= 1) {
    const bool more = l + kBK < l1;
    if (more) {
      na.load(pa, p.lda, i0, p.I, l + kBK, l1, a.va);
      nb.load(pb, p.ldb, j0, p.J, l + kBK, l1, a.vb);
    }
#pragma unroll
    for (int k = 0; k < kBK; ++k) {
      const ulonglong2 b01 = *reinterpret_cast<const ulonglong2*>(&sb[at][k][tx * 4]);
      const ulonglong2 b23 = *reinterpret_cast<const ulonglong2*>(&sb[at][k][64 + tx * 4]);
      float x[TM];
      if constexpr (TM == 8) {
        *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(&sa[at][k][ty * TM]);
        *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(&sa[at][k][ty * TM + 4]);
      } else {
        *reinterpret_cast<float2*>(x) = *reinterpret_cast<const float2*>(&sa[at][k][ty * TM]);
      }
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const uint64_t xx = pair_of(x[i], x[i]);
        fma_pair(acc[i][0], xx, b01.x);
        fma_pair(acc[i][1], xx, b01.y);
        fma_pair(acc[i][2], xx, b23.x);
        fma_pair(acc[i][3], xx, b23.y);
      }
    }
    if (more) {
      na.store(sa[at ^ 1]);
      nb.store(sb[at ^ 1]);
    }
    __syncthreads();
  }

#pragma unroll
  for (int i = 0; i < TM; ++i) {
    *reinterpret_cast<ulonglong2*>(&sums[ty * TM + i][tx * 4]) = make_ulonglong2(acc[i][0], acc[i][1]);
    *reinterpret_cast<ulonglong2*>(&sums[ty * TM + i][64 + tx * 4]) = make_ulonglong2(acc[i][2], acc[i][3]);
  }
  const int shares = gridDim.z;
  if (shares > 1)
    cluster_sync();
  else
    __syncthreads();
  // the rows go around among the CTAs of the cluster and their warps; a warp finishes a row of 128
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  for (int row = (int)blockIdx.z * 8 + warp; row < BM; row += 8 * shares) {
    if (i0 + row >= p.I) break;
    float v[4] = {};
    if (shares == 1) {
      const float4 t = *reinterpret_cast<const float4*>(&sums[row][lane * 4]);
      v[0] = t.x, v[1] = t.y, v[2] = t.z, v[3] = t.w;
    } else {
      for (int s = 0; s < shares; ++s) {
        const float4 t = cluster_load4(cluster_address(&sums[row][lane * 4], (uint32_t)s));
        v[0] += t.x, v[1] += t.y, v[2] += t.z, v[3] += t.w;
      }
    }
    finish4<T>(a, i0 + row, j0 + lane * 4, v);
  }
  if (shares > 1) cluster_sync();  // nobody leaves while its sums are read
}

bool can(const void* p, int64_t ld, size_t elem) { return (uintptr_t)p % (4 * elem) == 0 && ld % 4 == 0; }

template <class T, int BM, bool A_MN, bool B_MN>
cudaError_t launch_tile(const Args& a, int shares, cudaStream_t s) {
  constexpr int kSlices = 2 * kBK * (BM + kPad + kBN + kPad) * 4, kSums = BM * kBN * 4;
  constexpr int kBytes = kSlices > kSums ? kSlices : kSums;
  auto* f = simt_kernel<T, BM, A_MN, B_MN>;
  static std::atomic<uint64_t> allowed;
  const cudaError_t e = allow_shared(f, kBytes, allowed);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((a.p.I + BM - 1) / BM), (unsigned)((a.p.J + kBN - 1) / kBN), (unsigned)shares);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kBytes;
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim = {1, 1, (unsigned)shares};
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, f, a);
}

template <class T, bool A_MN, bool B_MN>
cudaError_t launch_as(const Args& a, int sms, cudaStream_t s) {
  Args b = a;
  const Product& p = a.p;
  const bool low = p.I <= 32;
  const int64_t bm = low ? 32 : 128;
  const int64_t tiles = (p.I + bm - 1) / bm * ((p.J + kBN - 1) / kBN);
  int shares = 1;
  // two CTAs fit on an SM; a share is at least 64 long
  while (shares < 8 && tiles * shares * 2 <= 2 * sms && p.L >= (int64_t)shares * 2 * 64) shares *= 2;
  b.l_share = (int)((p.L + shares * kBK - 1) / (shares * kBK) * kBK);
  return low ? launch_tile<T, 32, A_MN, B_MN>(b, shares, s) : launch_tile<T, 128, A_MN, B_MN>(b, shares, s);
}

template <class T>
cudaError_t launch_type(const Args& a, int sms, cudaStream_t s) {
  switch (a.p.mode) {
    case kForward: return launch_as<T, false, false>(a, sms, s);
    case kGradInput: return launch_as<T, false, true>(a, sms, s);
    default: return launch_as<T, true, true>(a, sms, s);
  }
}

}  // namespace

cudaError_t launch_simt(const Product& p, int sms, cudaStream_t s) {
  const size_t elem = p.dtype == SMAT_BF16 ? 2 : 4;
  Args a = {};
  a.p = p;
  a.va = can(p.a, p.lda, elem);
  a.vb = can(p.b, p.ldb, elem);
  a.vr = can(p.residual, p.ldr, elem);
  a.vo = can(p.out, p.ldo, elem);
  return p.dtype == SMAT_BF16 ? launch_type<__nv_bfloat16>(a, sms, s) : launch_type<float>(a, sms, s);
}

}  // namespace lin
}  // namespace smat
