// The loss over a vocabulary: what stands around its products (include/smat.h, "loss over a vocabulary").
//
// The rows that count are numbered and their rows of x copied together, so that the gradient's products run over them alone
// (half of a batch that is half prompt), over rows of any alignment, and nothing that other rows hold reaches a result.

#include "smat_loss.h"

#include "smat_linear.cuh"

namespace smat {
namespace loss {
namespace {

using lin::from_float;
using lin::to_float;
using bf16 = __nv_bfloat16;

constexpr int kScan = 1024, kScanEach = 8;

// One CTA: kScan threads take kScanEach neighbouring targets each at a time.
__global__ void __launch_bounds__(kScan) index_kernel(const Index a) {
  __shared__ int sums[32];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  int before = 0;  // that count, of the targets so far
  for (int64_t base = 0; base < a.rows; base += kScan * kScanEach) {
    const int64_t first = base + (int64_t)threadIdx.x * kScanEach;
    int64_t t[kScanEach];
    int mine = 0;
#pragma unroll
    for (int i = 0; i < kScanEach; ++i) {
      t[i] = first + i < a.rows ? a.targets[first + i] : a.ignore;
      mine += t[i] != a.ignore;
    }
    int up = mine;  // inclusive, over the warp
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, up, d);
      if (lane >= d) up += v;
    }
    if (lane == 31) sums[warp] = up;
    __syncthreads();
    int at = before + up - mine, all = 0;
    for (int w = 0; w < kScan / 32; ++w) {
      if (w < warp) at += sums[w];
      all += sums[w];
    }
    before += all;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kScanEach; ++i) {
      const int64_t row = first + i;
      if (row >= a.rows) break;
      const bool counts = t[i] != a.ignore;
      a.place[row] = counts ? at : -1;
      if (!counts) continue;
      const bool good = t[i] >= 0 && t[i] < a.n;
      const float lse = a.lse[row];
      a.info[at++] = {lse * lin::kLog2e, good ? a.g[row] : __int_as_float(0x7FC00000), good ? (int)t[i] : -1, lse};
    }
  }
  if (threadIdx.x == 0) *a.count = before;
}

// A CTA per row at a time.
template <class T, bool VEC>
__global__ void __launch_bounds__(256) gather_kernel(const T* x, int64_t ldx, const int* place, const int* count, T* to,
                                                     int64_t ldto, int64_t rows, int64_t k) {
  const int there = *count;
  // rows that a product meets behind the last one: up to a whole slice in bf16, all of them in fp32
  const int64_t slice = sizeof(T) == 2 ? (there + 63) / 64 * 64 : rows, end = slice < rows ? slice : rows;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const int at = place[row];
    if (at >= 0) {
      const T* from = x + row * ldx;
      T* p = to + at * ldto;
      if (VEC) {
        constexpr int kEach = 16 / (int)sizeof(T);
        for (int64_t j = threadIdx.x; j < k / kEach; j += 256)
          reinterpret_cast<uint4*>(p)[j] = reinterpret_cast<const uint4*>(from)[j];
        for (int64_t j = k / kEach * kEach + threadIdx.x; j < k; j += 256) p[j] = from[j];
      } else {
        for (int64_t j = threadIdx.x; j < k; j += 256) p[j] = from[j];
      }
    }
    if (row >= there && row < end)
      for (int64_t j = threadIdx.x; j < k; j += 256) to[row * ldto + j] = from_float<T>(0.0f);
  }
}

template <class T>
__global__ void __launch_bounds__(256) scatter_kernel(const float* from, int64_t ldfrom, const int* place, T* dx, int64_t lddx,
                                                      int64_t rows, int64_t k) {
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const int at = place[row];
    for (int64_t j = threadIdx.x; j < k; j += 256) dx[row * lddx + j] = from_float<T>(at >= 0 ? from[at * ldfrom + j] : 0.0f);
  }
}

// Largest value and sum of exponentials of what is left, joined with another's; NaN stays NaN.
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
  if (m2 == -INFINITY) return;
  const float top = m2 > m || m2 != m2 ? m2 : m;
  s = s * expf(m - top) + s2 * expf(m2 - top);
  m = top;
}

// A lane per row, the warps share the parts.
__global__ void __launch_bounds__(1024) join_kernel(const Join a) {
  __shared__ float2 space[32][33];
  const int lane = threadIdx.x, warp = threadIdx.y;
  const int64_t row = (int64_t)blockIdx.x * 32 + lane;
  float m = -INFINITY, s = 0.0f;
  if (row < a.rows) {
#pragma unroll 4
    for (int64_t p = warp; p < a.slots; p += blockDim.y) {
      const float2 v = a.partials[p * a.rows + row];
      join(m, s, v.x, v.y);
    }
  }
  space[warp][lane] = make_float2(m, s);
  __syncthreads();
  if (warp > 0 || row >= a.rows) return;
  for (int w = 1; w < (int)blockDim.y; ++w) join(m, s, space[w][lane].x, space[w][lane].y);
  const float lse = m == -INFINITY ? m : m + logf(s);
  const int64_t t = a.targets[row];
  a.lse[row] = lse;
  a.loss[row] = t == a.ignore ? 0.0f : t >= 0 && t < a.n ? lse - a.picked[row] : __int_as_float(0x7FC00000);
}

__device__ __forceinline__ float larger_of(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// A CTA per row at a time: the row's largest value, then the exponentials' sum.
__global__ void __launch_bounds__(256) row_part_kernel(const float* z, int64_t ldz, int64_t rows, int64_t cols,
                                                       int64_t first_col, const int64_t* targets, float2* part, float* picked) {
  __shared__ float space[2][8];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const float* p = z + row * ldz;
    float m = -INFINITY;
    for (int64_t j = threadIdx.x; j < cols; j += 256) m = larger_of(m, p[j]);
#pragma unroll
    for (int d = 16; d > 0; d /= 2) m = larger_of(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
    if (lane == 0) space[0][warp] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) m = larger_of(m, space[0][w]);
    float s = 0.0f;
    if (m != -INFINITY)
      for (int64_t j = threadIdx.x; j < cols; j += 256) s += expf(p[j] - m);
#pragma unroll
    for (int d = 16; d > 0; d /= 2) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    if (lane == 0) space[1][warp] = s;
    __syncthreads();
    if (threadIdx.x > 0) continue;
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += space[1][w];
    part[row] = make_float2(m, s);
    const int64_t t = targets[row] - first_col;
    if (t >= 0 && t < cols) picked[row] = p[t];
  }
}

__global__ void __launch_bounds__(256) row_grad_kernel(float* z, int64_t ldz, int64_t rows, int64_t cols, int64_t first_col,
                                                       const LossRow* info, const int* count) {
  const int there = *count;
  for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
    const LossRow r = row < there ? info[row] : LossRow{0.0f, 0.0f, -1, 0.0f};
    const int64_t t = r.target >= 0 ? r.target - first_col : -1;
    float* p = z + row * ldz;
    for (int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x; j < cols; j += (int64_t)gridDim.x * 256)
      p[j] = row < there ? (expf(p[j] - r.lse) - (j == t ? 1.0f : 0.0f)) * r.g : 0.0f;
  }
}

__global__ void __launch_bounds__(256) add_kernel(float* to, const float* from, int64_t ld, int64_t rows, int64_t cols) {
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x)
    for (int64_t j = threadIdx.x; j < cols; j += 256) to[row * ld + j] += from[row * ld + j];
}

unsigned row_ctas(int64_t rows, int sms) { return (unsigned)(rows < 8 * (int64_t)sms ? rows : 8 * (int64_t)sms); }

}  // namespace

cudaError_t launch_index(const Index& a, cudaStream_t s) {
  index_kernel<<<1, kScan, 0, s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_gather(const void* x, int64_t ldx, const int* place, const int* count, void* to, int64_t ldto, int64_t rows,
                          int64_t k, int dtype, int sms, cudaStream_t s) {
  if (rows == 0 || k == 0) return cudaSuccess;
  const int elem = dtype == SMAT_BF16 ? 2 : 4;
  const bool vec = (uintptr_t)x % 16 == 0 && (rows == 1 || ldx * elem % 16 == 0);
  const unsigned ctas = row_ctas(rows, sms);
  auto go = [&](auto t, auto v) {
    using T = decltype(t);
    gather_kernel<T, decltype(v)::value><<<ctas, 256, 0, s>>>((const T*)x, ldx, place, count, (T*)to, ldto, rows, k);
    return cudaGetLastError();
  };
  if (dtype == SMAT_BF16) return vec ? go(bf16(), std::true_type()) : go(bf16(), std::false_type());
  return vec ? go(float(), std::true_type()) : go(float(), std::false_type());
}

cudaError_t launch_scatter(const float* from, int64_t ldfrom, const int* place, void* dx, int64_t lddx, int64_t rows, int64_t k,
                           int dtype, int sms, cudaStream_t s) {
  if (rows == 0 || k == 0) return cudaSuccess;
  if (dtype == SMAT_BF16)
    scatter_kernel<bf16><<<row_ctas(rows, sms), 256, 0, s>>>(from, ldfrom, place, (bf16*)dx, lddx, rows, k);
  else
    scatter_kernel<float><<<row_ctas(rows, sms), 256, 0, s>>>(from, ldfrom, place, (float*)dx, lddx, rows, k);
  return cudaGetLastError();
}

cudaError_t launch_join(const Join& a, cudaStream_t s) {
  const unsigned warps = (unsigned)(a.slots < 32 ? a.slots : 32);
  join_kernel<<<(unsigned)((a.rows + 31) / 32), dim3(32, warps), 0, s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_row_part(const float* z, int64_t ldz, int64_t rows, int64_t cols, int64_t first_col, const int64_t* targets,
                            float2* part, float* picked, int sms, cudaStream_t s) {
  row_part_kernel<<<row_ctas(rows, sms), 256, 0, s>>>(z, ldz, rows, cols, first_col, targets, part, picked);
  return cudaGetLastError();
}

cudaError_t launch_row_grad(float* z, int64_t ldz, int64_t rows, int64_t cols, int64_t first_col, const LossRow* info,
                            const int* count, int sms, cudaStream_t s) {
  const int64_t wide = (cols + 1023) / 1024, high = 8 * (int64_t)sms / wide + 1;
  row_grad_kernel<<<dim3((unsigned)wide, (unsigned)(rows < high ? rows : high)), 256, 0, s>>>(z, ldz, rows, cols, first_col,
                                                                                             info, count);
  return cudaGetLastError();
}

cudaError_t launch_add(float* to, const float* from, int64_t ld, int64_t rows, int64_t cols, int sms, cudaStream_t s) {
  add_kernel<<<row_ctas(rows, sms), 256, 0, s>>>(to, from, ld, rows, cols);
  return cudaGetLastError();
}

}  // namespace loss
}  // namespace smat
