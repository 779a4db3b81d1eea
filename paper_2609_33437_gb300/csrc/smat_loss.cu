// The loss over a vocabulary: what stands around its products (include/smat.h, "loss over a vocabulary").
//
// The rows that count are numbered and their rows of x copied together, so that the gradient's products run over them alone
// (half of a batch that is half prompt), over rows of any alignment, and nothing that other rows hold reaches a result.

#include "smat_loss.h"

#include <algorithm>

#include "smat_linear.cuh"

namespace smat {
namespace loss {
namespace {

using lin::from_float;
using lin::to_float;
using bf16 = __nv_bfloat16;

constexpr int kScan = 1024, kScanEach = 8, kScanWarps = kScan / 32;

// One CTA: kScanEach x kScan targets at a time, a warp's 32 neighbours counted by a vote.
__global__ void __launch_bounds__(kScan) index_kernel(const Index a) {
  constexpr int kVotes = kScanEach * kScanWarps;  // in the rows' order
  __shared__ int counts[kVotes], sums[kVotes / 32];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  int before = 0;  // that count, of the targets so far
  for (int64_t base = 0; base < a.rows; base += kScan * kScanEach) {
    int64_t t[kScanEach];
    uint32_t votes[kScanEach];
#pragma unroll
    for (int i = 0; i < kScanEach; ++i) {
      const int64_t row = base + i * kScan + threadIdx.x;
      t[i] = row < a.rows ? a.targets[row] : a.ignore;
    }
#pragma unroll
    for (int i = 0; i < kScanEach; ++i) {
      votes[i] = __ballot_sync(0xFFFFFFFFu, t[i] != a.ignore);
      if (lane == 0) counts[i * kScanWarps + warp] = __popc(votes[i]);
    }
    __syncthreads();
    int up = 0;  // inclusive, over 32 votes
    if (threadIdx.x < kVotes) {
      up = counts[threadIdx.x];
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const int v = __shfl_up_sync(0xFFFFFFFFu, up, d);
        if (lane >= d) up += v;
      }
      if (lane == 31) sums[warp] = up;
    }
    __syncthreads();
    int all = 0, here = before;
#pragma unroll
    for (int w = 0; w < kVotes / 32; ++w) {
      if (w < warp) here += sums[w];
      all += sums[w];
    }
    if (threadIdx.x < kVotes) counts[threadIdx.x] = here + up - counts[threadIdx.x];  // before this vote
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kScanEach; ++i) {
      const int64_t row = base + i * kScan + threadIdx.x;
      const bool counted = votes[i] >> lane & 1;
      if (row < a.rows) a.place[row] = counted ? counts[i * kScanWarps + warp] + __popc(votes[i] & ((1u << lane) - 1)) : -1;
    }
    before += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) *a.count = a.twice ? 2 * before : before;
}

// A CTA per row at a time. VEC: rows of x, and of W in bf16, on 16 bytes.
//
// bf16: the target's logit is made here once more, in fp32, and its gradient g (exp(logit - lse) - 1) from it. Where a model is sure
// of a word the two nearly cancel, and what tensor memory cuts off a sum (2e-5 of a logit of 12) would be a tenth of a percent of
// the largest gradient there is.
template <class T, bool VEC>
__global__ void __launch_bounds__(256) gather_kernel(const Index a, const T* x, int64_t ldx, T* to, int64_t ldto, int64_t k,
                                                     bool to_end) {
  constexpr int kEach = 16 / (int)sizeof(T);
  __shared__ float space[8];
  const int there = *a.count;
  const int64_t rows = a.rows, room = a.twice ? 2 * rows : rows;
  // rows that a product meets behind the last one: up to a whole slice of its sum, or all of them
  const int64_t slice = to_end ? room : (there + (int64_t)63) / 64 * 64, end = slice < room ? slice : room;
  for (int64_t behind = there + blockIdx.x; behind < end; behind += gridDim.x)
    for (int64_t j = threadIdx.x; j < k; j += 256) to[behind * ldto + j] = from_float<T>(0.0f);
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const int at = a.place[row];
    if (at >= 0) {
      const int64_t t = a.targets[row];
      const bool good = t >= 0 && t < a.n;
      const T* from = x + row * ldx;
      const T* w = (const T*)a.w + (good ? t : 0) * a.ldw;
      T* p = to + at * ldto;
      T* second = a.twice ? to + (at + there / 2) * ldto : p;
      float dot = 0.0f;
      const int64_t whole = VEC ? k / kEach : 0;
      for (int64_t j = threadIdx.x; j < whole; j += 256) {
        const uint4 u = reinterpret_cast<const uint4*>(from)[j];
        reinterpret_cast<uint4*>(p)[j] = u;
        if (a.twice) reinterpret_cast<uint4*>(second)[j] = u;
        if (sizeof(T) == 2) {
          const uint4 v = reinterpret_cast<const uint4*>(w)[j];
          const uint32_t c[4] = {u.x, u.y, u.z, u.w}, d[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            dot = fmaf(__uint_as_float(c[i] << 16), __uint_as_float(d[i] << 16), dot);
            dot = fmaf(__uint_as_float(c[i] & 0xFFFF0000u), __uint_as_float(d[i] & 0xFFFF0000u), dot);
          }
        }
      }
      for (int64_t j = whole * kEach + threadIdx.x; j < k; j += 256) {
        p[j] = from[j];
        if (a.twice) second[j] = from[j];
        if (sizeof(T) == 2) dot = fmaf(to_float(from[j]), to_float(w[j]), dot);
      }
      if (sizeof(T) == 2) {
#pragma unroll
        for (int d = 16; d > 0; d /= 2) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, d);
        if (threadIdx.x % 32 == 0) space[threadIdx.x / 32] = dot;
        __syncthreads();
        dot = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) dot += space[i];
        __syncthreads();
      }
      if (threadIdx.x == 0) {
        const float lse = a.lse[row], g = good ? a.g[row] : __int_as_float(0x7FC00000);
        const LossRow r = {lse * lin::kLog2e, g, good ? (int)t : -1, sizeof(T) == 2 ? g * expm1f(dot - lse) : lse};
        a.info[at] = r;
        if (a.twice) a.info[at + there / 2] = r;
      }
    }
  }
}

// A CTA per row, or per 1024 of a row's columns where rows are few. A row's sums lie in as many places as its product was cut
// into, twice as many where d has two rows; 8 of them are asked for at a time (24 x 4096 in 8 places: 4.4 us, and 8.6 one after
// another and in 24 CTAs).
template <class T, bool VEC>
__global__ void __launch_bounds__(256) scatter_kernel(const Sums from, const Index a, T* dx, int64_t lddx, int64_t k) {
  const int64_t second = a.twice ? *a.count / 2 * from.ld : 0;
  const int places = a.twice ? 2 * from.splits : from.splits;
  const int64_t first = blockIdx.y * 256 + threadIdx.x, step = gridDim.y * 256;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int at = a.place[row];
    const float* p = from.at + at * from.ld;
    auto place = [&](int i) { return a.twice ? p + (i >> 1) * from.apart + (i & 1) * second : p + i * from.apart; };
    T* to = dx + row * lddx;
    const int64_t whole = VEC ? k / 4 : 0;
    for (int64_t j = first; j < whole; j += step) {
      float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      for (int i = 0; at >= 0 && i < places; i += 8) {
        float4 u[8];
#pragma unroll
        for (int t = 0; t < 8; ++t)
          if (i + t < places) u[t] = __ldcs(reinterpret_cast<const float4*>(place(i + t)) + j);
#pragma unroll
        for (int t = 0; t < 8; ++t)
          if (i + t < places) v.x += u[t].x, v.y += u[t].y, v.z += u[t].z, v.w += u[t].w;
      }
      if constexpr (sizeof(T) == 2) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
        reinterpret_cast<uint2*>(to)[j] = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
      } else {
        reinterpret_cast<float4*>(to)[j] = v;
      }
    }
    for (int64_t j = 4 * whole + first; j < k; j += step) {
      float v = 0.0f;
      for (int i = 0; at >= 0 && i < places; ++i) v += place(i)[j];
      to[j] = from_float<T>(v);
    }
  }
}

__device__ __forceinline__ float larger_of(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// kJoinRows neighbouring rows a CTA; the other lanes and the warps share the parts: first the largest, then the sum of what they
// stand for, so that no thread waits for its last step.
constexpr int kJoinRows = 8;
__global__ void __launch_bounds__(1024) join_kernel(const Join a) {
  __shared__ float space[2][32][kJoinRows];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, r = threadIdx.x % kJoinRows, warps = blockDim.x / 32;
  const int64_t row = (int64_t)blockIdx.x * kJoinRows + r, first = threadIdx.x / kJoinRows, step = blockDim.x / kJoinRows;
  float m = -INFINITY;
  if (row < a.rows) {
#pragma unroll 4
    for (int64_t p = first; p < a.slots; p += step) m = larger_of(m, a.partials[p * a.rows + row].x);
  }
#pragma unroll
  for (int d = kJoinRows; d < 32; d *= 2) m = larger_of(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
  if (lane < kJoinRows) space[0][warp][r] = m;
  __syncthreads();
  for (int w = 0; w < warps; ++w) m = larger_of(m, space[0][w][r]);
  float s = 0.0f;
  if (row < a.rows && m != -INFINITY) {
#pragma unroll 4
    for (int64_t p = first; p < a.slots; p += step) {
      const float2 v = a.partials[p * a.rows + row];
      if (v.x != -INFINITY) s += v.y * expf(v.x - m);
    }
  }
#pragma unroll
  for (int d = kJoinRows; d < 32; d *= 2) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
  if (lane < kJoinRows) space[1][warp][r] = s;
  __syncthreads();
  if (threadIdx.x >= kJoinRows || row >= a.rows) return;
  s = 0.0f;
  for (int w = 0; w < warps; ++w) s += space[1][w][r];
  const float lse = m == -INFINITY ? m : m + logf(s);
  const int64_t t = a.targets[row];
  a.lse[row] = lse;
  a.loss[row] = t == a.ignore ? 0.0f : t >= 0 && t < a.n ? lse - a.picked[row] : __int_as_float(0x7FC00000);
}

// A CTA per row at a time: the row's largest value, then the exponentials' sum.
__global__ void __launch_bounds__(256) row_part_kernel(const float* z, int64_t ldz, int64_t rows, int64_t cols,
                                                       int64_t first_col, const int64_t* targets, float2* part, float* picked) {
  __shared__ float space[2][8];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    const float* p = z + row * ldz;
    float m = -INFINITY;
    for (int64_t j = threadIdx.x; j < cols / 4; j += 256) {
      const float4 v = reinterpret_cast<const float4*>(p)[j];
      m = larger_of(larger_of(m, larger_of(v.x, v.y)), larger_of(v.z, v.w));
    }
    for (int64_t j = cols / 4 * 4 + threadIdx.x; j < cols; j += 256) m = larger_of(m, p[j]);
#pragma unroll
    for (int d = 16; d > 0; d /= 2) m = larger_of(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
    if (lane == 0) space[0][warp] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) m = larger_of(m, space[0][w]);
    float s = 0.0f;
    if (m != -INFINITY) {
      for (int64_t j = threadIdx.x; j < cols / 4; j += 256) {
        const float4 v = reinterpret_cast<const float4*>(p)[j];
        s += (expf(v.x - m) + expf(v.y - m)) + (expf(v.z - m) + expf(v.w - m));
      }
      for (int64_t j = cols / 4 * 4 + threadIdx.x; j < cols; j += 256) s += expf(p[j] - m);
    }
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
      p[j] = row < there ? (expf(p[j] - r.own) - (j == t ? 1.0f : 0.0f)) * r.g : 0.0f;
  }
}

// As cut_kernel of the linear layers: a thread has 8 neighbours of a row.
__global__ void __launch_bounds__(256) row_grad_cut_kernel(float* z, int64_t ldz, int64_t rows, int64_t cols, int64_t first_col,
                                                           const LossRow* info, const int* count, uint16_t* parts, int64_t ldp,
                                                           uint32_t* flags) {
  __shared__ uint32_t tops[8];
  const int there = *count;
  const int64_t slice = (there + (int64_t)63) / 64 * 64, end = slice < rows ? slice : rows, units = ldp / 8, plane = rows * ldp;
  const int wide = (int)(units < 256 ? units : 256), high = 256 / wide, tx = threadIdx.x % wide, ty = threadIdx.x / wide;
  uint32_t top = 0;
  if (ty < high)
    for (int64_t row = (int64_t)blockIdx.x * high + ty; row < end; row += (int64_t)gridDim.x * high) {
      const LossRow r = row < there ? info[row] : LossRow{0.0f, 0.0f, -1, 0.0f};
      const int64_t t = r.target >= 0 ? r.target - first_col : -1;
      for (int64_t u = tx; u < units; u += wide) {
        const int64_t at = 8 * u;
        float* p = z + row * ldz + at;
        float v[8];
        // z's rows have room for whole groups of 32
        *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(p);
        *reinterpret_cast<float4*>(v + 4) = *reinterpret_cast<const float4*>(p + 4);
        uint32_t w[3][4];
#pragma unroll
        for (int i = 0; i < 8; ++i)
          v[i] = row < there && at + i < cols ? (expf(v[i] - r.own) - (at + i == t ? 1.0f : 0.0f)) * r.g : 0.0f;
        *reinterpret_cast<float4*>(p) = *reinterpret_cast<const float4*>(v);
        *reinterpret_cast<float4*>(p + 4) = *reinterpret_cast<const float4*>(v + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t of[3];
          lin::cut2(v[2 * i], v[2 * i + 1], of, top);
          w[0][i] = of[0], w[1][i] = of[1], w[2][i] = of[2];
        }
#pragma unroll
        for (int q = 0; q < 3; ++q)
          *reinterpret_cast<uint4*>(parts + q * plane + row * ldp + at) = make_uint4(w[q][0], w[q][1], w[q][2], w[q][3]);
      }
    }
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  if (threadIdx.x % 32 == 0) tops[threadIdx.x / 32] = top;
  __syncthreads();
  if (threadIdx.x < 8) {
    top = __reduce_max_sync(0xFFu, tops[threadIdx.x]);
    if (threadIdx.x == 0) flags[blockIdx.x] = lin::flag_of(top);
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

cudaError_t launch_gather(const Index& a, const void* x, int64_t ldx, void* to, int64_t ldto, int64_t k, int dtype, bool to_end,
                          int sms, cudaStream_t s) {
  const int elem = dtype == SMAT_BF16 ? 2 : 4;
  const bool vec = (uintptr_t)x % 16 == 0 && (a.rows == 1 || ldx * elem % 16 == 0) &&
                   (dtype != SMAT_BF16 || ((uintptr_t)a.w % 16 == 0 && (a.n == 1 || a.ldw * elem % 16 == 0)));
  const unsigned ctas = row_ctas(a.rows, sms);
  auto go = [&](auto t, auto v) {
    using T = decltype(t);
    gather_kernel<T, decltype(v)::value><<<ctas, 256, 0, s>>>(a, (const T*)x, ldx, (T*)to, ldto, k, to_end);
    return cudaGetLastError();
  };
  if (dtype == SMAT_BF16) return vec ? go(bf16(), std::true_type()) : go(bf16(), std::false_type());
  return vec ? go(float(), std::true_type()) : go(float(), std::false_type());
}

cudaError_t launch_scatter(const Sums& from, const Index& a, void* dx, int64_t lddx, int64_t k, int dtype, int sms,
                           cudaStream_t s) {
  const int bytes = dtype == SMAT_BF16 ? 8 : 16;  // of four elements
  const bool vec = (uintptr_t)dx % bytes == 0 && (a.rows == 1 || lddx % 4 == 0);
  const unsigned ctas = row_ctas(a.rows, sms);
  const dim3 grid(ctas, (unsigned)std::max<int64_t>(1, std::min<int64_t>((k + 1023) / 1024, 4 * (int64_t)sms / ctas)));
  auto go = [&](auto t, auto v) {
    using T = decltype(t);
    scatter_kernel<T, decltype(v)::value><<<grid, 256, 0, s>>>(from, a, (T*)dx, lddx, k);
    return cudaGetLastError();
  };
  if (dtype == SMAT_BF16) return vec ? go(bf16(), std::true_type()) : go(bf16(), std::false_type());
  return vec ? go(float(), std::true_type()) : go(float(), std::false_type());
}

cudaError_t launch_join(const Join& a, int sms, cudaStream_t s) {
  // warps for all parts at once, but no more than run at once, or 8
  const int64_t ctas = (a.rows + kJoinRows - 1) / kJoinRows, all = (a.slots * kJoinRows + 31) / 32;
  int64_t warps = 32;
  while (warps > 8 && ctas * warps > (int64_t)sms * 64) warps /= 2;
  join_kernel<<<(unsigned)ctas, (unsigned)(32 * (all < warps ? all : warps)), 0, s>>>(a);
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

cudaError_t launch_row_grad_cut(float* z, int64_t ldz, int64_t rows, int64_t cols, int64_t first_col, const LossRow* info,
                                const int* count, const lin::Parts& parts, cudaStream_t s) {
  row_grad_cut_kernel<<<parts.n_flags, 256, 0, s>>>(z, ldz, rows, cols, first_col, info, count, (uint16_t*)parts.p,
                                                    lin::parts_ld(cols), parts.flags);
  return cudaGetLastError();
}

cudaError_t launch_add(float* to, const float* from, int64_t ld, int64_t rows, int64_t cols, int sms, cudaStream_t s) {
  add_kernel<<<row_ctas(rows, sms), 256, 0, s>>>(to, from, ld, rows, cols);
  return cudaGetLastError();
}

}  // namespace loss
}  // namespace smat
