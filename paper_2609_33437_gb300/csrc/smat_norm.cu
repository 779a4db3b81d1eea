// Layer norm and rms norm, forward and backward (include/smat.h, "norms").
//
// A row is held in registers by a group of warps, E values a thread, so that it is read once: its mean, then the squares of
// what is left (both sums in fp32, over lanes and then warps in a fixed order), then the result. The groups walk over the
// rows with the weights in registers and the next row's loads under way. Backward the columns a thread holds are the same for
// every row, so it adds up dw and db for them as it goes; every CTA leaves its sums in the workspace, and a second launch
// adds those in the CTAs' order: no atomics, the same bits every time. Rows of more than kMaxCols columns are read three
// times by a CTA each (the later times mostly from L2).

#include "smat_norm.h"

#include <type_traits>

#include "smat_linear.cuh"

namespace smat {
namespace norm {
namespace {

using lin::from_float;
using lin::to_float;
using bf16 = __nv_bfloat16;

constexpr int kMaxWarps = 32, kMaxCols = 16384;

// VEC neighbours as they lie in memory
template <class T, int VEC>
struct Raw {
  static constexpr int kBytes = VEC * (int)sizeof(T);
  using Word = std::conditional_t<kBytes == 16, uint4,
                                  std::conditional_t<kBytes == 8, uint2, std::conditional_t<kBytes == 4, uint32_t, uint16_t>>>;
  Word u;
  __device__ __forceinline__ void load(const T* p) { u = *reinterpret_cast<const Word*>(p); }
  __device__ __forceinline__ void zero() { u = Word{}; }
  __device__ __forceinline__ float at(int i) const { return to_float(reinterpret_cast<const T*>(&u)[i]); }
  __device__ __forceinline__ void set(int i, float v) { reinterpret_cast<T*>(&u)[i] = from_float<T>(v); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<Word*>(p) = u; }
};

// A vector of weights: its own alignment is any.
template <class W, int VEC>
__device__ __forceinline__ void load_weights(const W* p, int64_t at, bool there, float other, float (&v)[VEC]) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) v[i] = there && p ? to_float(p[at + i]) : other;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d /= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

// N sums over a row's warps. `space`: [rows of the CTA][warps][N], another one than the last call's: a thread that writes to
// the last call's place has passed this call's barrier, and so has everybody who read it.
template <int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* space) {
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = warp_sum(v[n]);
  const int warps = blockDim.x / 32;
  if (warps == 1) return;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  float* mine = space + (size_t)threadIdx.y * warps * N;
  if (lane == 0)
#pragma unroll
    for (int n = 0; n < N; ++n) mine[warp * N + n] = v[n];
  __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = warp_sum(lane < warps ? mine[lane * N + n] : 0.0f);
}

// CTA: blockDim.y rows at a time, blockDim.x threads each.
template <class T, class W, int VEC, int E>
__global__ void __launch_bounds__(32 * kMaxWarps) forward_kernel(const Forward a) {
  constexpr int C = E / VEC;
  __shared__ float space[2][kMaxWarps];
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  const float per = 1.0f / (float)a.cols;
  Raw<T, VEC> x[C], r[C];
  bool in[C];
#pragma unroll
  for (int c = 0; c < C; ++c) in[c] = (int64_t)(c * blockDim.x + threadIdx.x) * VEC < a.cols;
  auto at = [&](int c) { return (int64_t)(c * blockDim.x + threadIdx.x) * VEC; };
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const bool there = in[c] && row < a.rows;
      if (there)
        x[c].load((const T*)a.x + row * a.ldx + at(c));
      else
        x[c].zero();
      if (a.r) {
        if (there)
          r[c].load((const T*)a.r + row * a.ldr + at(c));
        else
          r[c].zero();
      }
    }
  };
  int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  fetch(row);
  // all rows of a CTA make the same number of steps: they meet in row_sums
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * blockDim.y; first < a.rows; first += step, row += step) {
    float v[E];
    const bool there = row < a.rows;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (a.r) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[c].set(i, x[c].at(i) + r[c].at(i));
        if (there && in[c]) x[c].store((T*)a.h + row * a.ldh + at(c));
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[c * VEC + i] = x[c].at(i);
    }
    fetch(row + step);
    float mean = 0.0f;
    if (!a.rms) {
      float sum[1] = {0.0f};
#pragma unroll
      for (int i = 0; i < E; ++i) sum[0] += v[i];
      row_sums(sum, space[turn]);
      turn ^= 1;
      mean = sum[0] * per;
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = in[i / VEC] ? v[i] - mean : 0.0f;
    }
    float sq[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < E; ++i) sq[0] = fmaf(v[i], v[i], sq[0]);
    row_sums(sq, space[turn]);
    turn ^= 1;
    const float inv = 1.0f / sqrtf(sq[0] * per + a.eps);
    if (!there) continue;
    if (a.stats && threadIdx.x == 0) {
      if (!a.rms) a.stats[row] = mean;
      a.stats[(a.rms ? 0 : a.rows) + row] = inv;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!in[c]) continue;
      float w[VEC], b[VEC];
      load_weights<W, VEC>((const W*)a.w, at(c), true, 1.0f, w);
      load_weights<W, VEC>((const W*)a.b, at(c), true, 0.0f, b);
      Raw<T, VEC> y;
#pragma unroll
      for (int i = 0; i < VEC; ++i) y.set(i, fmaf(v[c * VEC + i] * inv, w[i], b[i]));
      y.store((T*)a.y + row * a.ldy + at(c));
    }
  }
}

// Any number of columns: a CTA per row at a time.
template <class T, class W>
__global__ void __launch_bounds__(1024) forward_long_kernel(const Forward a) {
  __shared__ float space[2][kMaxWarps];
  const float per = 1.0f / (float)a.cols;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = (const T*)a.x + row * a.ldx;
    if (a.r) {
      const T* r = (const T*)a.r + row * a.ldr;
      T* h = (T*)a.h + row * a.ldh;
      for (int64_t j = threadIdx.x; j < a.cols; j += blockDim.x) h[j] = from_float<T>(to_float(x[j]) + to_float(r[j]));
      x = h;  // a thread reads what it wrote itself
    }
    float mean = 0.0f;
    if (!a.rms) {
      float sum[1] = {0.0f};
      for (int64_t j = threadIdx.x; j < a.cols; j += blockDim.x) sum[0] += to_float(x[j]);
      row_sums(sum, space[0]);
      mean = sum[0] * per;
    }
    float sq[1] = {0.0f};
    for (int64_t j = threadIdx.x; j < a.cols; j += blockDim.x) {
      const float d = to_float(x[j]) - mean;
      sq[0] = fmaf(d, d, sq[0]);
    }
    row_sums(sq, space[1]);
    const float inv = 1.0f / sqrtf(sq[0] * per + a.eps);
    if (a.stats && threadIdx.x == 0) {
      if (!a.rms) a.stats[row] = mean;
      a.stats[(a.rms ? 0 : a.rows) + row] = inv;
    }
    for (int64_t j = threadIdx.x; j < a.cols; j += blockDim.x) {
      const float w = a.w ? to_float(((const W*)a.w)[j]) : 1.0f, b = a.b ? to_float(((const W*)a.b)[j]) : 0.0f;
      ((T*)a.y)[row * a.ldy + j] = from_float<T>(fmaf((to_float(x[j]) - mean) * inv, w, b));
    }
    __syncthreads();  // the sums have been read
  }
}

// A CTA takes every gridDim.x'th set of blockDim.y rows. THREADS: the most it has.
template <class T, class W, int VEC, int E, int THREADS>
__global__ void __launch_bounds__(THREADS) backward_kernel(const Backward a) {
  constexpr int C = E / VEC;
  __shared__ float space[2][2 * kMaxWarps];
  extern __shared__ float sums[];  // [2][cols], where several rows' threads of the CTA meet at the end
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  const float per = 1.0f / (float)a.cols;
  float dw[E], db[E];
#pragma unroll
  for (int i = 0; i < E; ++i) dw[i] = db[i] = 0.0f;
  bool in[C];
#pragma unroll
  for (int c = 0; c < C; ++c) in[c] = (int64_t)(c * blockDim.x + threadIdx.x) * VEC < a.cols;
  auto at = [&](int c) { return (int64_t)(c * blockDim.x + threadIdx.x) * VEC; };
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * blockDim.y; first < a.rows; first += step, turn ^= 1) {
    const int64_t row = first + threadIdx.y;
    const bool there = row < a.rows;
    Raw<T, VEC> h[C], dy[C], dh[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (there && in[c]) {
        h[c].load((const T*)a.h + row * a.ldh + at(c));
        dy[c].load((const T*)a.dy + row * a.lddy + at(c));
        if (a.dh && a.dx) dh[c].load((const T*)a.dh + row * a.lddh + at(c));
      } else {
        h[c].zero();
        dy[c].zero();
      }
    }
    const float mean = there && !a.rms ? a.stats[row] : 0.0f;
    const float inv = there ? a.stats[(a.rms ? 0 : a.rows) + row] : 0.0f;
    float s[2] = {0.0f, 0.0f};
    float xh[E], g[E];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float w[VEC];
      load_weights<W, VEC>((const W*)a.w, at(c), in[c], 1.0f, w);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const int e = c * VEC + i;
        const float d = dy[c].at(i);
        xh[e] = there && in[c] ? (h[c].at(i) - mean) * inv : 0.0f;
        g[e] = d * w[i];
        dw[e] = fmaf(d, xh[e], dw[e]);
        db[e] += d;
        s[0] = fmaf(g[e], xh[e], s[0]);
        s[1] += g[e];
      }
    }
    if (!a.dx) continue;
    row_sums(s, space[turn]);
    const float by = s[0] * per, off = a.rms ? 0.0f : s[1] * per;
    if (!there) continue;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!in[c]) continue;
      Raw<T, VEC> dx;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const int e = c * VEC + i;
        float v = (g[e] - off - xh[e] * by) * inv;
        if (a.dh) v += dh[c].at(i);
        dx.set(i, v);
      }
      dx.store((T*)a.dx + row * a.lddx + at(c));
    }
  }
  if (!a.dw && !a.db) return;
  // the CTA's sums: its rows' threads in turn
  if (blockDim.y > 1) {
    for (int t = 0; t < (int)blockDim.y; ++t) {
      if ((int)threadIdx.y == t) {
#pragma unroll
        for (int c = 0; c < C; ++c)
          if (in[c])
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
              const int e = c * VEC + i;
              float* p = sums + at(c) + i;
              if (t > 0) dw[e] += p[0], db[e] += p[a.cols];
              p[0] = dw[e];
              p[a.cols] = db[e];
            }
      }
      __syncthreads();
    }
  }
  if (threadIdx.y == blockDim.y - 1) {
    float* to = a.parts + (size_t)blockIdx.x * ((a.dw != nullptr) + (a.db != nullptr)) * a.cols;
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (in[c])
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          float* p = to + at(c) + i;
          if (a.dw) {
            *p = dw[c * VEC + i];
            p += a.cols;
          }
          if (a.db) *p = db[c * VEC + i];
        }
  }
}

// Any number of columns: dx by a CTA per row at a time ...
template <class T, class W>
__global__ void __launch_bounds__(1024) backward_long_kernel(const Backward a) {
  __shared__ float space[2 * kMaxWarps];
  const float per = 1.0f / (float)a.cols;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T *h = (const T*)a.h + row * a.ldh, *dy = (const T*)a.dy + row * a.lddy;
    const float mean = a.rms ? 0.0f : a.stats[row], inv = a.stats[(a.rms ? 0 : a.rows) + row];
    float s[2] = {0.0f, 0.0f};
    for (int64_t j = threadIdx.x; j < a.cols; j += blockDim.x) {
      const float g = to_float(dy[j]) * (a.w ? to_float(((const W*)a.w)[j]) : 1.0f);
      s[0] = fmaf(g, (to_float(h[j]) - mean) * inv, s[0]);
      s[1] += g;
    }
    row_sums(s, space);
    const float by = s[0] * per, off = a.rms ? 0.0f : s[1] * per;
    for (int64_t j = threadIdx.x; j < a.cols; j += blockDim.x) {
      const float g = to_float(dy[j]) * (a.w ? to_float(((const W*)a.w)[j]) : 1.0f);
      float v = (g - off - (to_float(h[j]) - mean) * inv * by) * inv;
      if (a.dh) v += to_float(((const T*)a.dh)[row * a.lddh + j]);
      ((T*)a.dx)[row * a.lddx + j] = from_float<T>(v);
    }
    __syncthreads();
  }
}
// ... and the weights' sums by a thread per column over a share of the rows.
template <class T>
__global__ void __launch_bounds__(256) long_sums_kernel(const Backward a) {
  const int64_t share = (a.rows + a.shares - 1) / a.shares, from = blockIdx.y * share;
  const int64_t to = from + share < a.rows ? from + share : a.rows;
  for (int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x; j < a.cols; j += (int64_t)gridDim.x * 256) {
    float dw = 0.0f, db = 0.0f;
    for (int64_t row = from; row < to; ++row) {
      const float mean = a.rms ? 0.0f : a.stats[row], inv = a.stats[(a.rms ? 0 : a.rows) + row];
      const float d = to_float(((const T*)a.dy)[row * a.lddy + j]);
      dw = fmaf(d, (to_float(((const T*)a.h)[row * a.ldh + j]) - mean) * inv, dw);
      db += d;
    }
    float* p = a.parts + (size_t)blockIdx.y * ((a.dw != nullptr) + (a.db != nullptr)) * a.cols + j;
    if (a.dw) {
      *p = dw;
      p += a.cols;
    }
    if (a.db) *p = db;
  }
}

// The shares' sums in their order: a warp's lanes are 32 columns, its warps every 32nd share.
template <class W>
__global__ void __launch_bounds__(1024) join_kernel(const Backward a) {
  __shared__ float space[32][33];
  const int wanted = (a.dw != nullptr) + (a.db != nullptr);
  const int64_t width = wanted * a.cols, j = (int64_t)blockIdx.x * 32 + threadIdx.x;
  float v = 0.0f;
  if (j < width)
    for (int s = threadIdx.y; s < a.shares; s += 32) v += a.parts[(size_t)s * width + j];
  space[threadIdx.y][threadIdx.x] = v;
  __syncthreads();
  if (threadIdx.y != 0 || j >= width) return;
  v = 0.0f;
#pragma unroll
  for (int t = 0; t < 32; ++t) v += space[t][threadIdx.x];
  W* out = (W*)(a.dw && j < a.cols ? a.dw : a.db);
  const int64_t at = j < a.cols ? j : j - a.cols;
  out[at] = from_float<W>(a.accumulate ? to_float(out[at]) + v : v);
}

bool on(const void* p, int64_t ld, int64_t rows, int elem, int bytes) {
  return !p || ((uintptr_t)p % bytes == 0 && (rows <= 1 || (uint64_t)ld * elem % bytes == 0));
}

// Threads of a row, rows of a CTA.
dim3 block_of(int64_t cols, int per_thread, int threads) {
  const int warps = (int)((cols + 32 * per_thread - 1) / (32 * per_thread));
  const int rows = threads / (32 * warps);
  return dim3(32 * warps, rows > 1 ? rows : 1);
}

// Runs f with a type and a vector: f(T, W, integral_constant VEC)
template <class T, class W, class F>
cudaError_t with_vec(int bytes, F&& f) {
  constexpr int kWide = 16 / (int)sizeof(T);
  if (bytes == 16) return f(T(), W(), std::integral_constant<int, kWide>());
  if (bytes == 4 && sizeof(T) == 2) return f(T(), W(), std::integral_constant<int, 2>());
  return f(T(), W(), std::integral_constant<int, 1>());
}
template <class F>
cudaError_t with_types(int dtype, int weight_dtype, int bytes, F&& f) {
  if (dtype == SMAT_F32) return with_vec<float, float>(bytes, f);
  if (weight_dtype == SMAT_F32) return with_vec<bf16, float>(bytes, f);
  return with_vec<bf16, bf16>(bytes, f);
}

}  // namespace

cudaError_t launch_forward(const Forward& a, int dtype, int weight_dtype, int sms, cudaStream_t s) {
  const int elem = dtype == SMAT_BF16 ? 2 : 4;
  auto all_on = [&](int bytes) {
    return a.cols * elem % bytes == 0 && on(a.x, a.ldx, a.rows, elem, bytes) && on(a.r, a.ldr, a.rows, elem, bytes) &&
           on(a.h, a.ldh, a.rows, elem, bytes) && on(a.y, a.ldy, a.rows, elem, bytes);
  };
  const int bytes = all_on(16) ? 16 : all_on(4) ? 4 : 2;
  return with_types(dtype, weight_dtype, bytes, [&](auto t, auto w, auto vec) {
    using T = decltype(t);
    using W = decltype(w);
    constexpr int VEC = decltype(vec)::value;
    if (a.cols > kMaxCols) {
      const int64_t ctas = a.rows < 2 * sms ? a.rows : 2 * sms;
      forward_long_kernel<T, W><<<(unsigned)ctas, 1024, 0, s>>>(a);
      return cudaGetLastError();
    }
    auto go = [&](auto e) {
      constexpr int E = decltype(e)::value;
      const dim3 block = block_of(a.cols, E, 256);
      const int64_t sets = (a.rows + block.y - 1) / block.y;
      const int64_t room = (int64_t)sms * (2048 / (block.x * block.y) / 2 > 0 ? 2048 / (block.x * block.y) / 2 : 1);
      forward_kernel<T, W, VEC, E><<<(unsigned)(sets < room ? sets : room), block, 0, s>>>(a);
      return cudaGetLastError();
    };
    if (a.cols <= 2048) return go(std::integral_constant<int, 8>());
    return go(std::integral_constant<int, 16>());
  });
}

int backward_shares(int64_t rows, int64_t cols, int sms) {
  if (cols > kMaxCols) return (int)(rows < 16 ? rows : 16);
  const dim3 block = block_of(cols, cols <= 2048 ? 8 : 16, 256);
  const int64_t sets = (rows + block.y - 1) / block.y, room = 2 * (int64_t)sms;
  return (int)(sets < room ? sets : room);
}

cudaError_t launch_backward(const Backward& given, int dtype, int weight_dtype, int sms, cudaStream_t s) {
  Backward a = given;
  a.shares = backward_shares(a.rows, a.cols, sms);
  const int elem = dtype == SMAT_BF16 ? 2 : 4, wanted = (a.dw != nullptr) + (a.db != nullptr);
  auto all_on = [&](int bytes) {
    return a.cols * elem % bytes == 0 && on(a.dy, a.lddy, a.rows, elem, bytes) && on(a.h, a.ldh, a.rows, elem, bytes) &&
           on(a.dh, a.lddh, a.rows, elem, bytes) && on(a.dx, a.lddx, a.rows, elem, bytes);
  };
  const int bytes = all_on(16) ? 16 : all_on(4) ? 4 : 2;
  return with_types(dtype, weight_dtype, bytes, [&](auto t, auto w, auto vec) {
    using T = decltype(t);
    using W = decltype(w);
    constexpr int VEC = decltype(vec)::value;
    cudaError_t e = cudaSuccess;
    if (a.rows > 0 && a.cols > kMaxCols) {
      if (a.dx) {
        const int64_t ctas = a.rows < 2 * sms ? a.rows : 2 * sms;
        backward_long_kernel<T, W><<<(unsigned)ctas, 1024, 0, s>>>(a);
        e = cudaGetLastError();
      }
      if (e == cudaSuccess && wanted) {
        const int64_t ctas = (a.cols + 255) / 256;
        long_sums_kernel<T><<<dim3((unsigned)(ctas < 65535 ? ctas : 65535), a.shares), 256, 0, s>>>(a);
        e = cudaGetLastError();
      }
    } else if (a.rows > 0) {
      auto go = [&](auto e, auto threads) {
        constexpr int E = decltype(e)::value, THREADS = decltype(threads)::value;
        const dim3 block = block_of(a.cols, E, 256);
        const size_t bytes = block.y > 1 && wanted ? 2 * (size_t)a.cols * sizeof(float) : 0;
        backward_kernel<T, W, VEC, E, THREADS><<<a.shares, block, bytes, s>>>(a);
        return cudaGetLastError();
      };
      if (a.cols <= 2048)
        e = go(std::integral_constant<int, 8>(), std::integral_constant<int, 256>());
      else if (a.cols <= 8192)
        e = go(std::integral_constant<int, 16>(), std::integral_constant<int, 512>());
      else
        e = go(std::integral_constant<int, 16>(), std::integral_constant<int, 1024>());
    }
    if (e != cudaSuccess || !wanted) return e;
    join_kernel<W><<<(unsigned)((wanted * a.cols + 31) / 32), dim3(32, 32), 0, s>>>(a);
    return cudaGetLastError();
  });
}

}  // namespace norm
}  // namespace smat
