// Layer norm and rms norm, forward and backward (include/smat.h, "norms").
//
// A row is held in registers by some lanes of a warp, a warp or several, E values a thread, so that it is read once: its mean,
// then the squares of what is left (both sums in fp32, over lanes and then warps in a fixed order), then the result. The threads
// walk over the rows with the next row's loads under way. Backward the columns a thread holds are the same for every row, so it
// adds up dw and db for them as it goes; every CTA leaves its sums in the workspace, and a second launch adds those in the CTAs'
// order: no atomics, the same bits every time. Rows of more than kMaxCols columns are read three times by a CTA each (the later
// times mostly from L2).

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

// VEC neighbours as they lie in memory. (Pairs of bf16 are taken apart and made as whole words: element by element a row of 4,096
// took 39 instructions a value, and they bound it.)
template <class T, int VEC>
struct Raw {
  static constexpr int kBytes = VEC * (int)sizeof(T);
  using Word = std::conditional_t<kBytes == 16, uint4,
                                  std::conditional_t<kBytes == 8, uint2, std::conditional_t<kBytes == 4, uint32_t, uint16_t>>>;
  Word u;
  __device__ __forceinline__ void load(const T* p) { u = *reinterpret_cast<const Word*>(p); }
  __device__ __forceinline__ void zero() { u = Word{}; }
  // Those that `has` names, one by one; 0 for the others, which are not read.
  template <class Has>
  __device__ __forceinline__ void load_some(const T* p, Has&& has) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) reinterpret_cast<uint32_t*>(&u)[i] = has(i) ? reinterpret_cast<const uint32_t*>(p)[i] : 0u;
    } else {
      const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
      uint32_t x[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[i] = has(i) ? q[i] : 0u;
#pragma unroll
      for (int i = 0; i + 1 < VEC; i += 2) reinterpret_cast<uint32_t*>(&u)[i / 2] = x[i] | x[i + 1] << 16;
    }
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 4) return reinterpret_cast<const float*>(&u)[i];
    if constexpr (VEC == 1) return __uint_as_float((uint32_t)u << 16);
    if constexpr (sizeof(T) == 2 && VEC > 1) {
      const uint32_t w = reinterpret_cast<const uint32_t*>(&u)[i / 2];
      return __uint_as_float(i % 2 ? w & 0xFFFF0000u : w << 16);
    }
  }
  __device__ __forceinline__ void set(const float (&v)[VEC]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) reinterpret_cast<float*>(&u)[i] = v[i];
    } else if constexpr (VEC == 1) {
      u = __bfloat16_as_ushort(__float2bfloat16_rn(v[0]));
    } else {
#pragma unroll
      for (int i = 0; i < VEC; i += 2) {
        const __nv_bfloat162 w = __floats2bfloat162_rn(v[i], v[i + 1]);
        reinterpret_cast<uint32_t*>(&u)[i / 2] = *reinterpret_cast<const uint32_t*>(&w);
      }
    }
  }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<Word*>(p) = u; }
};

// A vector of weights, from a multiple of VEC on; whole vectors lie on 16 bytes.
template <class W, int VEC>
__device__ __forceinline__ void load_weights(const W* p, int64_t at, bool there, float other, float (&v)[VEC]) {
  constexpr int kWide = 16 / (int)sizeof(W);
#pragma unroll
  for (int i = 0; i < VEC; ++i) v[i] = other;
  if (!p || !there) return;
  if constexpr (VEC % kWide == 0) {
#pragma unroll
    for (int i = 0; i < VEC; i += kWide) {
      Raw<W, kWide> u;
      u.load(p + at + i);
#pragma unroll
      for (int j = 0; j < kWide; ++j) v[i + j] = u.at(j);
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = to_float(p[at + i]);
  }
}

// Weights as they lie in registers: bf16 in pairs
template <class W, int E>
struct Weights {
  float v[E];
  __device__ __forceinline__ void set(int i, float x) { v[i] = x; }
  __device__ __forceinline__ float at(int i) const { return v[i]; }
};
template <int E>
struct Weights<bf16, E> {
  uint32_t v[E / 2];
  __device__ __forceinline__ void set(int i, float x) {
    const uint32_t u = __float_as_uint(x) >> 16;  // a bf16 number's
    v[i / 2] = i % 2 ? v[i / 2] | u << 16 : u;
  }
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(i % 2 ? v[i / 2] & 0xFFFF0000u : v[i / 2] << 16); }
};

// over `width` neighbouring lanes, a power of two
__device__ __forceinline__ float lane_sum(float v, int width) {
#pragma unroll
  for (int d = 16; d > 0; d /= 2) {
    const float other = __shfl_xor_sync(0xFFFFFFFFu, v, d);
    v += d < width ? other : 0.0f;
  }
  return v;
}

// N sums over a row's threads: less than a warp, or whole ones. `space`: [rows of the CTA][warps][N], another one than the last
// call's: a thread that writes to the last call's place has passed this call's barrier, and so has everybody who read it.
template <int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* space) {
  const int width = blockDim.x < 32 ? blockDim.x : 32;
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = lane_sum(v[n], width);
  const int warps = blockDim.x / 32;
  if (warps <= 1) return;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  float* mine = space + (size_t)threadIdx.y * warps * N;
  if (lane == 0)
#pragma unroll
    for (int n = 0; n < N; ++n) mine[warp * N + n] = v[n];
  __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = lane_sum(lane < warps ? mine[lane * N + n] : 0.0f, 32);
}

// The columns that a thread holds, C vectors of VEC. SHIFT: rows do not all start on 16 bytes, but those of all matrices lie alike.
// Vectors are those of memory then, of which a row's first starts before it by as much as the row's address is past 16 bytes, and
// the same for all the rows of a thread, which are a multiple of 16 / sizeof(T) apart. Of a vector that reaches out of the row
// only what is inside is read and written, element by element; what is outside counts as 0.
template <class T, int VEC, int C, bool SHIFT>
struct Columns {
  // (in 32 bits a shifted row is faster, 4099 x 1023 19 us and not 33; a whole one in 64 bits, 8192 x 4096 in fp32 84 and not 110)
  using Place = std::conditional_t<SHIFT, int, int64_t>;
  Place cols, before;
  bool in[C], inside[C];  // the vector meets the row; lies in it
  // first: the thread's first row's place in memory, of any of the matrices
  __device__ __forceinline__ Columns(int64_t n, const void* base, int64_t first)
      : cols((Place)n), before(SHIFT ? (Place)(((uintptr_t)base + (uint64_t)first * sizeof(T)) % 16 / sizeof(T)) : 0) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      in[c] = at(c) < cols && (!SHIFT || at(c) + VEC > 0);
      inside[c] = !SHIFT || (at(c) >= 0 && at(c) + VEC <= cols);
    }
  }
  __device__ __forceinline__ Place at(int c) const {
    const Place first = (Place)(c * blockDim.x + threadIdx.x) * VEC;
    return SHIFT ? first - before : first;
  }
  __device__ __forceinline__ bool has(int c, int i) const { return !SHIFT || (at(c) + i >= 0 && at(c) + i < cols); }
  __device__ __forceinline__ bool whole(int c) const { return inside[c]; }
  __device__ __forceinline__ void load(Raw<T, VEC>& v, const T* row, int c) const {
    if (!SHIFT || whole(c)) {
      v.load(row + at(c));
    } else {
      v.load_some(row + at(c), [&](int i) { return has(c, i); });
    }
  }
  __device__ __forceinline__ void store(const Raw<T, VEC>& v, T* row, int c) const {
    if (whole(c)) {
      v.store(row + at(c));
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (has(c, i)) row[at(c) + i] = from_float<T>(v.at(i));
    }
  }
  template <class W>
  __device__ __forceinline__ void weights(const W* p, int c, float other, float (&v)[VEC]) const {
    if (!SHIFT) {
      load_weights<W, VEC>(p, at(c), in[c], other, v);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = p && has(c, i) ? to_float(p[at(c) + i]) : other;
    }
  }
};

// CTA: blockDim.y rows at a time, blockDim.x threads each.
template <class T, class W, int VEC, int E, int THREADS, bool SHIFT>
__global__ void __launch_bounds__(THREADS, E == 32 || SHIFT ? 512 / THREADS + (THREADS > 512) : 1024 / THREADS)
    forward_kernel(const Forward a) {
  constexpr int C = E / VEC;
  __shared__ float space[2][kMaxWarps];
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  const float per = 1.0f / (float)a.cols;
  Raw<T, VEC> x[C], r[C];
  const Columns<T, VEC, C, SHIFT> own(a.cols, a.x, ((int64_t)blockIdx.x * blockDim.y + threadIdx.y) * a.ldx);
  const bool(&in)[C] = own.in;
  Weights<W, E> ws, bs;  // SHIFT: a thread's weights lie off every boundary; it keeps them
  if (SHIFT) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float w[VEC], b[VEC];
      own.weights((const W*)a.w, c, 1.0f, w);
      own.weights((const W*)a.b, c, 0.0f, b);
#pragma unroll
      for (int i = 0; i < VEC; ++i) ws.set(c * VEC + i, w[i]), bs.set(c * VEC + i, b[i]);
    }
  }
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const bool there = in[c] && row < a.rows;
      if (there)
        own.load(x[c], (const T*)a.x + row * a.ldx, c);
      else
        x[c].zero();
      if (a.r) {
        if (there)
          own.load(r[c], (const T*)a.r + row * a.ldr, c);
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
        float sum[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum[i] = x[c].at(i) + r[c].at(i);
        x[c].set(sum);
        if (there && in[c]) own.store(x[c], (T*)a.h + row * a.ldh, c);
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
      for (int c = 0; c < C; ++c) {
        const float less = in[c] ? mean : 0.0f;  // columns that are not there hold 0
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[c * VEC + i] -= less;
        if (SHIFT && !own.whole(c)) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) v[c * VEC + i] = own.has(c, i) ? v[c * VEC + i] : 0.0f;
        }
      }
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
      if (SHIFT) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) w[i] = ws.at(c * VEC + i), b[i] = bs.at(c * VEC + i);
      } else {
        own.weights((const W*)a.w, c, 1.0f, w);
        own.weights((const W*)a.b, c, 0.0f, b);
      }
      float out[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) out[i] = fmaf(v[c * VEC + i] * inv, w[i], b[i]);
      Raw<T, VEC> y;
      y.set(out);
      own.store(y, (T*)a.y + row * a.ldy, c);
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

// A CTA takes every gridDim.x'th set of blockDim.y rows. THREADS: the most it has, CTAS: how many are to share an SM; AHEAD: the
// next rows' loads are under way while a row is worked on.
template <class T, class W, int VEC, int E, int THREADS, int CTAS, bool AHEAD, bool SHIFT>
__global__ void __launch_bounds__(THREADS, CTAS) backward_kernel(const Backward a) {
  constexpr int C = E / VEC;
  __shared__ float space[2][2 * kMaxWarps];
  extern __shared__ float sums[];  // [2][cols], where several rows' threads of the CTA meet at the end
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  const float per = 1.0f / (float)a.cols;
  const bool add = a.dh && a.dx;
  float dw[E], db[E];
  Weights<W, E> w;
  const Columns<T, VEC, C, SHIFT> own(a.cols, a.dy, ((int64_t)blockIdx.x * blockDim.y + threadIdx.y) * a.lddy);
  const bool(&in)[C] = own.in;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    float v[VEC];
    own.weights((const W*)a.w, c, 1.0f, v);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      w.set(c * VEC + i, v[i]);
      dw[c * VEC + i] = db[c * VEC + i] = 0.0f;
    }
  }
  struct Row {
    Raw<T, VEC> h[C], dy[C], dh[C];
    float mean, inv;
  };
  auto fetch = [&](int64_t row) {
    Row r;
    const bool there = row < a.rows;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      r.h[c].zero(), r.dy[c].zero(), r.dh[c].zero();
      if (there && in[c]) {
        own.load(r.h[c], (const T*)a.h + row * a.ldh, c);
        own.load(r.dy[c], (const T*)a.dy + row * a.lddy, c);
        if (add) own.load(r.dh[c], (const T*)a.dh + row * a.lddh, c);
      }
    }
    r.mean = there && !a.rms ? a.stats[row] : 0.0f;
    r.inv = there ? a.stats[(a.rms ? 0 : a.rows) + row] : 0.0f;
    return r;
  };
  int turn = 0;
  int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  Row next;
  if (AHEAD) next = fetch(row);
  for (int64_t first = (int64_t)blockIdx.x * blockDim.y; first < a.rows; first += step, row += step, turn ^= 1) {
    const bool there = row < a.rows;
    const Row r = AHEAD ? next : fetch(row);
    if (AHEAD) next = fetch(row + step);
    // of a row that is not there, or a column, dy is 0, and with it all that is added up
    auto xh = [&](int c, int i) { return (r.h[c].at(i) - r.mean) * r.inv; };
    auto g = [&](int c, int i) { return r.dy[c].at(i) * w.at(c * VEC + i); };
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const int e = c * VEC + i;
        const float d = r.dy[c].at(i), x = xh(c, i);
        dw[e] = fmaf(d, x, dw[e]);
        db[e] += d;
        s[0] = fmaf(g(c, i), x, s[0]);
        s[1] += g(c, i);
      }
    }
    if (!a.dx) continue;
    row_sums(s, space[turn]);
    const float by = s[0] * per, off = a.rms ? 0.0f : s[1] * per;
    if (!there) continue;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!in[c]) continue;
      float out[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) out[i] = fmaf(-by, xh(c, i), g(c, i) - off) * r.inv;
      if (add) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) out[i] += r.dh[c].at(i);
      }
      Raw<T, VEC> dx;
      dx.set(out);
      own.store(dx, (T*)a.dx + row * a.lddx, c);
    }
  }
  if (!a.dw && !a.db) return;
  // the CTA's sums: rows' lanes of a warp first (where they hold the same columns), then what is left in turn
  const bool narrow = !SHIFT && blockDim.x < 32;
  const int thread = threadIdx.y * blockDim.x + threadIdx.x;
  if (narrow) {
#pragma unroll
    for (int e = 0; e < E; ++e)
      for (int d = blockDim.x; d < 32; d *= 2) {
        dw[e] += __shfl_xor_sync(0xFFFFFFFFu, dw[e], d);
        db[e] += __shfl_xor_sync(0xFFFFFFFFu, db[e], d);
      }
  }
  const int turns = narrow ? (int)(blockDim.x * blockDim.y / 32) : (int)blockDim.y, mine = narrow ? thread / 32 : (int)threadIdx.y;
  const bool takes_part = !narrow || thread % 32 < (int)blockDim.x;
  for (int t = 0; t < turns - 1; ++t) {
    if (mine == t && takes_part) {
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (in[c])
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            const int e = c * VEC + i;
            float* p = sums + own.at(c) + i;
            if (!own.has(c, i)) continue;
            if (t > 0) dw[e] += p[0], db[e] += p[a.cols];
            p[0] = dw[e];
            p[a.cols] = db[e];
          }
    }
    __syncthreads();
  }
  if (mine != turns - 1 || !takes_part) return;
  float* to = a.parts + (size_t)blockIdx.x * ((a.dw != nullptr) + (a.db != nullptr)) * a.cols;
#pragma unroll
  for (int c = 0; c < C; ++c)
    if (in[c])
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const int e = c * VEC + i;
        const float* q = sums + own.at(c) + i;
        float* p = to + own.at(c) + i;
        if (!own.has(c, i)) continue;
        if (a.dw) {
          *p = turns > 1 ? dw[e] + q[0] : dw[e];
          p += a.cols;
        }
        if (a.db) *p = turns > 1 ? db[e] + q[a.cols] : db[e];
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
    for (int s = threadIdx.y; s < a.shares; s += 32 * 8) {
      float x[8];  // asked for together; those behind the last one are the last one's and are not added
#pragma unroll
      for (int t = 0; t < 8; ++t) x[t] = a.parts[(size_t)min(s + 32 * t, a.shares - 1) * width + j];
#pragma unroll
      for (int t = 0; t < 8; ++t) v += s + 32 * t < a.shares ? x[t] : 0.0f;
    }
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

// Threads of a row (some of a warp's lanes or whole warps), rows of a CTA.
dim3 block_of(int64_t cols, int per_thread, int threads) {
  const int64_t needed = (cols + per_thread - 1) / per_thread;
  int wide = 4;
  while (wide < 32 && wide < needed) wide *= 2;
  if (needed > 32) wide = (int)((needed + 31) / 32 * 32);
  return dim3(wide, threads / wide > 1 ? threads / wide : 1);
}

// How rows are read: whole vectors from 16 bytes on, vectors of memory that a row starts inside of, or element by element. The
// second pays forward in bf16 from some 800 columns on (4099 rows, layer norm with residual, us, shifted and one by one: 255 columns
// 12.5 and 7.6, 511 16.9 and 16.8, 767 20 and 18, 1023 19 and 22 to 26, 2039 34 and 42, 4095 72 and 105; in fp32 not: 4095 127 and
// 109), and back through long rows (with dh, bf16: 1023 31 and 18, 2039 37 and 32, 4095 100 and 137, 2048 x 11007 86 and 298; fp32:
// 1023 45 and 21, 4095 82 and 152, 2048 x 11007 120 and 247).
enum Way { kWhole, kShifted, kSingly };

// Runs f with types, a vector and whether rows are shifted: f(T, W, integral_constant VEC, bool_constant SHIFT). F32_SHIFTS: fp32
// rows may be.
template <class T, class W, bool SHIFTS, class F>
cudaError_t with_vec(Way way, F&& f) {
  constexpr int kWide = 16 / (int)sizeof(T);
  if (way == kWhole) return f(T(), W(), std::integral_constant<int, kWide>(), std::false_type());
  if constexpr (SHIFTS) {
    if (way == kShifted) return f(T(), W(), std::integral_constant<int, kWide>(), std::true_type());
  }
  return f(T(), W(), std::integral_constant<int, 1>(), std::false_type());
}
template <bool F32_SHIFTS, class F>
cudaError_t with_types(int dtype, int weight_dtype, Way way, F&& f) {
  if (dtype == SMAT_F32) return with_vec<float, float, F32_SHIFTS>(way, f);
  if (weight_dtype == SMAT_F32) return with_vec<bf16, float, true>(way, f);
  return with_vec<bf16, bf16, true>(way, f);
}

// Matrices of a call, those that are there
struct Lie {
  int elem;
  int64_t rows, cols;
  bool whole = true, alike = true;
  uintptr_t start = 0, stride = 0;
  bool any = false;
  Lie(int dtype, int64_t m, int64_t n) : elem(dtype == SMAT_BF16 ? 2 : 4), rows(m), cols(n) { whole = n * elem % 16 == 0; }
  Lie& add(const void* p, int64_t ld) {
    if (!p) return *this;
    const uintptr_t at = (uintptr_t)p % 16, by = rows > 1 ? (uint64_t)ld * elem % 16 : 0;
    whole = whole && at == 0 && by == 0;
    alike = alike && (!any || (at == start && by == stride));
    start = at, stride = by, any = true;
    return *this;
  }
  // `pays`: whether shifted rows are faster than single elements
  Way way(const void* w, const void* b, bool pays) const {
    if (whole && ((uintptr_t)w | (uintptr_t)b) % 16 == 0) return kWhole;
    return alike && pays ? kShifted : kSingly;
  }
};

// A grid whose rows of a thread lie alike: their distance is a multiple of 16 / elem rows.
int64_t whole_steps(int64_t ctas) { return (ctas + 7) / 8 * 8; }

}  // namespace

cudaError_t launch_forward(const Forward& a, int dtype, int weight_dtype, int sms, cudaStream_t s) {
  const Way way = Lie(dtype, a.rows, a.cols).add(a.x, a.ldx).add(a.r, a.ldr).add(a.h, a.ldh).add(a.y, a.ldy).way(a.w, a.b, dtype == SMAT_BF16 && a.cols > 800);
  return with_types<false>(dtype, weight_dtype, way, [&](auto t, auto w, auto vec, auto shift) {
    using T = decltype(t);
    using W = decltype(w);
    constexpr int VEC = decltype(vec)::value;
    constexpr bool SHIFT = decltype(shift)::value;
    const int64_t cols = a.cols + (SHIFT ? VEC - 1 : 0);  // with those before a row's first
    if (cols > kMaxCols) {
      const int64_t ctas = a.rows < 2 * sms ? a.rows : 2 * sms;
      forward_long_kernel<T, W><<<(unsigned)ctas, 1024, 0, s>>>(a);
      return cudaGetLastError();
    }
    auto go = [&](auto e, auto threads) {
      constexpr int E = decltype(e)::value, THREADS = decltype(threads)::value;
      const dim3 block = block_of(cols, E, 256);
      const int64_t sets = (a.rows + block.y - 1) / block.y;
      const int64_t room = (int64_t)sms * (E == 32 ? 3 : 1024 / THREADS), ctas = sets < room ? sets : room;
      forward_kernel<T, W, VEC, E, THREADS, SHIFT><<<(unsigned)(SHIFT ? whole_steps(ctas) : ctas), block, 0, s>>>(a);
      return cudaGetLastError();
    };
    using std::integral_constant;
    if constexpr (VEC * sizeof(T) == 16 && !SHIFT) {
      // a warp per row, which then meets nobody
      if (cols > 512 && cols <= 1024 && a.rows >= 4 * sms) return go(integral_constant<int, 32>(), integral_constant<int, 256>());
    }
    if (cols <= 256 || (cols <= 2048 && (cols > 512 || a.rows < 4 * sms)))
      return go(integral_constant<int, 8>(), integral_constant<int, 256>());
    if (cols <= 4096) return go(integral_constant<int, 16>(), integral_constant<int, 256>());
    if (cols <= 8192) return go(integral_constant<int, 16>(), integral_constant<int, 512>());
    return go(integral_constant<int, 16>(), integral_constant<int, 1024>());
  });
}

// Values a thread, most threads and CTAs per SM of backward_kernel for so many columns.
struct Shape {
  int each, threads, ctas;
};
// What was measured (layer norm with dh, us, memory would take): bf16 8223 x 1024 with 8 values 22, with 32 (a warp per row) 24, 10;
// 8192 x 4096 with 16 values 69, with 32 77, with 8 (512 threads) 71, 40; 2048 x 11008 with 16 values (1,024 threads, whose 64
// registers do not hold them) 102, with 32 64, 27. fp32 8223 x 1024 with 8 values 21, 20; 8192 x 4096 with 16 88, 79.
Shape shape_of(int64_t cols, bool f32) {
  if (cols <= 2048) return {8, 256, f32 ? 2 : 3};
  if (cols <= 4096) return {16, 256, 2};
  if (cols <= 8192) return {16, 512, 1};
  if (f32) return {16, 1024, 1};
  return cols <= 12288 ? Shape{32, 384, 1} : Shape{32, 512, 1};
}

int backward_shares(int64_t rows, int64_t cols, int dtype, int sms) {
  if (cols > kMaxCols) return (int)(rows < 16 ? rows : 16);
  const Shape shape = shape_of(cols, dtype == SMAT_F32);
  const dim3 block = block_of(cols, shape.each, 256);
  const int64_t sets = (rows + block.y - 1) / block.y, room = shape.ctas * (int64_t)sms;
  return (int)whole_steps(sets < room ? sets : room);
}

cudaError_t launch_backward(const Backward& given, int dtype, int weight_dtype, int sms, cudaStream_t s) {
  Backward a = given;
  a.shares = backward_shares(a.rows, a.cols, dtype, sms);
  const int wanted = (a.dw != nullptr) + (a.db != nullptr);
  const Way way = Lie(dtype, a.rows, a.cols)
                      .add(a.dy, a.lddy)
                      .add(a.h, a.ldh)
                      .add(a.dx ? a.dh : nullptr, a.lddh)
                      .add(a.dx, a.lddx)
                      .way(a.w, nullptr, a.cols > 2048);
  return with_types<true>(dtype, weight_dtype, way, [&](auto t, auto w, auto vec, auto shift) {
    using T = decltype(t);
    using W = decltype(w);
    constexpr int VEC = decltype(vec)::value;
    constexpr bool SHIFT = decltype(shift)::value;
    cudaError_t e = cudaSuccess;
    const int64_t cols = a.cols + (SHIFT ? VEC - 1 : 0);  // with those before a row's first
    if (a.rows > 0 && cols > kMaxCols) {
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
      const Shape shape = shape_of(cols, sizeof(T) == 4);
      const dim3 block = block_of(cols, shape.each, 256);
      const size_t bytes = block.y > 1 && wanted ? 2 * (size_t)a.cols * sizeof(float) : 0;
      // registers for the next rows' loads: rows in whole vectors, 8 values a thread or 16 in bf16
      constexpr bool kVec = VEC * sizeof(T) == 16;
      auto go = [&](auto e, auto threads, auto ctas) {
        constexpr int E = decltype(e)::value, THREADS = decltype(threads)::value, CTAS = decltype(ctas)::value;
        backward_kernel<T, W, VEC, E, THREADS, CTAS, kVec && (E == 8 || (E == 16 && sizeof(T) == 2)), SHIFT><<<a.shares, block, bytes, s>>>(a);
        return cudaGetLastError();
      };
      using std::integral_constant;
      if (shape.each == 8) {
        if constexpr (!SHIFT)  // shifted rows are longer
          e = go(integral_constant<int, 8>(), integral_constant<int, 256>(), integral_constant<int, sizeof(T) == 4 ? 2 : 3>());
      } else if (shape.threads == 256)
        e = go(integral_constant<int, 16>(), integral_constant<int, 256>(), integral_constant<int, 2>());
      else if (shape.threads == 512 && shape.each == 16)
        e = go(integral_constant<int, 16>(), integral_constant<int, 512>(), integral_constant<int, 1>());
      else if constexpr (sizeof(T) == 4)
        e = go(integral_constant<int, 16>(), integral_constant<int, 1024>(), integral_constant<int, 1>());
      else if (shape.threads == 384)
        e = go(integral_constant<int, 32>(), integral_constant<int, 384>(), integral_constant<int, 1>());
      else
        e = go(integral_constant<int, 32>(), integral_constant<int, 512>(), integral_constant<int, 1>());
    }
    if (e != cudaSuccess || !wanted) return e;
    join_kernel<W><<<(unsigned)((wanted * a.cols + 31) / 32), dim3(32, 32), 0, s>>>(a);
    return cudaGetLastError();
  });
}

}  // namespace norm
}  // namespace smat
