// Activations in 8 bits (include/smat.h, "linear layers"): a matrix saved, read back through an activation, a
// gradient times the activation's slope at saved values, and a gradient's sums over its rows.
//
// All are one pass over memory. A thread takes 16 columns of a row at a time: 32 bytes of bf16 (one 256-bit access, a whole
// sector, or two of 16 bytes) and 16 bytes of q (or two of 8); the two threads of a group of 32 exchange their largest
// magnitude by one shuffle. Matrices whose rows do not start there are taken by warps that read and write 32 neighbours at
// a time and hand each lane its 16 columns through shared memory (8192 x 8191 bf16 saved in 78 us and read back in 82;
// element by element 167 and 360). Rows on 32 bytes run at 6.1 to 6.6 TB/s from 8191 x 11008 on, unaligned ones at 2.5;
// reading back through the erf form of GELU (bf16 68 us for 8191 x 11008, others 45) is bound by its instructions. A gradient
// times slopes: bf16 76 us (6.0 TB/s; GELU 87), fp32 118 (6.9, part of it from L2); 8192 x 8191 141 and 130 us.

#include "smat_linear.cuh"
#include "smat_linear.h"

namespace smat {
namespace lin {
namespace {

constexpr int kUnit = 16;      // columns per thread and step
constexpr int kThreads = 256;  // of the elementwise kernels

// How a matrix' rows may be accessed: a whole unit of 16 values at once, in two halves, or value by value
enum Access : int { kWhole, kHalves, kEach };

template <class T>
__device__ __forceinline__ void load_unit(const T* p, int count, Access how, float (&v)[kUnit]) {
  if (how != kEach && count == kUnit) {
    if constexpr (sizeof(T) == 2) {
      uint32_t w[8];
      if (how == kWhole) {
        asm volatile("ld.global.nc.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                     : "l"(p));
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint4 u = __ldg(reinterpret_cast<const uint4*>(p) + h);
          w[4 * h] = u.x, w[4 * h + 1] = u.y, w[4 * h + 2] = u.z, w[4 * h + 3] = u.w;
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    } else if (how == kWhole) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        asm volatile("ld.global.nc.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=f"(v[8 * h]), "=f"(v[8 * h + 1]), "=f"(v[8 * h + 2]), "=f"(v[8 * h + 3]), "=f"(v[8 * h + 4]),
                       "=f"(v[8 * h + 5]), "=f"(v[8 * h + 6]), "=f"(v[8 * h + 7])
                     : "l"(p + 8 * h));
    } else {
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const float4 u = __ldg(reinterpret_cast<const float4*>(p) + h);
        v[4 * h] = u.x, v[4 * h + 1] = u.y, v[4 * h + 2] = u.z, v[4 * h + 3] = u.w;
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kUnit; ++i) v[i] = i < count ? to_float(p[i]) : 0.0f;
}

template <class T>
__device__ __forceinline__ void store_unit(T* p, int count, Access how, const float (&v)[kUnit]) {
  if (how != kEach && count == kUnit) {
    if constexpr (sizeof(T) == 2) {
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&b);
      }
      if (how == kWhole) {
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                     "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
      } else {
        reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
      }
    } else if (how == kWhole) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p + 8 * h), "f"(v[8 * h]),
                     "f"(v[8 * h + 1]), "f"(v[8 * h + 2]), "f"(v[8 * h + 3]), "f"(v[8 * h + 4]), "f"(v[8 * h + 5]),
                     "f"(v[8 * h + 6]), "f"(v[8 * h + 7])
                     : "memory");
    } else {
#pragma unroll
      for (int h = 0; h < 4; ++h)
        reinterpret_cast<float4*>(p)[h] = make_float4(v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kUnit; ++i)
    if (i < count) p[i] = from_float<T>(v[i]);
}

__device__ __forceinline__ void load_q(const int8_t* p, int count, Access how, uint32_t (&w)[4]) {
  if (how != kEach && count == kUnit) {
    if (how == kWhole) {
      const uint4 u = __ldg(reinterpret_cast<const uint4*>(p));
      w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
    } else {
      const uint2 u = __ldg(reinterpret_cast<const uint2*>(p)), t = __ldg(reinterpret_cast<const uint2*>(p) + 1);
      w[0] = u.x, w[1] = u.y, w[2] = t.x, w[3] = t.y;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = 0;
#pragma unroll
  for (int i = 0; i < kUnit; ++i)
    if (i < count) w[i / 4] |= (uint32_t)(uint8_t)p[i] << (8 * (i % 4));
}

__device__ __forceinline__ void store_q(int8_t* p, int count, Access how, const uint32_t (&w)[4]) {
  if (how != kEach && count == kUnit) {
    if (how == kWhole) {
      *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      reinterpret_cast<uint2*>(p)[0] = make_uint2(w[0], w[1]);
      reinterpret_cast<uint2*>(p)[1] = make_uint2(w[2], w[3]);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kUnit; ++i)
    if (i < count) p[i] = (int8_t)(w[i / 4] >> (8 * (i % 4)));
}

// q and e of 16 values, of which the other half of the group is the neighbouring lane's (`pair`: both lanes)
__device__ __forceinline__ uint32_t pack_unit(const float (&v)[kUnit], unsigned pair, uint32_t (&w)[4]) {
  float big = 0.0f;
#pragma unroll
  for (int i = 0; i < kUnit; ++i) big = larger(big, v[i]);
  uint32_t top = __float_as_uint(big);
  top = max(top, __shfl_xor_sync(pair, top, 1));
  const uint32_t ex = pack_exponent(top);
  pack_words<4>(v, ex, w);
  return ex;
}

// A warp's piece of a matrix whose rows start anywhere: 512 values, `seg` columns (a power of two from 32 on) of 512 / seg
// rows. They come and go 32 neighbours at a time; lane t's unit is values 16 t .. 16 t + 15, in shared memory 20 apart, so
// that eight lanes' accesses of 16 bytes meet in no bank.
constexpr int kPiece = 512, kPieceFloats = kPiece / kUnit * 20;
__device__ __forceinline__ int piece_place(int i) { return i / kUnit * 20 + i % kUnit; }

struct Piece {
  int shift;       // seg = 1 << shift
  int rows, cols;  // there, from the piece's first row and column on
  // 512 neighbours of one row, all there: no place to work out, nothing to leave out
  __device__ __forceinline__ bool full() const { return shift == 9 && cols >= kPiece; }
  __device__ __forceinline__ bool there(int i) const { return (i >> shift) < rows && (i & ((1 << shift) - 1)) < cols; }
  __device__ __forceinline__ int64_t at(int i, int64_t ld) const {
    return (int64_t)(i >> shift) * ld + (i & ((1 << shift) - 1));
  }
};
template <class T>
__device__ __forceinline__ void piece_in(const Piece& s, const T* p, int64_t ld, float* buf, float (&v)[kUnit]) {
  const int lane = threadIdx.x % 32;
  float x[kUnit];
  if (s.full()) {
#pragma unroll
    for (int t = 0; t < kUnit; ++t) x[t] = to_float(p[32 * t + lane]);
  } else {
#pragma unroll
    for (int t = 0; t < kUnit; ++t) x[t] = s.there(32 * t + lane) ? to_float(p[s.at(32 * t + lane, ld)]) : 0.0f;
  }
  __syncwarp();
#pragma unroll
  for (int t = 0; t < kUnit; ++t) buf[piece_place(lane) + 40 * t] = x[t];
  __syncwarp();
#pragma unroll
  for (int t = 0; t < kUnit; t += 4)
    *reinterpret_cast<float4*>(v + t) = *reinterpret_cast<const float4*>(buf + 20 * lane + t);
}
template <class T>
__device__ __forceinline__ void piece_out(const Piece& s, T* p, int64_t ld, float* buf, const float (&v)[kUnit]) {
  const int lane = threadIdx.x % 32;
  __syncwarp();
#pragma unroll
  for (int t = 0; t < kUnit; t += 4)
    *reinterpret_cast<float4*>(buf + 20 * lane + t) = make_float4(v[t], v[t + 1], v[t + 2], v[t + 3]);
  __syncwarp();
  if (s.full()) {
#pragma unroll
    for (int t = 0; t < kUnit; ++t) p[32 * t + lane] = from_float<T>(buf[piece_place(lane) + 40 * t]);
  } else {
#pragma unroll
    for (int t = 0; t < kUnit; ++t)
      if (s.there(32 * t + lane)) p[s.at(32 * t + lane, ld)] = from_float<T>(buf[piece_place(lane) + 40 * t]);
  }
}
__device__ __forceinline__ void piece_q_in(const Piece& s, const int8_t* p, int64_t ld, float* buf, uint32_t (&w)[4]) {
  const int lane = threadIdx.x % 32;
  int8_t* bytes = reinterpret_cast<int8_t*>(buf);
  int8_t x[kUnit];
  if (s.full()) {
#pragma unroll
    for (int t = 0; t < kUnit; ++t) x[t] = p[32 * t + lane];
  } else {
#pragma unroll
    for (int t = 0; t < kUnit; ++t) x[t] = s.there(32 * t + lane) ? p[s.at(32 * t + lane, ld)] : 0;
  }
  __syncwarp();
#pragma unroll
  for (int t = 0; t < kUnit; ++t) bytes[32 * t + lane] = x[t];
  __syncwarp();
  const uint4 u = *reinterpret_cast<const uint4*>(bytes + kUnit * lane);
  w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
}
__device__ __forceinline__ void piece_q_out(const Piece& s, int8_t* p, int64_t ld, float* buf, const uint32_t (&w)[4]) {
  const int lane = threadIdx.x % 32;
  int8_t* bytes = reinterpret_cast<int8_t*>(buf);
  __syncwarp();
  *reinterpret_cast<uint4*>(bytes + kUnit * lane) = make_uint4(w[0], w[1], w[2], w[3]);
  __syncwarp();
  if (s.full()) {
#pragma unroll
    for (int t = 0; t < kUnit; ++t) p[32 * t + lane] = bytes[32 * t + lane];
  } else {
#pragma unroll
    for (int t = 0; t < kUnit; ++t)
      if (s.there(32 * t + lane)) p[s.at(32 * t + lane, ld)] = bytes[32 * t + lane];
  }
}
// The pieces of a matrix, dealt out to `warps` warps: body(piece, row, column) with `unit` = this lane's row and column in it
template <class Body>
__device__ __forceinline__ void each_piece(int64_t rows, int64_t cols, int64_t warp, int64_t warps, Body&& body) {
  int shift = 9;
  while (shift > 5 && (1 << (shift - 1)) >= cols) --shift;
  const int64_t high = kPiece >> shift, across = (cols + (1 << shift) - 1) >> shift, down = (rows + high - 1) / high;
  for (int64_t n = warp; n < across * down; n += warps) {
    const int64_t r = n / across * high, c = (n % across) << shift;
    const Piece s = {shift, (int)(rows - r < high ? rows - r : high),
                     (int)(cols - c < kPiece ? cols - c : kPiece)};
    body(s, r, c);
  }
}

// The threads' walk over a matrix: blockDim.x threads side by side along a row, blockDim.y rows, steps of the grid.
// Units come in pairs (a group of 32), so both threads of a pair run every step.
#define SMAT_EACH_UNIT(cols, rows)                                                                     \
  const int pairs = (int)(((cols) + kGroup - 1) / kGroup) * 2;                                         \
  for (int64_t r = (int64_t)blockIdx.y * blockDim.y + threadIdx.y; r < (rows);                         \
       r += (int64_t)gridDim.y * blockDim.y)                                                           \
    for (int u = (int)(blockIdx.x * blockDim.x + threadIdx.x); u < pairs; u += (int)(gridDim.x * blockDim.x))

template <class T>
__global__ void __launch_bounds__(kThreads) pack8_kernel(const T* x, int64_t ldx, int8_t* q, int64_t ldq, uint8_t* e,
                                                         int64_t lde, int64_t rows, int64_t cols, Access ax, Access aq) {
  SMAT_EACH_UNIT(cols, rows) {
    const int64_t c = (int64_t)u * kUnit;
    const int count = (int)(cols - c < 0 ? 0 : (cols - c < kUnit ? cols - c : kUnit));
    float v[kUnit];
    load_unit(x + r * ldx + c, count, ax, v);
    // the other half of the group: the neighbouring thread (blockDim.x is even, so both are in this warp and run
    // the same steps)
    uint32_t w[4];
    const uint32_t ex = pack_unit(v, 3u << ((threadIdx.x + threadIdx.y * blockDim.x) & 30), w);
    if ((u & 1) == 0) e[r * lde + u / 2] = (uint8_t)ex;
    store_q(q + r * ldq + c, count, aq, w);
  }
}

// The same for rows that start anywhere.
template <class T>
__global__ void __launch_bounds__(kThreads, 4)
    pack8_pieces_kernel(const T* x, int64_t ldx, int8_t* q, int64_t ldq, uint8_t* e, int64_t lde, int64_t rows, int64_t cols) {
  __shared__ __align__(16) float space[kThreads / 32][kPieceFloats];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  float* buf = space[warp];
  each_piece(rows, cols, (int64_t)blockIdx.x * (kThreads / 32) + warp, (int64_t)gridDim.x * (kThreads / 32),
             [&](const Piece& s, int64_t r, int64_t c) {
               float v[kUnit];
               piece_in(s, x + r * ldx + c, ldx, buf, v);
               uint32_t w[4];
               const uint32_t ex = pack_unit(v, 0xFFFFFFFFu, w);
               const int first = lane * kUnit;
               if ((lane & 1) == 0 && s.there(first))
                 e[(r + (first >> s.shift)) * lde + (c + (first & ((1 << s.shift) - 1))) / kGroup] = (uint8_t)ex;
               piece_q_out(s, q + r * ldq + c, ldq, buf, w);
             });
}

// act(h^) of one unit, or dy * act'(h^) where DY (v: dy in, the result out)
template <class T, int ACT, bool DY>
__device__ __forceinline__ void value_unit(const uint32_t (&w)[4], uint32_t e, float (&v)[kUnit]) {
  float h[kUnit];
  unpack_words8<4>(w, e, h);
#pragma unroll
  for (int i = 0; i < kUnit; ++i) v[i] = DY ? v[i] * act_slope<ACT, T>(h[i]) : act_value<ACT, T>(h[i]);
}

template <class T, int ACT, bool DY>
__global__ void __launch_bounds__(kThreads)
    unpack8_kernel(const int8_t* q, int64_t ldq, const uint8_t* e, int64_t lde, const T* dy, int64_t lddy, T* out,
                   int64_t ldout, int64_t rows, int64_t cols, Access aq, Access ady, Access aout) {
  SMAT_EACH_UNIT(cols, rows) {
    const int64_t c = (int64_t)u * kUnit;
    const int count = (int)(cols - c < 0 ? 0 : (cols - c < kUnit ? cols - c : kUnit));
    if (count == 0) continue;
    uint32_t w[4];
    load_q(q + r * ldq + c, count, aq, w);
    const uint32_t ex = e[r * lde + u / 2];
    float v[kUnit];
    if (DY) load_unit(dy + r * lddy + c, count, ady, v);
    value_unit<T, ACT, DY>(w, ex, v);
    store_unit(out + r * ldout + c, count, aout, v);
  }
}

// The same for rows that start anywhere; `aligned`: those of out start on 32 bytes.
template <class T, int ACT, bool DY>
__device__ __forceinline__ void unpack_pieces(const int8_t* q, int64_t ldq, const uint8_t* e, int64_t lde, const T* dy,
                                              int64_t lddy, T* out, int64_t ldout, int64_t rows, int64_t cols, bool aligned,
                                              int64_t warp, int64_t warps, float* buf) {
  const int lane = threadIdx.x % 32;
  each_piece(rows, cols, warp, warps, [&](const Piece& s, int64_t r, int64_t c) {
    const int first = lane * kUnit;  // this lane's unit in the piece
    const int64_t row = r + (first >> s.shift), col = c + (first & ((1 << s.shift) - 1));
    const bool there = s.there(first);
    uint32_t w[4];
    piece_q_in(s, q + r * ldq + c, ldq, buf, w);
    const uint32_t ex = there ? e[row * lde + col / kGroup] : 1u;
    float v[kUnit];
    if (DY) piece_in(s, dy + r * lddy + c, lddy, buf, v);
    value_unit<T, ACT, DY>(w, ex, v);
    if (aligned) {
      if (there) store_unit(out + row * ldout + col, (int)(cols - col < kUnit ? cols - col : kUnit), kWhole, v);
    } else {
      piece_out(s, out + r * ldout + c, ldout, buf, v);
    }
  });
}
template <class T, int ACT, bool DY>
__global__ void __launch_bounds__(kThreads, 4)
    unpack8_pieces_kernel(const int8_t* q, int64_t ldq, const uint8_t* e, int64_t lde, const T* dy, int64_t lddy, T* out,
                          int64_t ldout, int64_t rows, int64_t cols) {
  __shared__ __align__(16) float space[kThreads / 32][kPieceFloats];
  const int warp = threadIdx.x / 32;
  unpack_pieces<T, ACT, DY>(q, ldq, e, lde, dy, lddy, out, ldout, rows, cols, false,
                            (int64_t)blockIdx.x * (kThreads / 32) + warp, (int64_t)gridDim.x * (kThreads / 32), space[warp]);
}

// db[n] = sum over rows of dy (added to db where `add`). A CTA takes 64 columns and, with the other CTAs of its
// cluster, every row: a thread adds 8 columns of every 32nd row of the CTA's share in fp32, eight rows' loads at a time,
// shared memory joins the threads, the first CTA of the cluster adds the shares in order. One launch, no atomics.
constexpr int kSumCols = 64, kSumLanes = 8, kSumRows = kThreads / kSumLanes;

template <class T>
__device__ __forceinline__ void add8(const uint4* u, float (&s)[8]) {
#pragma unroll
  for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
    const uint32_t w[4] = {u[h].x, u[h].y, u[h].z, u[h].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) {
        s[2 * i] += __uint_as_float(w[i] << 16);
        s[2 * i + 1] += __uint_as_float(w[i] & 0xFFFF0000u);
      } else {
        s[4 * h + i] += __uint_as_float(w[i]);
      }
    }
  }
}

struct __align__(16) SumSpace {
  float part[kSumRows][kSumCols + 1];
  float total[kSumCols];
};

// total[c] = the sum of column 64 * block + c over the rows of a share: every 32 * shares-th block of 32 rows
template <class T>
__device__ __forceinline__ void column_sums(const T* dy, int64_t lddy, int64_t rows, int64_t cols, bool vec, int64_t block,
                                            int64_t share, int64_t shares, SumSpace& space) {
  float (*part)[kSumCols + 1] = space.part;
  float* total = space.total;
  const int lane = threadIdx.x % kSumLanes, row = threadIdx.x / kSumLanes;
  const int64_t c = (int64_t)block * kSumCols + lane * 8;
  const int count = (int)(cols - c < 0 ? 0 : (cols - c < 8 ? cols - c : 8));
  float s[8] = {};
  const int64_t step = (int64_t)kSumRows * shares;
  int64_t r = (int64_t)share * kSumRows + row;
  if (vec && count == 8) {
    // eight rows' loads in flight per thread: with one at a time the pass waits for memory (23 us instead of 6 at
    // 8224 x 1024 bf16)
    constexpr int kAhead = 8, kLoads = sizeof(T) / 2;
    for (; r + (kAhead - 1) * step < rows; r += kAhead * step) {
      uint4 u[kAhead][kLoads];
#pragma unroll
      for (int t = 0; t < kAhead; ++t)
#pragma unroll
        for (int h = 0; h < kLoads; ++h) u[t][h] = __ldg(reinterpret_cast<const uint4*>(dy + (r + t * step) * lddy + c) + h);
#pragma unroll
      for (int t = 0; t < kAhead; ++t) add8<T>(u[t], s);
    }
    for (; r < rows; r += step) {
      uint4 u[kLoads];
#pragma unroll
      for (int h = 0; h < kLoads; ++h) u[h] = __ldg(reinterpret_cast<const uint4*>(dy + r * lddy + c) + h);
      add8<T>(u, s);
    }
  } else {
#pragma unroll 4
    for (; r < rows; r += step)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < count) s[i] += to_float(dy[r * lddy + c + i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) part[row][lane * 8 + i] = s[i];
  __syncthreads();
  if (threadIdx.x < kSumCols) {
    float t = 0.0f;
    for (int i = 0; i < kSumRows; ++i) t += part[i][threadIdx.x];
    total[threadIdx.x] = t;
  }
}

template <class T>
__global__ void __launch_bounds__(kThreads)
    row_sums_kernel(const T* dy, int64_t lddy, T* db, int64_t rows, int64_t cols, bool vec, bool add) {
  __shared__ SumSpace space;
  column_sums(dy, lddy, rows, cols, vec, blockIdx.x, blockIdx.y, gridDim.y, space);
  const float* total = space.total;
  cluster_sync();
  const int64_t n = (int64_t)blockIdx.x * kSumCols + threadIdx.x;
  if (blockIdx.y == 0 && threadIdx.x < kSumCols && n < cols) {
    float t = 0.0f;
    for (unsigned i = 0; i < gridDim.y; ++i) t += cluster_load(&total[threadIdx.x], i);
    db[n] = from_float<T>(add ? to_float(db[n]) + t : t);
  }
  cluster_sync();  // the shares stay until they have been read
}

// What a bf16 product on the tensor cores needs done first, in one launch: rows copied to rows that start on 16 bytes, x^
// read back from 8 bits, and shares of dy's sums over its rows (which the product's kernel adds up). The CTAs are dealt
// out to the jobs; each walks its job's rows with threads side by side along a row. Copies run at 4 TB/s read and written (9216
// x 4292: 39 us); 8224 x 4096 values through quick GELU and the sums of 8224 x 1024 take 26 us for 118 MB.
template <int ACT>
__global__ void __launch_bounds__(kThreads) prepare_kernel(const Prepare a) {
  __shared__ union {
    SumSpace sums;
    float pieces[kThreads / 32][kPieceFloats];
  } shared_space;
  SumSpace& space = shared_space.sums;
  float (*pieces)[kPieceFloats] = shared_space.pieces;
  int cta = blockIdx.x;
  for (int k = 0; k < 2; ++k) {
    const Prepare::Copy& c = a.copy[k];
    if (cta < c.ctas) {
      const int64_t units = (c.cols + 7) / 8;
      const int wide = (int)(units < kThreads ? units : kThreads), high = kThreads / wide;
      const int tx = threadIdx.x % wide, ty = threadIdx.x / wide;
      const uint16_t* from = (const uint16_t*)c.from;
      uint16_t* to = (uint16_t*)c.to;
      if (ty < high)
        for (int64_t r = (int64_t)cta * high + ty; r < c.rows; r += (int64_t)c.ctas * high)
          for (int64_t u = tx; u < units; u += wide) {
            const int64_t at = 8 * u;
            uint32_t w[4] = {};
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (at + i < c.cols) w[i / 2] |= (uint32_t)from[r * c.ld + at + i] << (16 * (i % 2));
            *reinterpret_cast<uint4*>(to + r * c.ldto + at) = make_uint4(w[0], w[1], w[2], w[3]);
          }
      return;
    }
    cta -= c.ctas;
  }
  const Prepare::Unpack& p = a.unpack;
  if (cta < p.ctas) {
    __nv_bfloat16* to = (__nv_bfloat16*)p.to;
    if (!p.whole) {
      const int warp = threadIdx.x / 32;
      unpack_pieces<__nv_bfloat16, ACT, false>(p.q, p.ldq, p.e, p.lde, nullptr, 0, to, p.ldto, p.rows, p.cols, true,
                                               (int64_t)cta * (kThreads / 32) + warp, (int64_t)p.ctas * (kThreads / 32),
                                               pieces[warp]);
      return;
    }
    const int64_t units = (p.cols + kUnit - 1) / kUnit;
    const int wide = (int)(units < kThreads ? units : kThreads), high = kThreads / wide;
    const int tx = threadIdx.x % wide, ty = threadIdx.x / wide;
    if (ty < high)
      for (int64_t r = (int64_t)cta * high + ty; r < p.rows; r += (int64_t)p.ctas * high)
        for (int64_t u = tx; u < units; u += wide) {
          const int64_t c = u * kUnit;
          const int count = (int)(p.cols - c < kUnit ? p.cols - c : kUnit);
          uint32_t w[4];
          load_q(p.q + r * p.ldq + c, count, kWhole, w);
          float v[kUnit];
          value_unit<__nv_bfloat16, ACT, false>(w, p.e[r * p.lde + u / 2], v);
          store_unit(to + r * p.ldto + c, count, kWhole, v);
        }
    return;
  }
  cta -= p.ctas;
  const Prepare::Sums& m = a.sums;
  const int64_t block = cta / m.shares, share = cta % m.shares, n = block * kSumCols + threadIdx.x;
  column_sums((const __nv_bfloat16*)m.dy, m.lddy, m.rows, m.cols, m.vec, block, share, m.shares, space);
  if (threadIdx.x < kSumCols && n < m.cols) m.to[share * m.cols + n] = space.total[threadIdx.x];
}

bool can(const void* p, int64_t ld, size_t elem, size_t bytes) {
  return (uintptr_t)p % bytes == 0 && (uint64_t)ld * elem % bytes == 0;
}

struct Shape {
  dim3 grid, block;
};

// A block is as wide as a row has units, at most 256 threads; the grid has enough blocks for 64
// per SM (with 16 the last rows' blocks keep 3% of 8191 x 11008 waiting).
Shape shape_for(int64_t rows, int64_t units, int sms) {
  unsigned x = 2;
  while (x < kThreads && x < units) x *= 2;
  const unsigned y = kThreads / x;
  const int64_t bx = (units + x - 1) / x, by = (rows + y - 1) / y;
  const int64_t most = (int64_t)sms * 64;
  const int64_t gx = bx < most ? bx : most;
  int64_t gy = (most + gx - 1) / gx;
  gy = gy < by ? gy : by;
  return {dim3((unsigned)gx, (unsigned)(gy < 65535 ? gy : 65535)), dim3(x, y)};
}

Shape shape_of(int64_t rows, int64_t cols, int sms) { return shape_for(rows, (cols + kGroup - 1) / kGroup * 2, sms); }

// bytes: of a whole unit
Access access_of(const void* p, int64_t ld, size_t elem, size_t bytes) {
  return can(p, ld, elem, bytes) ? kWhole : can(p, ld, elem, elem == 1 ? 8 : 16) ? kHalves : kEach;
}

// CTAs of eight warps for a matrix in pieces, eight per SM at most
unsigned pieces_grid(int64_t rows, int64_t cols, int sms) {
  const int64_t ctas = (rows * ((cols + 31) / 32) * 32 / kPiece + kThreads / 32) / (kThreads / 32) + 1;
  return (unsigned)(ctas < 8 * sms ? ctas : 8 * sms);
}

template <class T, bool DY>
cudaError_t unpack_as(const int8_t* q, int64_t ldq, const uint8_t* e, int64_t lde, const void* dy, int64_t lddy,
                      void* out, int64_t ldout, int64_t rows, int64_t cols, int act, int sms, cudaStream_t s) {
  const Access aq = access_of(q, ldq, 1, 16), ady = DY ? access_of(dy, lddy, sizeof(T), 32) : kWhole,
               aout = access_of(out, ldout, sizeof(T), 32);
  if (aq == kEach || ady == kEach || aout == kEach) {
    const unsigned grid = pieces_grid(rows, cols, sms);
    SMAT_WITH_ACT(act, (unpack8_pieces_kernel<T, ACT, DY><<<grid, kThreads, 0, s>>>(
                           q, ldq, e, lde, (const T*)dy, lddy, (T*)out, ldout, rows, cols)))
  } else {
    const Shape h = shape_of(rows, cols, sms);
    SMAT_WITH_ACT(act, (unpack8_kernel<T, ACT, DY><<<h.grid, h.block, 0, s>>>(
                           q, ldq, e, lde, (const T*)dy, lddy, (T*)out, ldout, rows, cols, aq, ady, aout)))
  }
  return cudaGetLastError();
}

template <class T>
cudaError_t pack_as(const void* x, int64_t ldx, int8_t* q, int64_t ldq, uint8_t* e, int64_t lde, int64_t rows, int64_t cols,
                    int sms, cudaStream_t s) {
  const Access ax = access_of(x, ldx, sizeof(T), 32), aq = access_of(q, ldq, 1, 16);
  if (ax == kEach || aq == kEach) {
    pack8_pieces_kernel<T><<<pieces_grid(rows, cols, sms), kThreads, 0, s>>>((const T*)x, ldx, q, ldq, e, lde, rows, cols);
  } else {
    const Shape h = shape_of(rows, cols, sms);
    pack8_kernel<T><<<h.grid, h.block, 0, s>>>((const T*)x, ldx, q, ldq, e, lde, rows, cols, ax, aq);
  }
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_pack8(const void* x, int64_t ldx, int8_t* q, int64_t ldq, uint8_t* e, int64_t lde, int64_t rows,
                         int64_t cols, int dtype, int sms, cudaStream_t s) {
  return dtype == SMAT_BF16 ? pack_as<__nv_bfloat16>(x, ldx, q, ldq, e, lde, rows, cols, sms, s)
                            : pack_as<float>(x, ldx, q, ldq, e, lde, rows, cols, sms, s);
}

cudaError_t launch_unpack8(const int8_t* q, int64_t ldq, const uint8_t* e, int64_t lde, const void* dy, int64_t lddy,
                           void* out, int64_t ldout, int64_t rows, int64_t cols, int dtype, int act, int sms,
                           cudaStream_t s) {
  if (dtype == SMAT_BF16)
    return dy ? unpack_as<__nv_bfloat16, true>(q, ldq, e, lde, dy, lddy, out, ldout, rows, cols, act, sms, s)
              : unpack_as<__nv_bfloat16, false>(q, ldq, e, lde, dy, lddy, out, ldout, rows, cols, act, sms, s);
  return dy ? unpack_as<float, true>(q, ldq, e, lde, dy, lddy, out, ldout, rows, cols, act, sms, s)
            : unpack_as<float, false>(q, ldq, e, lde, dy, lddy, out, ldout, rows, cols, act, sms, s);
}

int sum_shares(int64_t rows) { return (int)(rows < 256 ? 1 : rows / 128 < 16 ? rows / 128 : 16); }

cudaError_t launch_prepare(Prepare a, int act, int sms, cudaStream_t s) {
  // CTAs by the threads that a job keeps busy with 16 bytes to write each, eight CTAs per SM for all copying at most
  auto ctas_of = [&](int64_t rows, int64_t units) {
    if (rows == 0 || units == 0) return 0;
    const int64_t wide = units < kThreads ? units : kThreads, high = kThreads / wide, n = (rows + high - 1) / high;
    return (int)(n < 8 * sms ? n : 8 * sms);
  };
  for (Prepare::Copy& c : a.copy) c.ctas = c.from ? ctas_of(c.rows, (c.cols + 7) / 8) : 0;
  a.unpack.ctas = a.unpack.q ? ctas_of(a.unpack.rows, (a.unpack.cols + kUnit - 1) / kUnit) : 0;
  a.unpack.whole = can(a.unpack.q, a.unpack.ldq, 1, 16);
  a.sums.vec = can(a.sums.dy, a.sums.lddy, 2, 16);
  const int sums = a.sums.to ? (int)((a.sums.cols + kSumCols - 1) / kSumCols) * a.sums.shares : 0;
  const int ctas = a.copy[0].ctas + a.copy[1].ctas + a.unpack.ctas + sums;
  if (ctas == 0) return cudaSuccess;
  SMAT_WITH_ACT(act, (prepare_kernel<ACT><<<ctas, kThreads, 0, s>>>(a)))
  return cudaGetLastError();
}

cudaError_t launch_row_sums(const void* dy, int64_t lddy, void* db, int64_t rows, int64_t cols, int dtype, bool add,
                            int sms, cudaStream_t s) {
  const unsigned gx = (unsigned)((cols + kSumCols - 1) / kSumCols);
  // as many CTAs per cluster as fill the chip with two each, at least 64 rows for each
  unsigned split = 1;
  while (split < 8 && gx * split < 2u * (unsigned)sms && (int64_t)split * 2 * 64 <= rows) split *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(gx, split);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim = {1, split, 1};
  cfg.attrs = at;
  cfg.numAttrs = 1;
  if (dtype == SMAT_BF16)
    return cudaLaunchKernelEx(&cfg, row_sums_kernel<__nv_bfloat16>, (const __nv_bfloat16*)dy, lddy, (__nv_bfloat16*)db,
                              rows, cols, can(dy, lddy, 2, 16), add);
  return cudaLaunchKernelEx(&cfg, row_sums_kernel<float>, (const float*)dy, lddy, (float*)db, rows, cols,
                            can(dy, lddy, 4, 16), add);
}

}  // namespace lin
}  // namespace smat
