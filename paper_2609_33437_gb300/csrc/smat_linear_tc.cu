// The linear layers' products of bf16 matrices on the tensor cores (tcgen05; smat_linear.h, Product).
//
// In every CTA one warp fetches 64-deep slices of both operands by TMA into a ring of 128-byte-swizzled buffers, one
// thread multiplies them into tensor memory (fp32), and further warps take finished sums out of it, 32 columns at a time,
// and finish them (bias, activation, 8-bit form, residual, slope, older gradient) while the next tile's sums are made in
// the other half of tensor memory.
//
// Wide products (pair_kernel): two CTAs on neighbouring SMs make a tile of 256 x `width` sums, each 128 of its rows. Each
// fetches its rows of one operand and half of the other, which the pair's multiplications read from both: 32 KB a slice
// and CTA for 256 columns, where a CTA by itself needs 48 KB and the copies bound it (8192 x 11008 x 4096: 484 us).
// `width` and the shares of the sum are chosen by an estimate of the time, see plan_pair. The tile's rows are rows i of
// the result. A thread holds 32 columns of a row, whole groups of the 8-bit form; 32 columns of a warp's 32 rows leave
// through shared memory by TMA, and what is added to them comes in that way; rows that do not start on 16 bytes are
// copied to and from there by the warp itself, a column per lane.
// Measured: 8192 x 11008 x 4096 with residual 405 us from cold (1,825 TFLOP/s, 94% of cuBLAS's burst, tensor pipe 86% busy)
// and 446 us call after call, when the power limit holds the clock down; the weight gradient of 4099 x 4096 x 4096 98 us
// (1,410 TFLOP/s): 256 tiles for 76 pairs are four rounds for 3.4, and L2 hands out 15 TB/s. 2056 x 1024 x 4096 with bias,
// activation and 8 bits 21 us with operands in L2: two rounds of 1.9, each ended by 10 MB of results at once, and some 5 us to
// start and end.
//
// Products of at most 128 rows (narrow_kernel): the tile's 128 rows are columns j and its 32, 64 or 128 columns are rows
// i, so that a wide weight fills the 128 and the few rows cost a narrow tile. A warp holds 32 neighbouring columns of a
// row, one per lane. With a weight that is not in L2 24 x 4096 x 11008 takes 20.4 us (4.4 TB/s) and one row of 4096 x 4096
// 12.3 us (2.7 TB/s), with one that is 13.6 and 9.3: the weight's bytes, and some 7 us to launch, start, join the shares and
// end. 4096 x 4096 in wide tiles takes longer up to 128 rows (weight not in L2: 33 rows 11.5 us and 16.9 wide, 128 rows 14.5
// and 17.9).
//
// Where the tiles are fewer than the SMs, the sum is cut among the CTAs (or pairs) of a cluster: each leaves its share of
// the sums, then every CTA adds up some of the columns in the cluster's order and finishes them. No atomics, the same
// result every time.
//
// Tensor memory's additions cut off instead of rounding: 1,024 terms come out 0.8e-6 of the sum too small in the mean, 4,096
// 1.8e-6. A rounding to bf16 hides that, the 8-bit form nearly (3 to 8 of 100,000 bytes are one step off, of exact fp32 sums 1
// to 2); adding slices in registers, as fp32 products do, would take warps the pair's products need.

#include "smat_linear.h"

#include <algorithm>

#include "smat_linear_tc.cuh"

namespace smat {
namespace lin {

__device__ int g_errors;  // bit 0: a wait inside a product ran out of time

namespace {

constexpr int kBytesA = kBM * kBK * 2;
// Narrow tiles are bound by the weight's bytes: two CTAs per SM, so that one's start and end lie beside the other's
// copies.
template <int BN>
struct Ring {
  static constexpr int kBytesB = BN * kBK * 2;
  static constexpr int kStages = BN == 32 ? 5 : BN == 64 ? 4 : 3;
  static constexpr int kStage = kBytesA + kBytesB;
  static constexpr int kBytes = kStages * kStage + 1024;
  static constexpr int kCtas = 2;  // per SM
};

constexpr int kPairRows = 2 * kBM, kPairStages = 5, kPairStage = 2 * kBytesA;
// Warps that finish a pair's sums, and slices on their way. Finishing waits for latencies: with 8 warps 2056 x 1024 x 4096
// saved in 8 bits takes 2.4 us longer, with 4 (and a sixth slice) 9 us, with 16 (96 registers) 1.6 us. With 4 slices
// 8192 x 11008 x 4096 takes 480 us instead of 446; with a sixth, and 8 warps to make room for it, the weight gradient of
// 4099 x 4096 x 4096 115 instead of 117, the first MLP layer 29.5 instead of 26.9.
constexpr int kPairEpi = 12;
constexpr int kPairThreads = 32 * (kPairEpi + 2);
// A finishing warp's own shared memory: 32 rows of 32 results (64 bytes, swizzled) and of 32 q (32 bytes, swizzled).
// Results in fp32 take 128 bytes a row and leave no q.
constexpr int kDeskRows = 32 * 64, kDeskQ = 32 * 32;
template <int MODE>
constexpr int kDesk = MODE == kGradInputSum ? 32 * 128 : kDeskRows + kDeskQ;
template <int MODE>
constexpr int kPairBytes = kPairStages * kPairStage + kPairEpi * kDesk<MODE> + 1024;
constexpr int kSums = 256;  // columns of tensor memory for one tile's sums

struct Args {
  Product p;
  int64_t tiles, tiles_r, tiles_c;  // along the tile's rows and columns
  int slices;                       // of 64 along the sum
  int share;                        // slices per CTA (or pair) of a cluster
  int width;                        // columns of a pair's tile
  float* parts;                     // the shares' sums, or NULL
  int* errors;                      // device error bits
  bool by_rows;                     // rows of out, residual and q start on 16 bytes: TMA copies them
  bool whole_ends;                  // and those that are written end on 16 bytes
  bool wide_bias;                   // bias on 16 bytes
};

using bf16 = __nv_bfloat16;

template <int MODE>
constexpr bool kWeightGrad = MODE == kGradWeight || MODE == kGradWeightRows;
// Whether the tile's columns run along the other operand's rows, the sum down them.
template <int MODE>
constexpr bool kSumDown = MODE == kGradInput || MODE == kGradInputSum || kWeightGrad<MODE>;

__device__ __forceinline__ void unpack_words(const uint32_t* w, int words, float* v) {
#pragma unroll
  for (int i = 0; i < words; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
// A warp's desk: where its 32 rows of 32 columns wait for TMA, and come from it. 16 bytes of a row lie at a place that
// changes with the row, as the copies' swizzle has it, so that 8 rows' accesses meet in no bank.
struct Desk {
  uint32_t rows, q, bar;  // shared addresses; a barrier for copies in
  uint32_t phase;
  __device__ __forceinline__ uint32_t row_at(int lane, int chunk) const {
    return rows + lane * 64 + ((chunk ^ (lane >> 1 & 3)) << 4);
  }
  __device__ __forceinline__ uint32_t q_at(int lane, int chunk) const {
    return q + lane * 32 + ((chunk ^ (lane >> 2 & 1)) << 4);
  }
};
__device__ __forceinline__ uint4 desk_load(uint32_t at) {
  uint4 u;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "r"(at) : "memory");
  return u;
}
__device__ __forceinline__ void desk_store(uint32_t at, const uint32_t* w) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
}

// The same by the warp's own accesses, for rows that TMA cannot copy: a column per lane, all 32 rows' loads in flight.
template <class T>
__device__ __forceinline__ uint32_t desk_place(const Desk& desk, int row, int column) {
  if (sizeof(T) == 2) return desk.row_at(row, column >> 3) + (column & 7) * 2;
  return desk.q_at(row, column >> 4) + (column & 15);
}
template <class T>  // uint16_t: rows of bf16; uint8_t: q
__device__ __forceinline__ void desk_fetch(const Desk& desk, const void* from, int64_t ld, int64_t i, int64_t j, int64_t I,
                                           int64_t J) {
  const int lane = threadIdx.x % 32;
  const int rows = j + lane < J ? (int)(I - i < 32 ? I - i : 32) : 0;
  const T* p = (const T*)from + i * ld + j + lane;
  T x[32];
#pragma unroll
  for (int t = 0; t < 32; ++t) x[t] = t < rows ? p[t * ld] : (T)0;
#pragma unroll
  for (int t = 0; t < 32; ++t) {
    if (sizeof(T) == 2)
      asm volatile("st.shared.u16 [%0], %1;" ::"r"(desk_place<T>(desk, t, lane)), "h"((uint16_t)x[t]) : "memory");
    else
      asm volatile("st.shared.u8 [%0], %1;" ::"r"(desk_place<T>(desk, t, lane)), "r"((uint32_t)x[t]) : "memory");
  }
}
template <class T>
__device__ __forceinline__ void desk_send(const Desk& desk, void* to, int64_t ld, int64_t i, int64_t j, int64_t I, int64_t J) {
  const int lane = threadIdx.x % 32;
  const int rows = j + lane < J ? (int)(I - i < 32 ? I - i : 32) : 0;
  T* p = (T*)to + i * ld + j + lane;
  T x[32];
#pragma unroll
  for (int t = 0; t < 32; ++t) {
    if (sizeof(T) == 2) {
      uint16_t u;
      asm volatile("ld.shared.u16 %0, [%1];" : "=h"(u) : "r"(desk_place<T>(desk, t, lane)) : "memory");
      x[t] = (T)u;
    } else {
      uint32_t u;
      asm volatile("ld.shared.u8 %0, [%1];" : "=r"(u) : "r"(desk_place<T>(desk, t, lane)) : "memory");
      x[t] = (T)u;
    }
  }
#pragma unroll
  for (int t = 0; t < 32; ++t)
    if (t < rows) p[t * ld] = x[t];
}

// Columns j .. j + 31 of rows i .. i + 31, a row per lane, out by TMA or by hand. A copy out leaves out rows outside the
// result, but writes whole 16 bytes at a row's end: one that ends elsewhere has its last columns sent by hand, so that what
// lies beside the result stays as it is. sums(v): their sums. False if a wait for what comes in has given up. rows: how many
// count (kLogitGrad).
template <int MODE, class Sums>
__device__ __forceinline__ bool finish_block(const Args& a, const CUtensorMap* map_out, const CUtensorMap* map_in,
                                            const CUtensorMap* map_q, int64_t i, int64_t j, int64_t rows, Desk& desk,
                                            volatile int* dead, Sums&& sums) {
  const Product& p = a.p;
  const int lane = threadIdx.x % 32;
  const bool there = i + lane < p.I;
  const bool slope = MODE == kGradInput && p.act != SMAT_ACT_NONE;
  const bool add = MODE == kForward ? p.residual != nullptr : kWeightGrad<MODE> && p.accumulate;
  const bool save = MODE == kForward && p.q;
  const void* from = MODE == kForward ? p.residual : p.out;  // what is added
  const int64_t ld_from = MODE == kForward ? p.ldr : p.ldo;
  const bool tma = a.by_rows && (a.whole_ends || j + 32 <= p.J);
  const bool copied = tma && (add || slope);
  if (tma) {
    if (lane == 0) {
      asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // the last block has left the desk
      if (copied) {
        bar_expect(desk.bar, add ? kDeskRows : kDeskQ);
        if (add)
          tma_load(desk.rows, map_in, (int)j, (int)i, desk.bar);
        else
          tma_load(desk.q, map_q, (int)j, (int)i, desk.bar);
      }
    }
  } else {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();  // the last block has been read
    if (add) desk_fetch<uint16_t>(desk, from, ld_from, i, j, p.I, p.J);
    if (slope) desk_fetch<uint8_t>(desk, p.q, p.ldq, i, j, p.I, p.J);
  }
  uint32_t e = 1;
  if (slope && there) e = p.e[(i + lane) * p.lde + j / kGroup];
  LossRow row = {0.0f, 0.0f, -1, 0.0f};
  bool counts = false;
  if (MODE == kLogitGrad) {
    counts = there && i + lane < rows;
    if (counts) row = p.loss_rows[i + lane];
  }
  __syncwarp();
  float v[32];
  sums(v);
  if (MODE == kLogitGrad) {
#pragma unroll
    for (int t = 0; t < 32; ++t) v[t] = exp2_fast(fmaf(v[t], kLog2e, -row.lse2)) * row.g;
    const int64_t at = row.target - p.first_col - j;  // of the target among the columns
    if (row.target >= 0 && at >= 0 && at < 32) {
#pragma unroll
      for (int t = 0; t < 32; ++t) v[t] = t == at ? row.own : v[t];
    }
    if (p.halves && i + lane >= rows / 2) {
#pragma unroll
      for (int t = 0; t < 32; ++t) v[t] -= to_float(from_float<bf16>(v[t]));
    }
    if (!counts) {  // rows behind the last one: they meet other rows in the weight's gradient
#pragma unroll
      for (int t = 0; t < 32; ++t) v[t] = 0.0f;
    }
  }
  if (MODE == kForward) {
    if (p.bias) {
      const bf16* b = (const bf16*)p.bias + j;
      if (a.wide_bias && j + 32 <= p.J) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const uint4 u = __ldg(reinterpret_cast<const uint4*>(b) + t);
          const uint32_t w[4] = {u.x, u.y, u.z, u.w};
          float f[8];
          unpack_words(w, 4, f);
#pragma unroll
          for (int s = 0; s < 8; ++s) v[8 * t + s] += f[s];
        }
      } else {
#pragma unroll
        for (int t = 0; t < 32; ++t)
          if (j + t < p.J) v[t] += to_float(b[t]);
      }
    }
    if (save) {
      float big[8];  // a tree: one chain of 32 would wait for each step
#pragma unroll
      for (int t = 0; t < 8; ++t) big[t] = larger(larger(v[t], v[t + 8]), larger(v[t + 16], v[t + 24]));
#pragma unroll
      for (int t = 4; t > 0; t /= 2)
#pragma unroll
        for (int u = 0; u < t; ++u) big[u] = larger(big[u], big[u + t]);
      const uint32_t ex = pack_exponent(__float_as_uint(big[0]));
      uint32_t w[8];
      pack_words<8>(v, ex, w);
      desk_store(desk.q_at(lane, 0), w);
      desk_store(desk.q_at(lane, 1), w + 4);
      if (there && j < p.J) p.e[(i + lane) * p.lde + j / kGroup] = (uint8_t)ex;
    }
    SMAT_WITH_ACT(p.act, _Pragma("unroll") for (int t = 0; t < 32; ++t) v[t] = act_value<ACT, bf16>(v[t]))
  }
  if (copied) {
    if (!bar_wait_warp(desk.bar, desk.phase & 1, dead, a.errors)) {
      bar_drain(desk.bar, desk.phase & 1);
      return false;
    }
    ++desk.phase;
  }
  if (slope) {
    uint32_t w[8];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint4 u = desk_load(desk.q_at(lane, t));
      w[4 * t] = u.x, w[4 * t + 1] = u.y, w[4 * t + 2] = u.z, w[4 * t + 3] = u.w;
    }
    float x[32];
    unpack_words8<8>(w, e, x);
    SMAT_WITH_ACT(p.act, _Pragma("unroll") for (int t = 0; t < 32; ++t) v[t] *= act_slope<ACT, bf16>(x[t]))
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const uint32_t at = desk.row_at(lane, c);
    if (add) {
      const uint4 u = desk_load(at);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
      float f[8];
      unpack_words(w, 4, f);
#pragma unroll
      for (int t = 0; t < 8; ++t) v[8 * c + t] += f[t];
    }
    uint32_t w[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[8 * c + 2 * t], v[8 * c + 2 * t + 1]);
      w[t] = *reinterpret_cast<const uint32_t*>(&b);
    }
    desk_store(at, w);
  }
  if (tma) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
      tma_store(map_out, desk.rows, (int)j, (int)i);
      if (save) tma_store(map_q, desk.q, (int)j, (int)i);
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
  } else {
    __syncwarp();
    desk_send<uint16_t>(desk, p.out, p.ldo, i, j, p.I, p.J);
    if (save) desk_send<uint8_t>(desk, p.q, p.ldq, i, j, p.I, p.J);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the next block may come and go by TMA
    __syncwarp();
  }
  return true;
}

// The same in fp32, out by TMA, stored or added to what is there: one addition for each element and launch, so the order of the
// launches is that of the additions.
template <class Sums>
__device__ __forceinline__ void finish_sum_block(const Args& a, const CUtensorMap* map_out, int64_t i, int64_t j, Desk& desk,
                                                 Sums&& sums) {
  const int lane = threadIdx.x % 32;
  float v[32];
  sums(v);
  if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // the last block has left the desk
  __syncwarp();
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    const uint32_t w[4] = {__float_as_uint(v[4 * c]), __float_as_uint(v[4 * c + 1]), __float_as_uint(v[4 * c + 2]),
                           __float_as_uint(v[4 * c + 3])};
    desk_store(desk.rows + lane * 128 + ((c ^ (lane & 7)) << 4), w);
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
  if (lane == 0) {
    if (a.p.accumulate)
      tma_add(map_out, desk.rows, (int)j, (int)i);
    else
      tma_store(map_out, desk.rows, (int)j, (int)i);
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  }
}

// Column j of rows i .. i + N - 1, one thread; the warp holds 32 neighbouring columns from a multiple of 32 on. What
// the rows read is asked for first, all of it.
template <int MODE, int N>
__device__ __forceinline__ void finish_column(const Args& a, int64_t i, int64_t j, float (&v)[N]) {
  static_assert(MODE != kGradWeight, "weight gradients are wide products");
  const Product& p = a.p;
  if (i >= p.I) return;
  const int rows = (int)(p.I - i < N ? p.I - i : N);
  const bool there = j < p.J;
  const int mine = there ? rows : 0;
  const int lane = threadIdx.x % 32;
  bf16* out = (bf16*)p.out + i * p.ldo + j;
  if (MODE == kForward) {
    float x[N];
    const float bias = p.bias && there ? to_float(((const bf16*)p.bias)[j]) : 0.0f;
    if (p.residual) {
      const bf16* r = (const bf16*)p.residual + i * p.ldr + j;
#pragma unroll
      for (int t = 0; t < N; ++t) x[t] = t < mine ? to_float(r[t * p.ldr]) : 0.0f;
    }
#pragma unroll
    for (int t = 0; t < N; ++t) v[t] += bias;
    if (p.q) {
#pragma unroll
      for (int t = 0; t < N; ++t) {
        const uint32_t top = __reduce_max_sync(0xFFFFFFFFu, there ? __float_as_uint(fabsf(v[t])) : 0u);
        const uint32_t ex = pack_exponent(top);
        if (t < mine) {
          p.q[(i + t) * p.ldq + j] = (int8_t)pack_one(v[t], ex);
          if (lane == 0) p.e[(i + t) * p.lde + j / kGroup] = (uint8_t)ex;
        }
      }
    }
    SMAT_WITH_ACT(p.act, _Pragma("unroll") for (int t = 0; t < N; ++t) v[t] = act_value<ACT, bf16>(v[t]))
    if (p.residual) {
#pragma unroll
      for (int t = 0; t < N; ++t) v[t] += x[t];
    }
  } else if (p.act != SMAT_ACT_NONE) {
    float x[N];
    const int8_t* q = p.q + i * p.ldq + j;
    const uint8_t* e = p.e + i * p.lde + j / kGroup;
    int qs[N];
    uint32_t es[N];
#pragma unroll
    for (int t = 0; t < N; ++t) {
      qs[t] = t < mine ? q[t * p.ldq] : 0;
      es[t] = t < mine ? e[t * p.lde] : 0;
    }
#pragma unroll
    for (int t = 0; t < N; ++t) x[t] = (float)qs[t] * unpack_scale(es[t]);
    SMAT_WITH_ACT(p.act, _Pragma("unroll") for (int t = 0; t < N; ++t) v[t] *= act_slope<ACT, bf16>(x[t]))
  }
#pragma unroll
  for (int t = 0; t < N; ++t)
    if (t < mine) out[t * p.ldo] = from_float<bf16>(v[t]);
}

// Blocks `first`, `first + step`, ... below `end` of 32 columns of a tile that begins at row row0 (this warp's 32) and
// column col0 of the result: `sums(c, v)` gives block c's sums. False: as finish_block, the blocks after it left out.
template <int MODE, class Sums>
__device__ __forceinline__ bool finish_blocks(const Args& a, const CUtensorMap* map_out, const CUtensorMap* map_in,
                                              const CUtensorMap* map_q, int64_t row0, int64_t col0, int first, int end,
                                              int step, int64_t rows, int64_t slab, Desk& desk, volatile int* dead,
                                              Sums&& sums) {
#pragma unroll 1
  for (int c = first; c < end; c += step) {
    const int64_t col = col0 + 32 * c;
    if (row0 < a.p.I && col < a.p.J) {
      if constexpr (MODE == kGradInputSum)
        finish_sum_block(a, map_out, slab + row0, col, desk, [&](float(&v)[32]) { sums(c, v); });
      else if (!finish_block<MODE>(a, map_out, map_in, map_q, row0, col, rows, desk, dead, [&](float(&v)[32]) { sums(c, v); }))
        return false;
    } else {
      float v[32];
      sums(c, v);
    }
  }
  return true;
}

template <int MODE, int BN>
__global__ void __launch_bounds__(kThreads, Ring<BN>::kCtas)
    narrow_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
              const __grid_constant__ Args a) {
  // the tile's rows come from W, its columns from x or dy
  constexpr bool A_MN = MODE == kGradInput, B_MN = false;
  constexpr int kStages = Ring<BN>::kStages, kStage = Ring<BN>::kStage;

  extern __shared__ uint8_t raw[];
  __shared__ __align__(8) uint64_t bars[2 * kStages + 5];
  __shared__ uint32_t tmem_at;
  __shared__ int dead_flag;
  uint8_t* ring = raw + ((1024 - (smem_address(raw) & 1023)) & 1023);
  volatile int* dead = &dead_flag;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t full = smem_address(bars), empty = full + 8 * kStages, sums_full = empty + 8 * kStages,
                 sums_empty = sums_full + 16, drained = sums_empty + 16;

  uint32_t shares, rank;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(shares));
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const int slice0 = (int)rank * a.share;
  const int slices = max(0, min(a.share, a.slices - slice0));
  const int64_t first_tile = blockIdx.x / shares, step = gridDim.x / shares;

  auto fetch = [&](uint32_t s, int r0, int c0, int k) {
    const int l = (slice0 + k) * kBK;
    const uint32_t bar = full + 8 * s, to_a = smem_address(ring) + s * kStage, to_b = to_a + kBytesA;
    bar_expect(bar, kStage);
    if (A_MN) {
#pragma unroll
      for (int b = 0; b < kBM / 64; ++b) tma_load(to_a + b * 8192, &map_a, r0 + 64 * b, l, bar);
    } else {
      tma_load(to_a, &map_a, l, r0, bar);
    }
    tma_load(to_b, &map_b, l, c0, bar);
  };
  const int ahead = first_tile < a.tiles ? min(slices, kStages) : 0;  // slices fetched before the CTA meets

  if (warp == kTmaWarp && lane == 0) {
    dead_flag = 0;
    for (int s = 0; s < kStages; ++s) {
      bar_init(full + 8 * s, 1);
      bar_init(empty + 8 * s, 1);
    }
    bar_init(drained, 1);
    for (int b = 0; b < 2; ++b) {
      bar_init(sums_full + 8 * b, 1);
      bar_init(sums_empty + 8 * b, kEpiWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    int64_t tr, tc;
    tile_place<16>(a.tiles_r, a.tiles_c, first_tile, tr, tc);
    for (int k = 0; k < ahead; ++k) fetch(k, (int)(tr * kBM), (int)(tc * BN), k);
  }
  __syncwarp();
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_address(&tmem_at)),
                 "r"(2 * BN)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    fence_before();
  }
  __syncthreads();
  fence_after();
  const uint32_t tmem = tmem_at;

  if (warp == kTmaWarp && lane == 0) {
    uint32_t n = (uint32_t)ahead;  // slices fetched so far
    bool ok = true;
    for (int64_t tile = first_tile; ok && tile < a.tiles; tile += step) {
      int64_t tr, tc;
      tile_place<16>(a.tiles_r, a.tiles_c, tile, tr, tc);
      for (int k = tile == first_tile ? ahead : 0; k < slices; ++k, ++n) {
        const uint32_t s = n % kStages;
        ok = bar_wait(empty + 8 * s, (n / kStages + 1) & 1, dead, a.errors);
        if (!ok) break;
        fetch(s, (int)(tr * kBM), (int)(tc * BN), k);
      }
    }
    if (!ok)  // copies in flight land before the CTA ends
      for (uint32_t s = 0; s < kStages && s < n; ++s) {
        const uint32_t last = n - 1 - s;
        bar_drain(full + 8 * (last % kStages), last / kStages & 1);
      }
  } else if (warp == kMmaWarp && lane == 0) {
    constexpr uint32_t kInst = kInstruction<A_MN, B_MN, BN>;
    uint32_t n = 0, made = 0;
    bool ok = true;
    for (int64_t tile = first_tile; ok && tile < a.tiles; tile += step, ++made) {
      const uint32_t half = made & 1, sums = tmem + half * BN;
      ok = bar_wait(sums_empty + 8 * half, (made / 2 + 1) & 1, dead, a.errors);
      if (!ok) break;
      fence_after();
      for (int k = 0; k < slices; ++k, ++n) {
        const uint32_t s = n % kStages;
        ok = bar_wait(full + 8 * s, n / kStages & 1, dead, a.errors);
        if (!ok) break;
        fence_after();
        const uint32_t at_a = smem_address(ring) + s * kStage;
        const uint64_t da = descriptor<A_MN>(at_a), db = descriptor<B_MN>(at_a + kBytesA);
#pragma unroll
        for (int t = 0; t < kBK / 16; ++t)
          mma(sums, da + t * kStep16<A_MN>, db + t * kStep16<B_MN>, kInst, k > 0 || t > 0);
        mma_commit(empty + 8 * s);
      }
      if (ok) mma_commit(sums_full + 8 * half);
    }
    if (!ok) {  // products in flight end before the CTA does
      mma_commit(drained);
      bar_drain(drained, 0);
    }
  } else if (warp < kEpiWarps) {
    const int quarter = warp % 4;  // the 32 rows of tensor memory that this warp may read
    // this thread's row of the CTA's share of the sums. The ring is free by then: every product that read it is done
    float* part = (a.parts ? a.parts + ((size_t)first_tile * shares + rank) * BN * kBM : reinterpret_cast<float*>(ring)) +
                  32 * quarter + lane;
    uint32_t made = 0;
    for (int64_t tile = first_tile; tile < a.tiles; tile += step, ++made) {
      int64_t tr, tc;
      tile_place<16>(a.tiles_r, a.tiles_c, tile, tr, tc);
      const int64_t r0 = tr * kBM + 32 * quarter, c0 = tc * BN;
      const uint32_t half = made & 1, sums = tmem + half * BN + ((uint32_t)(32 * quarter) << 16);
      if (!bar_wait_warp(sums_full + 8 * half, made / 2 & 1, dead, a.errors, kWaitNs + slices * kSliceNs)) break;
      fence_after();
      auto release = [&] {  // this warp has what it needs of these sums
        fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(sums_empty + 8 * half);
      };
      const int blocks = (int)((min((int64_t)BN, a.p.I - c0) + 7) / 8);  // of 8 columns of the tile, rows of the result
      for (int c = warp / 4; c < blocks; c += kEpiWarps / 4) {
        float v[8];
        if (slices > 0) {
          take8(sums + 8 * c, v);
        } else {
#pragma unroll
          for (int t = 0; t < 8; ++t) v[t] = 0.0f;
        }
        if (shares == 1) {
          if (r0 < a.p.J) finish_column<MODE, 8>(a, c0 + 8 * c, r0 + lane, v);
        } else {
          put_part(part + 8 * c * kBM, v);
        }
      }
      release();
    }
  }
  __syncwarp();
  if (shares > 1) {
    // one tile per cluster: its CTAs add up and finish blocks of its columns in turn
    __syncthreads();
    cluster_sync();
    if (warp < kEpiWarps && !__any_sync(0xFFFFFFFFu, *dead)) {
      int64_t tr, tc;
      tile_place<16>(a.tiles_r, a.tiles_c, first_tile, tr, tc);
      const int quarter = warp % 4;
      const int64_t r0 = tr * kBM + 32 * quarter, c0 = tc * BN;
      const float* part = (a.parts ? a.parts + (size_t)first_tile * shares * BN * kBM : reinterpret_cast<float*>(ring)) +
                          32 * quarter + lane;
      const int first = (int)rank + (int)shares * (warp / 4), turns = (int)shares * (kEpiWarps / 4);
      const int cols = (int)min((int64_t)BN, a.p.I - c0);
      for (int c = first; 8 * c < cols && r0 < a.p.J; c += turns) {
        float v[8];
        if (a.parts)
          add_parts(shares, v, [&](uint32_t s, int t) { return __ldcg(part + ((size_t)s * BN + 8 * c + t) * kBM); });
        else
          add_parts(shares, v, [&](uint32_t s, int t) {
            return 8 * c + t < cols ? cluster_load(part + (8 * c + t) * kBM, s) : 0.0f;
          });
        finish_column<MODE, 8>(a, c0 + 8 * c, r0 + lane, v);
      }
    }
    cluster_sync();
  }
  fence_before();
  __syncthreads();
  if (warp == kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * BN));
}

// A pair's tile: see the head of this file. The pair's first CTA ("leader") multiplies for both.
template <int MODE>
__global__ void __launch_bounds__(kPairThreads, 1)
    pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                const __grid_constant__ CUtensorMap map_out, const __grid_constant__ CUtensorMap map_in,
                const __grid_constant__ CUtensorMap map_q, const __grid_constant__ Args a) {
  constexpr bool A_MN = kWeightGrad<MODE>, B_MN = kSumDown<MODE>;
  constexpr int kStages = kPairStages, kStage = kPairStage;

  extern __shared__ uint8_t raw[];
  __shared__ __align__(8) uint64_t bars[2 * kStages + 5 + kPairEpi];
  __shared__ uint32_t tmem_at;
  __shared__ int dead_flag;
  uint8_t* ring = raw + ((1024 - (smem_address(raw) & 1023)) & 1023);
  volatile int* dead = &dead_flag;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t full = smem_address(bars), empty = full + 8 * kStages, sums_full = empty + 8 * kStages,
                 sums_empty = sums_full + 16, drained = sums_empty + 16;
  uint8_t* own = ring + kStages * kStage + warp * kDesk<MODE>;  // a finishing warp's desk
  Desk desk = {smem_address(own), smem_address(own) + kDeskRows, drained + 8 + 8 * (uint32_t)warp, 0};

  uint32_t ctas, rank;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const uint32_t shares = ctas / 2, share = rank / 2, member = rank & 1, leader = rank & ~1u;
  // rows that only the device counts: tiles and slices behind the last one are left out
  int64_t tiles_r = a.tiles_r, tiles = a.tiles, rows = a.p.I;
  int slices_there = a.slices;
  if (MODE == kGradWeightRows) slices_there = min(slices_there, (*a.p.count + kBK - 1) / kBK);
  if (MODE == kLogitGrad || MODE == kGradInputSum) {
    rows = min(rows, (int64_t)*a.p.count);
    tiles_r = (rows + kPairRows - 1) / kPairRows;
    tiles = tiles_r * a.tiles_c;
  }
  // kGradInputSum: a tile comes once for every part of its sum
  int64_t units = tiles;
  int slice0 = (int)share * a.share;
  int slices = max(0, min(a.share, slices_there - slice0));
  if (MODE == kGradInputSum) units *= max(1, a.p.splits);
  auto part_of = [&](int64_t unit, int& first_slice, int& count) {  // the unit's tile, and its slices
    if (MODE != kGradInputSum) return unit;
    const int64_t split = unit / tiles;
    first_slice = (int)(share + split) * a.share;
    count = max(0, min(a.share, slices_there - first_slice));
    return unit - split * tiles;
  };
  const int64_t first_tile = blockIdx.x / ctas, step = gridDim.x / ctas;
  const int half_width = a.width / 2;

  if (warp == kPairEpi && lane == 0) {
    dead_flag = 0;
    for (int s = 0; s < kStages; ++s) {
      bar_init(full + 8 * s, 1);
      bar_init(empty + 8 * s, 1);
    }
    bar_init(drained, 1);
    for (int w = 0; w < kPairEpi; ++w) bar_init(drained + 8 + 8 * w, 1);
    for (int b = 0; b < 2; ++b) {
      bar_init(sums_full + 8 * b, 1);
      bar_init(sums_empty + 8 * b, 2 * kPairEpi);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  if (warp == kPairEpi + 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_address(&tmem_at)),
                 "r"(2 * kSums)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    fence_before();
  }
  __syncthreads();
  cluster_sync();  // the partner's barriers are there
  fence_after();
  const uint32_t tmem = tmem_at;

  if (warp == kPairEpi && lane == 0) {
    const int blocks_b = B_MN ? (half_width + 63) / 64 : 1;  // copies of this CTA's half of the other operand
    const uint32_t bytes = kBytesA + (B_MN ? blocks_b * 8192 : half_width * kBK * 2);
    const uint32_t full_there = cluster_address_of(full, leader);
    uint32_t n = 0;  // slices fetched so far
    bool ok = true;
    for (int64_t unit = first_tile; ok && unit < units; unit += step) {
      const int64_t tile = part_of(unit, slice0, slices);
      int64_t tr, tc;
      tile_place<8>(tiles_r, a.tiles_c, tile, tr, tc);
      const int r0 = (int)(tr * kPairRows) + (int)member * kBM, c0 = (int)(tc * a.width) + (int)member * half_width;
      for (int k = 0; k < slices; ++k, ++n) {
        const uint32_t s = n % kStages;
        ok = bar_wait(empty + 8 * s, (n / kStages + 1) & 1, dead, a.errors);
        if (!ok) break;
        const int l = (slice0 + k) * kBK;
        const uint32_t bar = full_there + 8 * s, to_a = smem_address(ring) + s * kStage, to_b = to_a + kBytesA;
        if (member == 0) bar_expect(full + 8 * s, 2 * bytes);
        if (A_MN) {
          tma_load_pair(to_a, &map_a, r0, l, bar);
          tma_load_pair(to_a + 8192, &map_a, r0 + 64, l, bar);
        } else {
          tma_load_pair(to_a, &map_a, l, r0, bar);
        }
        if (B_MN) {
          for (int b = 0; b < blocks_b; ++b) tma_load_pair(to_b + b * 8192, &map_b, c0 + 64 * b, l, bar);
        } else {
          tma_load_pair(to_b, &map_b, l, c0, bar);
        }
      }
    }
    // both CTAs' copies in flight land before either ends (they meet below)
    if (!ok && member == 0)
      for (uint32_t s = 0; s < kStages && s < n; ++s) {
        const uint32_t last = n - 1 - s;
        bar_drain(full + 8 * (last % kStages), last / kStages & 1);
      }
    else if (!ok)  // they signal the other CTA's barriers, which may have given up on them
      drain_pause();
  } else if (warp == kPairEpi + 1 && lane == 0 && member == 0) {
    const uint32_t inst = kInstruction<A_MN, B_MN, 0, kPairRows> | (uint32_t)(a.width >> 3) << 17;
    const uint16_t both = (uint16_t)(3u << rank);
    uint32_t n = 0, made = 0;
    bool ok = true;
    for (int64_t unit = first_tile; ok && unit < units; unit += step, ++made) {
      part_of(unit, slice0, slices);
      const uint32_t half = made & 1, sums = tmem + half * kSums;
      ok = bar_wait(sums_empty + 8 * half, (made / 2 + 1) & 1, dead, a.errors);
      if (!ok) break;
      fence_after();
      for (int k = 0; k < slices; ++k, ++n) {
        const uint32_t s = n % kStages;
        ok = bar_wait(full + 8 * s, n / kStages & 1, dead, a.errors);
        if (!ok) break;
        fence_after();
        const uint32_t at_a = smem_address(ring) + s * kStage;
        const uint64_t da = descriptor<A_MN>(at_a), db = descriptor<B_MN>(at_a + kBytesA);
#pragma unroll
        for (int t = 0; t < kBK / 16; ++t)
          mma_pair(sums, da + t * kStep16<A_MN>, db + t * kStep16<B_MN>, inst, k > 0 || t > 0);
        mma_commit_pair(empty + 8 * s, both);
      }
      if (ok) mma_commit_pair(sums_full + 8 * half, both);
    }
    if (!ok) {  // products in flight end before the CTAs do
      mma_commit_pair(drained, (uint16_t)(1u << rank));
      bar_drain(drained, 0);
    }
  } else if (warp < kPairEpi) {
    if (MODE == kGradWeight && a.p.db) {  // db, while the first sums are made
      bf16* db = (bf16*)a.p.db;
      for (int64_t n = (int64_t)blockIdx.x * (32 * kPairEpi) + threadIdx.x; n < a.p.I; n += (int64_t)gridDim.x * (32 * kPairEpi)) {
        float t = 0.0f;
#pragma unroll 4
        for (int s = 0; s < a.p.sum_shares; ++s) t += a.p.sums[s * a.p.I + n];
        db[n] = from_float<bf16>(a.p.add_db ? to_float(db[n]) + t : t);
      }
    }
    const int quarter = warp % 4;  // the 32 rows of tensor memory that this warp may read
    const uint32_t sums_empty_there = cluster_address_of(sums_empty, leader);
    // this warp's blocks of 32 columns
    constexpr int kBeside = kPairEpi / 4;  // warps that share 32 rows
    const int blocks = a.width / 32, first = warp / 4 * blocks / kBeside, end = (warp / 4 + 1) * blocks / kBeside;
    uint32_t made = 0;
    for (int64_t unit = first_tile; unit < units; unit += step, ++made) {
      const int64_t tile = part_of(unit, slice0, slices);
      int64_t tr, tc;
      tile_place<8>(tiles_r, a.tiles_c, tile, tr, tc);
      const int64_t r0 = tr * kPairRows + (int)member * kBM + 32 * quarter, c0 = tc * a.width;
      const int64_t slab = MODE == kGradInputSum ? unit / tiles * a.p.slab : 0;  // where this part's rows begin
      const uint32_t half = made & 1, sums = tmem + half * kSums + ((uint32_t)(32 * quarter) << 16);
      if (!bar_wait_warp(sums_full + 8 * half, made / 2 & 1, dead, a.errors, kWaitNs + slices * kSliceNs)) break;
      fence_after();
      auto release = [&] {  // this warp has what it needs of these sums
        fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive_there(sums_empty_there + 8 * half);
      };
      auto take = [&](int c, float(&v)[32]) {
        if (slices > 0) {
          take32(sums + 32 * c, v);
        } else {
#pragma unroll
          for (int t = 0; t < 32; ++t) v[t] = 0.0f;
        }
        if (c + 1 == end) release();
      };
      if (first == end) release();  // none of a narrow tile's columns
      if (shares == 1) {
        if (!finish_blocks<MODE>(a, &map_out, &map_in, &map_q, r0, c0, first, end, 1, rows, slab, desk, dead, take)) break;
      } else {
        float* part = a.parts + ((size_t)first_tile * ctas + rank) * a.width * kBM + 32 * quarter + lane;
        for (int c = first; c < end; ++c) {
          float v[32];
          take(c, v);
          if (c0 + 32 * c < a.p.J && r0 < a.p.I) put_part(part + 32 * c * kBM, v);
        }
      }
    }
  }
  __syncwarp();
  if (shares > 1) {
    // one tile per cluster: its CTAs add up and finish blocks of their rows' columns in turn
    __syncthreads();
    cluster_sync();
    if (warp < kPairEpi && first_tile < tiles && !__any_sync(0xFFFFFFFFu, *dead)) {
      int64_t tr, tc;
      tile_place<8>(tiles_r, a.tiles_c, first_tile, tr, tc);
      const int quarter = warp % 4;
      const int64_t r0 = tr * kPairRows + (int)member * kBM + 32 * quarter, c0 = tc * a.width;
      const float* part = a.parts + ((size_t)first_tile * ctas + member) * a.width * kBM + 32 * quarter + lane;
      const size_t apart = (size_t)2 * a.width * kBM;
      const int blocks = r0 < a.p.I ? (int)((min((int64_t)a.width, a.p.J - c0) + 31) / 32) : 0;
      finish_blocks<MODE>(a, &map_out, &map_in, &map_q, r0, c0, (int)share + (int)shares * (warp / 4), blocks,
                          (int)shares * (kPairEpi / 4), rows, 0, desk, dead, [&](int c, float(&v)[32]) {
                           add_parts(shares, v, [&](uint32_t s, int t) { return __ldcg(part + s * apart + (32 * c + t) * kBM); });
                         });
    }
  }
  if (warp < kPairEpi && lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // the desk has been read
  __syncwarp();
  fence_before();
  __syncthreads();
  cluster_meet();  // the partner's multiplications read this CTA's shared memory, and its arrivals write it
  if (warp == kPairEpi + 1)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * kSums));
}

// One product's launch: tiles, shares of the sum, workspace.
struct Plan {
  int64_t tiles_r, tiles_c, ctas;
  int slices, share, shares, width;
  size_t bytes;  // of the shares' sums
};

template <int MODE, int BN>
cudaError_t plan_narrow(const Product& p, int sms, Plan* plan) {
  static std::atomic<uint64_t> allowed;
  const cudaError_t e = allow_shared(narrow_kernel<MODE, BN>, Ring<BN>::kBytes, allowed);
  if (e != cudaSuccess) return e;
  Plan g = {};
  g.width = BN;
  g.tiles_r = (p.J + kBM - 1) / kBM;
  g.tiles_c = (p.I + BN - 1) / BN;
  g.slices = (int)((p.L + kBK - 1) / kBK);
  const int64_t tiles = g.tiles_r * g.tiles_c, room = (int64_t)Ring<BN>::kCtas * sms;
  // Shares of the sum as long as all CTAs have room at once, three slices in each at least.
  int shares = 8;
  while (shares > 1 && (tiles * shares > room || g.slices < 3 * shares)) --shares;
  g.share = (g.slices + shares - 1) / shares;
  g.shares = shares > 1 ? (g.slices + g.share - 1) / g.share : 1;
  g.ctas = g.shares > 1 ? tiles * g.shares : (tiles < room ? tiles : room);
  if (g.shares > 1 && p.I > 8) g.bytes = (size_t)tiles * g.shares * BN * kBM * sizeof(float);
  *plan = g;
  return cudaSuccess;
}

// Width and shares of a pair's tile: the least estimate of the time in cycles. A slice takes the longer of its
// multiplications (2 per column) and its copies (16 KB and 64 bytes per column at 64 bytes a cycle); a tile's columns take
// about 16 each to finish, beside the next tile's products, and at the end by themselves; shares are written and read through
// L2. All clusters of a shared sum run at once. The estimate orders choices, it is no time: a slice of 256 columns was 0.41 us
// in 2056 x 4096 with k from 1024 to 4096, where 512 cycles are 0.25. Of the 28 choices it took the fastest, or one within 1%,
// in each of six forward shapes from 257 x 1024 x 4096 to 4096 x 592 x 1024, and among 15 others (five input gradients, three
// of them with slopes, from 515 x 4864 x 896 to 8192 x 11008 x 4096; seven weight gradients from 300 x 512 x 512 to 8224 x 4096 x
// 1024; three forward ones with bias, activation and 8 bits) one that no other beat by more than the 2 us that were resolved.
template <int MODE>
cudaError_t plan_pair(const Product& p, Plan* plan) {
  static std::atomic<uint64_t> allowed;
  static std::atomic<int> clusters[64][9];
  auto* f = pair_kernel<MODE>;
  const cudaError_t e = allow_shared(f, kPairBytes<MODE>, allowed);
  if (e != cudaSuccess) return e;
  Plan best = {};
  double least = 0;
  const int slices = (int)((p.L + kBK - 1) / kBK);
  const int64_t tiles_r = (p.I + kPairRows - 1) / kPairRows;
  if (MODE == kGradInputSum && p.splits > 1) {  // a pair for each part of each tile
    const int64_t at_once = clusters_at_once(f, 2, kPairThreads, kPairBytes<MODE>, clusters);
    const int64_t tiles_c = (p.J + 255) / 256, units = tiles_r * tiles_c * p.splits;
    *plan = {tiles_r, tiles_c, 2 * std::min(units, at_once), slices, (slices + p.splits - 1) / p.splits, 1, 256, 0};
    return cudaSuccess;
  }
  for (int width = 256; width >= 64; width -= 32) {
    const int64_t tiles_c = (p.J + width - 1) / width, tiles = tiles_r * tiles_c;
    for (int shares = 1; shares <= 4; ++shares) {
      const int64_t at_once = clusters_at_once(f, 2 * shares, kPairThreads, kPairBytes<MODE>, clusters);
      if (shares > 1 && (tiles > at_once || slices < 3 * shares)) break;
      const int share = (slices + shares - 1) / shares;
      const double rounds = (double)((tiles + at_once - 1) / at_once);
      const double slice = 2.0 * width > 256.0 + width ? 2.0 * width : 256.0 + width;
      const double products = share * slice, finish = 16.0 * width;
      const double time = rounds * (products > finish ? products : finish) + finish / shares + 400.0 * rounds +
                          (shares > 1 ? 3000.0 + 14.0 * width : 0.0);
      if (best.width == 0 || time < least) {
        least = time;
        best.width = width;
        best.tiles_r = tiles_r, best.tiles_c = tiles_c;
        best.slices = slices, best.share = share;
        best.shares = shares > 1 ? (slices + share - 1) / share : 1;
        best.ctas = 2 * best.shares * (best.shares > 1 ? tiles : (tiles < at_once ? tiles : at_once));
        best.bytes = best.shares > 1 ? (size_t)tiles * 2 * best.shares * width * kBM * sizeof(float) : 0;
      }
    }
  }
  *plan = best;
  return cudaSuccess;
}

// What both kernels take.
cudaError_t fill_args(const Product& p, const Plan& g, void* workspace, Args* args) {
  Args a = {};
  a.p = p;
  a.tiles_r = g.tiles_r, a.tiles_c = g.tiles_c, a.tiles = g.tiles_r * g.tiles_c;
  a.slices = g.slices, a.share = g.share, a.width = g.width;
  const cudaError_t e = error_word(&a.errors);
  a.parts = g.bytes ? (float*)workspace : nullptr;
  auto rows_on = [](const void* q, int64_t ld, int elem, int bytes) {
    return (uintptr_t)q % bytes == 0 && (uint64_t)ld * elem % bytes == 0;
  };
  a.by_rows = rows_on(p.out, p.ldo, p.mode == kGradInputSum ? 4 : 2, 16) && (!p.residual || rows_on(p.residual, p.ldr, 2, 16)) &&
              (!p.q || rows_on(p.q, p.ldq, 1, 16));
  a.whole_ends = p.J % 8 == 0 && (p.mode != kForward || !p.q || p.J % 16 == 0);
  a.wide_bias = (uintptr_t)p.bias % 16 == 0;
  *args = a;
  return e;
}

template <int MODE, int BN>
cudaError_t launch_narrow(const Product& p, int sms, void* workspace, cudaStream_t s) {
  Plan g;
  Args a;
  cudaError_t e = plan_narrow<MODE, BN>(p, sms, &g);
  if (e == cudaSuccess) e = fill_args(p, g, workspace, &a);
  if (e != cudaSuccess) return e;
  CUtensorMap ma = {}, mb = {};  // not read where the sum is over nothing
  if (p.L > 0 &&
      !((MODE == kGradInput ? encode(&ma, p.b, p.J, p.L, p.ldb, kBK) : encode(&ma, p.b, p.L, p.J, p.ldb, kBM)) &&
        encode(&mb, p.a, p.L, p.I, p.lda, BN)))
    return cudaErrorNotSupported;
  return launch(narrow_kernel<MODE, BN>, g.ctas, g.shares, kThreads, Ring<BN>::kBytes, s, ma, mb, a);
}

template <int MODE>
cudaError_t launch_pair(const Product& p, void* workspace, cudaStream_t s) {
  constexpr bool A_MN = kWeightGrad<MODE>, B_MN = kSumDown<MODE>;
  Plan g;
  Args a;
  cudaError_t e = plan_pair<MODE>(p, &g);
  if (e == cudaSuccess) e = fill_args(p, g, workspace, &a);
  if (e != cudaSuccess) return e;
  CUtensorMap ma = {}, mb = {};
  if (p.L > 0 && !((A_MN ? encode(&ma, p.a, p.I, p.L, p.lda, kBK) : encode(&ma, p.a, p.L, p.I, p.lda, kBM)) &&
                   (B_MN ? encode(&mb, p.b, p.J, p.L, p.ldb, kBK) : encode(&mb, p.b, p.L, p.J, p.ldb, g.width / 2))))
    return cudaErrorNotSupported;
  // the results' rows, what is added to them, and q: those that are copied by TMA
  CUtensorMap mo = {}, mi = {}, mq = {};
  const void* in = MODE == kForward ? p.residual : kWeightGrad<MODE> && p.accumulate ? p.out : nullptr;
  if (MODE == kGradInputSum) {
    const int64_t rows = p.splits > 1 ? p.splits * p.slab : p.I;
    if (!a.by_rows || !encode(&mo, p.out, p.J, rows, p.ldo, 32, 32, 4)) return cudaErrorNotSupported;
  } else if (a.by_rows && !(encode(&mo, p.out, p.J, p.I, p.ldo, 32, 32) &&
                     (!in || encode(&mi, in, p.J, p.I, MODE == kForward ? p.ldr : p.ldo, 32, 32)) &&
                     (!p.q || encode(&mq, p.q, p.J, p.I, p.ldq, 32, 32, 1))))
    return cudaErrorNotSupported;
  return launch(pair_kernel<MODE>, g.ctas, 2 * g.shares, kPairThreads, kPairBytes<MODE>, s, ma, mb, mo, mi, mq, a);
}

// A product's kernel: go.narrow<MODE, BN>() or go.pair<MODE>(). Up to 128 rows the weight's columns take the tile's rows.
template <int MODE, class Go>
cudaError_t choose_mode(const Product& p, Go&& go) {
  if constexpr (MODE == kForward || MODE == kGradInput) {
    if (p.I <= 32) return go.template narrow<MODE, 32>();
    if (p.I <= 64) return go.template narrow<MODE, 64>();
    if (p.I <= 128) return go.template narrow<MODE, 128>();
  }
  return go.template pair<MODE>();
}
template <class Go>
cudaError_t choose(const Product& p, Go&& go) {
  switch (p.mode) {
    case kForward: return choose_mode<kForward>(p, go);
    case kGradInput: return choose_mode<kGradInput>(p, go);
    case kLogitGrad: return choose_mode<kLogitGrad>(p, go);
    case kGradInputSum: return choose_mode<kGradInputSum>(p, go);
    case kGradWeightRows: return choose_mode<kGradWeightRows>(p, go);
    default: return choose_mode<kGradWeight>(p, go);
  }
}

struct Launch {
  const Product& p;
  int sms;
  void* workspace;
  cudaStream_t s;
  template <int MODE, int BN>
  cudaError_t narrow() const {
    return launch_narrow<MODE, BN>(p, sms, workspace, s);
  }
  template <int MODE>
  cudaError_t pair() const {
    return launch_pair<MODE>(p, workspace, s);
  }
};
struct Size {
  const Product& p;
  int sms;
  size_t* bytes;
  cudaError_t take(cudaError_t e, const Plan& g) const {
    *bytes = e == cudaSuccess ? g.bytes : 0;
    return e;
  }
  template <int MODE, int BN>
  cudaError_t narrow() const {
    Plan g = {};
    return take(plan_narrow<MODE, BN>(p, sms, &g), g);
  }
  template <int MODE>
  cudaError_t pair() const {
    Plan g = {};
    return take(plan_pair<MODE>(p, &g), g);
  }
};

}  // namespace

cudaError_t tc_workspace(const Product& p, int sms, size_t* bytes) { return choose(p, Size{p, sms, bytes}); }
cudaError_t launch_tc(const Product& p, int sms, void* workspace, cudaStream_t s) {
  return choose(p, Launch{p, sms, workspace, s});
}

// Few rows have few tiles and a sum as long as the vocabulary. A cluster's shares, four at most, left most of the GPU idle: 100 x 256
// back from 100000 words took 120 us with 32 CTAs, and 26 in 32 parts with 64; 24 x 4096 from 32000 63 and 51, 300 x 1024 from 8000
// 20 and 14, 8 x 512 from 5000 15 and 9.5. The parts are added in one order by whoever reads them. At least four slices each, one
// round of pairs, and no more than 32 parts to be read again; 1 where the tiles fill the GPU by themselves.
cudaError_t grad_input_splits(const Product& p, int* splits) {
  static std::atomic<uint64_t> allowed;
  static std::atomic<int> clusters[64][9];
  auto* f = pair_kernel<kGradInputSum>;
  *splits = 1;
  const cudaError_t e = allow_shared(f, kPairBytes<kGradInputSum>, allowed);
  if (e != cudaSuccess || p.I == 0 || p.J == 0) return e;
  const int64_t at_once = clusters_at_once(f, 2, kPairThreads, kPairBytes<kGradInputSum>, clusters);
  const int64_t tiles = (p.I + kPairRows - 1) / kPairRows * ((p.J + 255) / 256), slices = (p.L + kBK - 1) / kBK;
  *splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(at_once / tiles, slices / 4), 32));
  return cudaSuccess;
}

cudaError_t error_word(int** at) {
  static std::atomic<int*> known[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && dev < 64 && (*at = known[dev].load(std::memory_order_relaxed))) return e;
  void* p = nullptr;
  if (e == cudaSuccess) e = cudaGetSymbolAddress(&p, g_errors);
  *at = (int*)p;
  if (e == cudaSuccess && dev < 64) known[dev].store(*at, std::memory_order_relaxed);
  return e;
}

cudaError_t read_errors(int* out, cudaStream_t s) {
  int* at = nullptr;
  cudaError_t e = error_word(&at);
  if (e == cudaSuccess) e = cudaMemcpyAsync(out, at, sizeof(int), cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e == cudaSuccess && *out) e = cudaMemsetAsync(at, 0, sizeof(int), s);
  return e;
}

}  // namespace lin
}  // namespace smat
