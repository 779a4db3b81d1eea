// The linear layers' products of bf16 matrices on the tensor cores (tcgen05; smat_linear.h, Product).
//
// A CTA makes tiles of 128 x BN sums: one warp fetches 64-deep slices of both operands by TMA into a ring of
// 128-byte-swizzled buffers, one thread multiplies them into tensor memory (fp32), eight warps take finished sums
// out of it, 32 at a time, and finish them (bias, activation, 8-bit form, residual, slope, older gradient) while the
// next tile's sums are made in the other half of tensor memory.
//
// SWAP false: the tile's 128 rows are rows i of the result, its columns are j. A thread then holds 32 columns of a
// row, whole groups of the 8-bit form, and reads and writes 64 bytes of a row at a time (whole sectors).
// SWAP true, for results of few rows: the 128 rows are columns j and the tile's columns are rows i, so that a wide
// weight fills the 128 and the few rows cost a narrow tile. A warp then holds 32 neighbouring columns of a row, one
// per lane. The same form finishes results whose rows do not start on 32 bytes, after a turn through shared memory.
//
// Where the tiles are fewer than the SMs, the sum is cut among the CTAs of a cluster: each leaves its share of the
// sums in its shared memory, then every CTA adds up some of the columns in the cluster's order and finishes them. No
// workspace, no atomics, the same result every time.

#include <cuda.h>

#include "smat_linear.cuh"
#include "smat_linear.h"

namespace smat {
namespace lin {

__device__ int g_errors;  // bit 0: a wait inside a product ran out of time

namespace {

constexpr int kBM = 128, kBK = 64;
constexpr int kEpiWarps = 8;
constexpr int kThreads = 32 * (kEpiWarps + 2);
constexpr int kTmaWarp = kEpiWarps, kMmaWarp = kEpiWarps + 1;
constexpr int kBytesA = kBM * kBK * 2;
constexpr int kTurn = 32 * 33 * 4;  // a warp's 32 x 32 sums, turned
constexpr unsigned long long kWaitNs = 2000000000ull;

template <int BN>
struct Ring {
  static constexpr int kBytesB = BN * kBK * 2;
  static constexpr int kStages = BN == 256 ? 4 : (BN == 128 ? 6 : 8);
  static constexpr int kStage = kBytesA + kBytesB;
  static constexpr int kBytes = kStages * kStage + kEpiWarps * kTurn + 1024;
};

struct Args {
  Product p;
  int64_t tiles, tiles_r, tiles_c;  // of the tile's rows and columns (of 128 and BN)
  int slices;                       // of 64 along the sum
  int share;                        // slices per CTA of a cluster
  bool wide;                        // rows of out, residual and q start on 32 bytes: 32 columns of a row at a time
  bool wide_bias;                   // bias on 16 bytes
};

__device__ __forceinline__ uint32_t smem_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}

// Waits until the barrier's phase `parity` is over; false after kWaitNs, or once another wait of this CTA has given
// up: the caller then leaves its loop, the CTA gives back its tensor memory and ends, and g_errors tells the host.
__device__ __noinline__ bool bar_wait_long(uint32_t bar, uint32_t parity, volatile int* dead) {
  unsigned long long begin, now;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(begin));
  for (;;) {
    for (int i = 0; i < 256; ++i)
      if (bar_try(bar, parity)) return true;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
    if (*dead) return false;
    if (now - begin > kWaitNs) {
      *dead = 1;
      atomicOr(&g_errors, 1);
      return false;
    }
  }
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* dead) {
  return bar_try(bar, parity) || bar_wait_long(bar, parity, dead);
}

__device__ __forceinline__ void tma_load(uint32_t to, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(to),
      "l"(map), "r"(bar), "r"(x), "r"(y)
      : "memory");
}

// Shared-memory matrix descriptor (128-byte swizzle). K-major: rows of 128 bytes (64 along the sum), 8 rows per
// 1024-byte block, blocks of rows 1024 bytes apart; 16 along the sum are 32 bytes. MN-major: 128 bytes hold 64 rows
// of the tile at one place of the sum, 8 places per 1024-byte block; 8 places further on is 1024 bytes, 64 rows
// further on 64 * 128 bytes; 16 along the sum are 2048 bytes.
template <bool MN>
__device__ __forceinline__ uint64_t descriptor(uint32_t address) {
  const uint64_t lbo = MN ? (kBK * 128) >> 4 : 1;
  return (uint64_t)((address & 0x3FFFF) >> 4) | lbo << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
         (uint64_t)2 << 61;
}
template <bool MN>
constexpr uint64_t kStep16 = (MN ? 2048 : 32) >> 4;

// kind::f16: fp32 sums of bf16 products, 128 x n
template <bool A_MN, bool B_MN, int N>
constexpr uint32_t kInstruction = 1u << 4 | 1u << 7 | 1u << 10 | (uint32_t)A_MN << 15 | (uint32_t)B_MN << 16 |
                                  (uint32_t)(N >> 3) << 17 | (uint32_t)(kBM >> 4) << 24;

__device__ __forceinline__ void mma(uint32_t sums, uint64_t a, uint64_t b, uint32_t instruction, bool add) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(sums),
      "l"(a), "l"(b), "r"(instruction), "r"((uint32_t)add)
      : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }

// 32 columns of the warp's 32 rows of tensor memory: thread's row, columns in order. The load and its wait are one
// statement, so that nothing can read the registers in between.
__device__ __forceinline__ void take32(uint32_t at, float (&v)[32]) {
  uint32_t u[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
      "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\ntcgen05.wait::ld.sync.aligned;"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
        "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]),
        "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]),
        "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
      : "r"(at)
      : "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(u[i]);
}

using bf16 = __nv_bfloat16;

__device__ __forceinline__ void unpack_words(const uint32_t* w, int words, float* v) {
#pragma unroll
  for (int i = 0; i < words; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load_words8(const void* p, uint32_t (&w)[8]) {
  asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(p));
}
__device__ __forceinline__ void store_words8(void* p, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
               "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

// What finishing 32 columns of a row reads, asked for before the sums are there: the residual, the older gradient or
// q, and e.
struct Beside {
  uint32_t w[16];
  uint32_t e;
};

template <int MODE>
__device__ __forceinline__ void ask_row(const Args& a, int64_t i, int64_t j, Beside& in) {
  const Product& p = a.p;
  if (i >= p.I) return;
  if (MODE == kGradInput) {
    if (p.act == SMAT_ACT_NONE) return;
    load_words8(p.q + i * p.ldq + j, *reinterpret_cast<uint32_t (*)[8]>(&in.w[0]));
    in.e = p.e[i * p.lde + j / kGroup];
    return;
  }
  const bf16* from = MODE == kForward ? (const bf16*)p.residual + i * p.ldr + j
                                      : (const bf16*)p.out + i * p.ldo + j;
  if (MODE == kForward ? p.residual != nullptr : p.accumulate != 0) {
    load_words8(from, *reinterpret_cast<uint32_t (*)[8]>(&in.w[0]));
    load_words8(from + 16, *reinterpret_cast<uint32_t (*)[8]>(&in.w[8]));
  }
}

// 32 columns j .. j + 31 of row i, one thread: whole sectors in and out. Returns the saved group's e.
template <int MODE>
__device__ __forceinline__ uint32_t finish_row(const Args& a, int64_t i, int64_t j, float (&v)[32], const Beside& in) {
  const Product& p = a.p;
  bf16* out = (bf16*)p.out + i * p.ldo + j;
  const bool there = i < p.I;
  uint32_t ex = 0;
  if (MODE == kForward) {
    if (p.bias) {
      const bf16* b = (const bf16*)p.bias + j;
      if (a.wide_bias) {
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
        for (int t = 0; t < 32; ++t) v[t] += to_float(b[t]);
      }
    }
    if (p.q) {
      float big = 0.0f;
#pragma unroll
      for (int t = 0; t < 32; ++t) big = larger(big, v[t]);
      ex = pack_exponent(__float_as_uint(big));
      uint32_t w[8];
      pack_words<8>(v, ex, w);
      if (there) store_words8(p.q + i * p.ldq + j, w);
    }
    SMAT_WITH_ACT(p.act, _Pragma("unroll") for (int t = 0; t < 32; ++t) v[t] = act_value<ACT>(v[t]))
  }
  if (MODE == kGradInput) {
    if (p.act != SMAT_ACT_NONE) {
      float h[32];
      unpack_words8<8>(in.w, in.e, h);
      SMAT_WITH_ACT(p.act, _Pragma("unroll") for (int t = 0; t < 32; ++t) v[t] *= act_slope<ACT>(h[t]))
    }
  } else if (MODE == kForward ? p.residual != nullptr : p.accumulate != 0) {
    float f[32];
    unpack_words(in.w, 16, f);
#pragma unroll
    for (int t = 0; t < 32; ++t) v[t] += f[t];
  }
  if (there) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t w[8];
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[16 * h + 2 * t], v[16 * h + 2 * t + 1]);
        w[t] = *reinterpret_cast<const uint32_t*>(&b);
      }
      store_words8(out + 16 * h, w);
    }
  }
  return ex;
}

// Column j of rows i .. i + 31, one thread; the warp holds 32 neighbouring columns from a multiple of 32 on. Rows are
// taken 8 at a time, what they read first.
template <int MODE>
__device__ __forceinline__ void finish_column(const Args& a, int64_t i, int64_t j, float (&v)[32]) {
  const Product& p = a.p;
  const bool there = j < p.J;
  const int lane = threadIdx.x % 32;
  bf16* out = (bf16*)p.out + i * p.ldo + j;
  const float bias = MODE == kForward && p.bias && there ? to_float(((const bf16*)p.bias)[j]) : 0.0f;
#pragma unroll
  for (int s = 0; s < 32; s += 8) {
    const int rows = (int)(p.I - i - s < 8 ? p.I - i - s : 8);
    if (rows <= 0) return;
    float x[8];
    if (MODE == kForward) {
#pragma unroll
      for (int t = 0; t < 8; ++t)
        x[t] = p.residual && there && t < rows
                   ? to_float(((const bf16*)p.residual)[(i + s + t) * p.ldr + j])
                   : 0.0f;
#pragma unroll
      for (int t = 0; t < 8; ++t) v[s + t] += bias;
      if (p.q) {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          const uint32_t top =
              __reduce_max_sync(0xFFFFFFFFu, there ? __float_as_uint(fabsf(v[s + t])) : 0u);
          const uint32_t ex = pack_exponent(top);
          if (there && t < rows) {
            p.q[(i + s + t) * p.ldq + j] = (int8_t)pack_one(v[s + t], ex);
            if (lane == 0) p.e[(i + s + t) * p.lde + j / kGroup] = (uint8_t)ex;
          }
        }
      }
      SMAT_WITH_ACT(p.act, _Pragma("unroll") for (int t = 0; t < 8; ++t) v[s + t] = act_value<ACT>(v[s + t]) + x[t])
    }
    if (MODE == kGradInput && p.act != SMAT_ACT_NONE) {
#pragma unroll
      for (int t = 0; t < 8; ++t)
        x[t] = there && t < rows ? (float)p.q[(i + s + t) * p.ldq + j] *
                                       unpack_scale(p.e[(i + s + t) * p.lde + j / kGroup])
                                 : 0.0f;
      SMAT_WITH_ACT(p.act, _Pragma("unroll") for (int t = 0; t < 8; ++t) v[s + t] *= act_slope<ACT>(x[t]))
    }
    if (MODE == kGradWeight && p.accumulate) {
#pragma unroll
      for (int t = 0; t < 8; ++t) x[t] = there && t < rows ? to_float(out[(s + t) * p.ldo]) : 0.0f;
#pragma unroll
      for (int t = 0; t < 8; ++t) v[s + t] += x[t];
    }
#pragma unroll
    for (int t = 0; t < 8; ++t)
      if (there && t < rows) out[(s + t) * p.ldo] = from_float<bf16>(v[s + t]);
  }
}

// `count` blocks of 32 columns of the tile, from column col0 of the result on, of the warp's 32 rows (row0 on; rows
// and columns of the tile, that is): `sums(c, v)` gives block c's sums.
template <int MODE, bool SWAP, class Sums>
__device__ __forceinline__ void finish(const Args& a, int64_t row0, int64_t col0, int first, int end, int step,
                                       float* turn, Sums&& sums) {
  const int lane = threadIdx.x % 32;
  if (first >= end) return;
  const bool rows = !SWAP && a.wide;
  Beside in;
  if (rows && col0 + 32 * first + 32 <= a.p.J) ask_row<MODE>(a, row0 + lane, col0 + 32 * first, in);
  for (int c = first; c < end; c += step) {
    const int64_t col = col0 + 32 * c;
    float v[32];
    sums(c, v);
    if (SWAP) {
      if (col < a.p.I && row0 < a.p.J) finish_column<MODE>(a, col, row0 + lane, v);
      continue;
    }
    if (rows && col + 32 <= a.p.J) {
      const Beside now = in;
      if (c + step < end && col + 32 * step + 32 <= a.p.J) ask_row<MODE>(a, row0 + lane, col + 32 * step, in);
      const uint32_t ex = finish_row<MODE>(a, row0 + lane, col, v, now);
      if (MODE == kForward && a.p.q && row0 + lane < a.p.I)
        a.p.e[(row0 + lane) * a.p.lde + col / kGroup] = (uint8_t)ex;
      continue;
    }
    if (row0 >= a.p.I || col >= a.p.J) continue;
    __syncwarp();
#pragma unroll
    for (int t = 0; t < 32; ++t) turn[lane * 33 + t] = v[t];
    __syncwarp();
#pragma unroll
    for (int t = 0; t < 32; ++t) v[t] = turn[t * 33 + lane];
    finish_column<MODE>(a, row0, col + lane, v);
  }
}

// The tiles' order: strips of 16 tiles of rows, down a strip's rows first, so that the tiles in work at one time
// share rows and columns of the operands in L2.
__device__ __forceinline__ void tile_place(const Args& a, int64_t tile, int64_t& r, int64_t& c) {
  constexpr int64_t kStrip = 16;
  const int64_t per = kStrip * a.tiles_c, strip = tile / per, in = tile - strip * per;
  const int64_t high = a.tiles_r - strip * kStrip < kStrip ? a.tiles_r - strip * kStrip : kStrip;
  c = in / high;
  r = strip * kStrip + in - c * high;
}

template <int MODE, bool SWAP, int BN>
__global__ void __launch_bounds__(kThreads, 1)
    tc_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
              const __grid_constant__ Args a) {
  // the tile's rows come from W where swapped, from the other operand else
  constexpr bool A_MN = SWAP ? MODE == kGradInput : MODE == kGradWeight;
  constexpr bool B_MN = SWAP ? false : MODE != kForward;
  static_assert(!(SWAP && MODE == kGradWeight), "a weight gradient's rows and columns are both a layer's");
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

  if (threadIdx.x == 0) {
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
  }
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

  uint32_t shares, rank;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(shares));
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const int slice0 = (int)rank * a.share;
  const int slices = max(0, min(a.share, a.slices - slice0));
  const int64_t step = gridDim.x / shares;

  if (warp == kTmaWarp && lane == 0) {
    uint32_t n = 0;  // slices fetched so far
    bool ok = true;
    for (int64_t tile = blockIdx.x / shares; ok && tile < a.tiles; tile += step) {
      int64_t tr, tc;
      tile_place(a, tile, tr, tc);
      const int r0 = (int)(tr * kBM), c0 = (int)(tc * BN);
      for (int k = 0; k < slices; ++k, ++n) {
        const uint32_t s = n % kStages;
        ok = bar_wait(empty + 8 * s, (n / kStages + 1) & 1, dead);
        if (!ok) break;
        const uint32_t bar = full + 8 * s, to_a = smem_address(ring) + s * kStage, to_b = to_a + kBytesA;
        const int l = (slice0 + k) * kBK;
        bar_expect(bar, kStage);
        if (A_MN) {
#pragma unroll
          for (int b = 0; b < kBM / 64; ++b) tma_load(to_a + b * 8192, &map_a, r0 + 64 * b, l, bar);
        } else {
          tma_load(to_a, &map_a, l, r0, bar);
        }
        if (B_MN) {
#pragma unroll
          for (int b = 0; b < BN / 64; ++b) tma_load(to_b + b * 8192, &map_b, c0 + 64 * b, l, bar);
        } else {
          tma_load(to_b, &map_b, l, c0, bar);
        }
      }
    }
    if (!ok)  // copies in flight land before the CTA ends
      for (uint32_t s = 0; s < kStages && s < n; ++s) {
        const uint32_t last = n - 1 - s;
        for (int i = 0; i < (1 << 20) && !bar_try(full + 8 * (last % kStages), last / kStages & 1); ++i) {
        }
      }
  } else if (warp == kMmaWarp && lane == 0) {
    constexpr uint32_t kInst = kInstruction<A_MN, B_MN, BN>;
    uint32_t n = 0, made = 0;
    bool ok = true;
    for (int64_t tile = blockIdx.x / shares; ok && tile < a.tiles; tile += step, ++made) {
      const uint32_t half = made & 1, sums = tmem + half * BN;
      ok = bar_wait(sums_empty + 8 * half, (made / 2 + 1) & 1, dead);
      if (!ok) break;
      fence_after();
      for (int k = 0; k < slices; ++k, ++n) {
        const uint32_t s = n % kStages;
        ok = bar_wait(full + 8 * s, n / kStages & 1, dead);
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
      for (int i = 0; i < (1 << 20) && !bar_try(drained, 0); ++i) {
      }
    }
  } else if (warp < kEpiWarps) {
    const int quarter = warp % 4;  // the 32 rows of tensor memory that this warp may read
    float* turn = reinterpret_cast<float*>(ring + kStages * kStage + warp * kTurn);
    uint32_t made = 0;
    for (int64_t tile = blockIdx.x / shares; tile < a.tiles; tile += step, ++made) {
      int64_t tr, tc;
      tile_place(a, tile, tr, tc);
      const int64_t r0 = tr * kBM + 32 * quarter, c0 = tc * BN;
      const uint32_t half = made & 1, sums = tmem + half * BN + ((uint32_t)(32 * quarter) << 16);
      if (!bar_wait(sums_full + 8 * half, made / 2 & 1, dead)) break;
      fence_after();
      // this warp's blocks of 32 columns: the first or the second half of the tile's
      constexpr int kBlocks = BN / 32, kMine = (kBlocks + 1) / 2;
      const int first = warp / 4 * kMine, end = min(kBlocks, first + kMine);
      auto take = [&](int c, float(&v)[32]) {
        if (slices > 0) {
          take32(sums + 32 * c, v);
        } else {
#pragma unroll
          for (int t = 0; t < 32; ++t) v[t] = 0.0f;
        }
      };
      if (shares == 1) {
        if (first >= end && lane == 0) bar_arrive(sums_empty + 8 * half);  // none of a narrow tile's columns
        finish<MODE, SWAP>(a, r0, c0, first, end, 1, turn, [&](int c, float(&v)[32]) {
          take(c, v);
          if (c + 1 == end) {  // the last of this warp's columns are out
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(sums_empty + 8 * half);
          }
        });
      } else {
        // the ring is free: every product that read it is done. [column][128 rows]
        float* part = reinterpret_cast<float*>(ring) + 32 * quarter + lane;
        for (int c = first; c < end; ++c) {
          float v[32];
          take(c, v);
#pragma unroll
          for (int t = 0; t < 32; ++t) part[(32 * c + t) * kBM] = v[t];
        }
      }
    }
  }
  __syncwarp();
  if (shares > 1) {
    // one tile per cluster: its CTAs add up and finish 32 columns each in turn
    __syncthreads();
    cluster_sync();
    if (warp < kEpiWarps && !*dead) {
      int64_t tr, tc;
      tile_place(a, blockIdx.x / shares, tr, tc);
      const int quarter = warp % 4;
      const float* part = reinterpret_cast<const float*>(ring) + 32 * quarter + lane;
      float* turn = reinterpret_cast<float*>(ring + kStages * kStage + warp * kTurn);
      finish<MODE, SWAP>(
          a, tr * kBM + 32 * quarter, tc * BN, (int)rank + (int)shares * (warp / 4), BN / 32,
          (int)shares * (kEpiWarps / 4), turn, [&](int c, float(&v)[32]) {
#pragma unroll
            for (int t = 0; t < 32; ++t) v[t] = 0.0f;
            for (uint32_t s = 0; s < shares; ++s)
#pragma unroll
              for (int t = 0; t < 32; ++t) v[t] += cluster_load(part + (32 * c + t) * kBM, s);
          });
    }
    cluster_sync();
  }
  fence_before();
  __syncthreads();
  if (warp == kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * BN));
}

}  // namespace

namespace {

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                            const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

Encode encoder() {
  static const Encode f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<Encode>(p);
  }();
  return f;
}

// A row-major bf16 matrix [outer, inner] in boxes of 64 x `box`; what lies outside reads as 0.
bool encode(CUtensorMap* map, const void* p, int64_t inner, int64_t outer, int64_t ld, int box) {
  const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)outer};
  const cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t boxes[2] = {64, (cuuint32_t)box}, ones[2] = {1, 1};
  const Encode f = encoder();
  return f && f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims, strides, boxes, ones,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool can(const void* p, int64_t ld, size_t elem) { return (uintptr_t)p % 32 == 0 && (uint64_t)ld * elem % 32 == 0; }

template <int MODE, bool SWAP, int BN>
cudaError_t launch_tile(const Product& p, int sms, cudaStream_t s) {
  constexpr bool A_MN = SWAP ? MODE == kGradInput : MODE == kGradWeight;
  constexpr bool B_MN = SWAP ? false : MODE != kForward;
  Args a = {};
  a.p = p;
  const int64_t R = SWAP ? p.J : p.I, C = SWAP ? p.I : p.J;
  a.tiles_r = (R + kBM - 1) / kBM;
  a.tiles_c = (C + BN - 1) / BN;
  a.tiles = a.tiles_r * a.tiles_c;
  a.slices = (int)((p.L + kBK - 1) / kBK);
  a.wide = can(p.out, p.ldo, 2) && (!p.residual || can(p.residual, p.ldr, 2)) && (!p.q || can(p.q, p.ldq, 1));
  a.wide_bias = (uintptr_t)p.bias % 16 == 0;
  // shares of the sum while the CTAs are fewer than the SMs, four slices in each at least
  int shares = 1;
  while (shares < 8 && a.tiles * shares * 2 <= sms && a.slices >= shares * 2 * 4) shares *= 2;
  a.share = (a.slices + shares - 1) / shares;

  CUtensorMap ma = {}, mb = {};  // not read where the sum is over nothing
  if (p.L > 0) {
    const void *pa = SWAP ? p.b : p.a, *pb = SWAP ? p.a : p.b;
    const int64_t lda = SWAP ? p.ldb : p.lda, ldb = SWAP ? p.lda : p.ldb;
    const bool ok = (A_MN ? encode(&ma, pa, R, p.L, lda, kBK) : encode(&ma, pa, p.L, R, lda, kBM)) &&
                    (B_MN ? encode(&mb, pb, C, p.L, ldb, kBK) : encode(&mb, pb, p.L, C, ldb, BN));
    if (!ok) return cudaErrorNotSupported;
  }
  auto* f = tc_kernel<MODE, SWAP, BN>;
  static std::atomic<uint64_t> allowed;
  const cudaError_t e = allow_shared(f, Ring<BN>::kBytes, allowed);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  const int64_t ctas = shares > 1 ? a.tiles * shares : (a.tiles < sms ? a.tiles : sms);
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Ring<BN>::kBytes;
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim = {(unsigned)shares, 1, 1};
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, f, ma, mb, a);
}

template <int MODE>
cudaError_t launch_mode(const Product& p, int sms, cudaStream_t s) {
  if (MODE != kGradWeight) {
    constexpr int M = MODE == kGradWeight ? (int)kForward : MODE;
    if (p.I <= 32) return launch_tile<M, true, 32>(p, sms, s);
    if (p.I <= 64) return launch_tile<M, true, 64>(p, sms, s);
    if (p.I <= 128) return launch_tile<M, true, 128>(p, sms, s);
  }
  return launch_tile<MODE, false, 256>(p, sms, s);
}

}  // namespace

cudaError_t launch_tc(const Product& p, int sms, cudaStream_t s) {
  switch (p.mode) {
    case kForward: return launch_mode<kForward>(p, sms, s);
    case kGradInput: return launch_mode<kGradInput>(p, sms, s);
    default: return launch_mode<kGradWeight>(p, sms, s);
  }
}

cudaError_t read_errors(int* out, cudaStream_t s) {
  void* at = nullptr;
  cudaError_t e = cudaGetSymbolAddress(&at, g_errors);
  if (e == cudaSuccess) e = cudaMemcpyAsync(out, at, sizeof(int), cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e == cudaSuccess && *out) e = cudaMemsetAsync(at, 0, sizeof(int), s);
  return e;
}

}  // namespace lin
}  // namespace smat
