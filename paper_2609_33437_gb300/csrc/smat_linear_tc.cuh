// What the tensor-core products share: barriers, TMA copies, tcgen05 instructions and their descriptors.
#pragma once

#include <atomic>

#include <cuda.h>

#include "smat_linear.cuh"

namespace smat {
namespace lin {

constexpr int kBM = 128, kBK = 64;  // a tile's rows; a slice of the sum
constexpr int kEpiWarps = 8;
constexpr int kThreads = 32 * (kEpiWarps + 2);
constexpr int kTmaWarp = kEpiWarps, kMmaWarp = kEpiWarps + 1;
// A wait's limit; one that lasts for a whole share of a sum has kSliceNs more for each slice of it. (A slice takes 290 ns where
// one cluster works by itself and up to 450 with every SM copying; the largest share has 2^23 of them, 2.4 s.)
constexpr unsigned long long kWaitNs = 2000000000ull, kSliceNs = 2000ull;

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

// Waits until the barrier's phase `parity` is over; false after `limit`, or once another wait of this CTA has given
// up: the caller then leaves its loop, the CTA gives back its tensor memory and ends, and *errors tells the host.
static __device__ __noinline__ bool bar_wait_long(uint32_t bar, uint32_t parity, volatile int* dead, int* errors,
                                                  unsigned long long limit) {
  unsigned long long begin, now;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(begin));
  for (;;) {
    for (int i = 0; i < 256; ++i)
      if (bar_try(bar, parity)) return true;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
    if (*dead) return false;
    if (now - begin > limit) {
      *dead = 1;
      atomicOr(errors, 1);
      return false;
    }
  }
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* dead, int* errors,
                                         unsigned long long limit = kWaitNs) {
  return bar_try(bar, parity) || bar_wait_long(bar, parity, dead, errors, limit);
}

// A whole warp's wait: its lanes may time out one by one, but they all go on, or all give up.
__device__ __forceinline__ bool bar_wait_warp(uint32_t bar, uint32_t parity, volatile int* dead, int* errors,
                                              unsigned long long limit = kWaitNs) {
  return __all_sync(0xFFFFFFFFu, bar_wait(bar, parity, dead, errors, limit));
}

// After a wait has given up: what this CTA has under way itself (copies into its shared memory, multiplications) ends before
// the CTA does. Until the phase is over, or kDrainNs; and for what signals another CTA's barrier, kPauseNs.
constexpr unsigned long long kDrainNs = 100000000ull, kPauseNs = 1000000ull;
static __device__ __noinline__ void bar_drain(uint32_t bar, uint32_t parity) {
  unsigned long long begin, now;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(begin));
  do {
    if (bar_try(bar, parity)) return;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
  } while (now - begin < kDrainNs);
}
static __device__ __noinline__ void drain_pause() {
  unsigned long long begin, now;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(begin));
  do {
    __nanosleep(1000);
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
  } while (now - begin < kPauseNs);
}

__device__ __forceinline__ void tma_load(uint32_t to, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(to),
      "l"(map), "r"(bar), "r"(x), "r"(y)
      : "memory");
}

__device__ __forceinline__ void tma_store(const CUtensorMap* map, uint32_t from, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(from), "r"(x),
               "r"(y)
               : "memory");
}
__device__ __forceinline__ void tma_add(const CUtensorMap* map, uint32_t from, int x, int y) {
  asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map),
               "r"(from), "r"(x), "r"(y)
               : "memory");
}
__device__ __forceinline__ void tma_load3(uint32_t to, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(
          to),
      "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
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

// kind::f16: fp32 sums of bf16 products, M x N
template <bool A_MN, bool B_MN, int N, int M = kBM>
constexpr uint32_t kInstruction = 1u << 4 | 1u << 7 | 1u << 10 | (uint32_t)A_MN << 15 | (uint32_t)B_MN << 16 |
                                  (uint32_t)(N >> 3) << 17 | (uint32_t)(M >> 4) << 24;

__device__ __forceinline__ void mma(uint32_t sums, uint64_t a, uint64_t b, uint32_t instruction, bool add) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(sums),
      "l"(a), "l"(b), "r"(instruction), "r"((uint32_t)add)
      : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// The same for a pair of CTAs (cta_group::2): copies signal a barrier of either CTA (its address across the cluster), one
// thread of the first CTA multiplies from both CTAs' shared memory into both's tensor memory, and what it commits to is a
// barrier of each CTA in `mask`.
__device__ __forceinline__ uint32_t cluster_address_of(uint32_t shared, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(shared), "r"(rank));
  return a;
}
__device__ __forceinline__ void bar_arrive_there(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_pair(uint32_t to, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], "
      "[%2];" ::"r"(to),
      "l"(map), "r"(bar), "r"(x), "r"(y)
      : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t sums, uint64_t a, uint64_t b, uint32_t instruction, bool add) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(sums),
      "l"(a), "l"(b), "r"(instruction), "r"((uint32_t)add)
      : "memory");
}
__device__ __forceinline__ void mma_commit_pair(uint32_t bar, uint16_t mask) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
      "h"(mask)
      : "memory");
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

__device__ __forceinline__ void take16(uint32_t at, float (&v)[16]) {
  uint32_t u[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
        "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
      : "r"(at)
      : "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(u[i]);
}
__device__ __forceinline__ void take8(uint32_t at, float (&v)[8]) {
  uint32_t u[8];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\ntcgen05.wait::ld.sync.aligned;"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7])
      : "r"(at)
      : "memory");
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(u[i]);
}

// A thread's row of a tile's sums, 32 x N of a warp: [column][128 rows], see the products.
template <int N>
__device__ __forceinline__ void put_part(float* p, const float (&v)[N]) {
#pragma unroll
  for (int t = 0; t < N; ++t) p[t * kBM] = v[t];
}
// The shares' sums added in the cluster's order, several CTAs' loads in flight.
template <int N, class Load>
__device__ __forceinline__ void add_parts(uint32_t shares, float (&v)[N], Load&& load) {
  constexpr int kAhead = N == 32 ? 1 : 4;
#pragma unroll
  for (int t = 0; t < N; ++t) v[t] = 0.0f;
  for (uint32_t s = 0; s < shares; s += kAhead) {
    float x[kAhead][N];
#pragma unroll
    for (int h = 0; h < kAhead; ++h)
#pragma unroll
      for (int t = 0; t < N; ++t) x[h][t] = s + h < shares ? load(s + h, t) : 0.0f;
#pragma unroll
    for (int h = 0; h < kAhead; ++h)
#pragma unroll
      for (int t = 0; t < N; ++t) v[t] += x[h][t];
  }
}

// The tiles' order: strips of STRIP tiles of rows, down a strip's rows first, so that the tiles in work at one time
// share rows and columns of the operands in L2.
template <int64_t STRIP>
__device__ __forceinline__ void tile_place(int64_t tiles_r, int64_t tiles_c, int64_t tile, int64_t& r, int64_t& c) {
  const int64_t per = STRIP * tiles_c, strip = tile / per, in = tile - strip * per;
  const int64_t high = tiles_r - strip * STRIP < STRIP ? tiles_r - strip * STRIP : STRIP;
  c = in / high;
  r = strip * STRIP + in - c * high;
}

// ---- host side ----

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                            const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline Encode encoder() {
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

// A row-major matrix [outer, inner] of bf16, bytes or fp32 in boxes of `wide` x `high`, swizzled over a box's row; what lies
// outside reads as 0.
inline bool encode(CUtensorMap* map, const void* p, int64_t inner, int64_t outer, int64_t ld, int high, int wide = 64,
            int elem = 2) {
  const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)outer};
  const cuuint64_t strides[1] = {(cuuint64_t)ld * elem};
  const cuuint32_t boxes[2] = {(cuuint32_t)wide, (cuuint32_t)high}, ones[2] = {1, 1};
  const int row = wide * elem;
  const Encode f = encoder();
  return f && f(map, elem == 1   ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                     : elem == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32,
                2, const_cast<void*>(p), dims, strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                row == 128  ? CU_TENSOR_MAP_SWIZZLE_128B
                : row == 64 ? CU_TENSOR_MAP_SWIZZLE_64B
                            : CU_TENSOR_MAP_SWIZZLE_32B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class F, class... A>
cudaError_t launch(F* f, int64_t ctas, int cluster, int threads, int bytes, cudaStream_t s, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim = {(unsigned)cluster, 1, 1};
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, f, args...);
}

// How many clusters of `shares` CTAs of a kernel run at once on the current device, asked for once (a GPU's parts hold
// different numbers of SMs, so this is less than SMs / shares).
template <class F>
int64_t clusters_at_once(F* f, int shares, int threads, int bytes, std::atomic<int> (&known)[64][9]) {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev >= 64) return 1;
  if ((n = known[dev][shares].load(std::memory_order_relaxed)) > 0) return n;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)shares);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = bytes;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim = {(unsigned)shares, 1, 1};
  cfg.attrs = at;
  cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&n, f, &cfg) != cudaSuccess || n < 1) {
    cudaGetLastError();
    n = 1;
  }
  known[dev][shares].store(n, std::memory_order_relaxed);
  return n;
}

}  // namespace lin
}  // namespace smat
