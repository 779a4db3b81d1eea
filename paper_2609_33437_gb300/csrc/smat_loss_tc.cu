// The logits of the loss over a vocabulary on the tensor cores (bf16; smat_loss.h, Logits): every tile of x W^T is reduced to its
// rows' largest logits and sums of exponentials where it is made, and the targets' logits are picked out of it.
//
// The copies, barriers and multiplications are those of the linear layers' products (smat_linear_tc.cu). What differs is the sum:
// tensor memory's additions cut off what does not fit, 1.8e-6 of a sum of 4,096 terms in the mean, which shows in a loss (fp32,
// the difference of two such sums). So the sum is made in parts there, three at least and none of more than 512 terms, and the
// finishing warps add these up in registers, rounding to nearest, while the next one is made in tensor memory's other half. The
// error of losses beside that of plain fp32 products, 300 rows, 20,000 words: of 4,096 terms 0.4 of it, 1,024 0.7, 896 0.7, 512 0.7,
// 256 0.8; in parts of 512 whatever the sum's length 0.4, 1.1, 1.1, 1.8, 1.3. What the parts cost, 2049 x 896 x 151936: 401 us in
// one, 433 in two, 482 in three, 521 in four (a tile's exponentials take as long as 8 slices' products, and at the power limit
// every instruction counts); 8192 x 4096 x 32000 1.14 ms in 8.
//
// Wide products (wide_kernel): tiles of 256 rows x `width` words by pairs of CTAs; a thread holds a row's sums of a
// quarter of the tile's words, 64 registers. Products of at most 128 rows (narrow_kernel): tiles of 128 words x BN rows, bound by W's
// bytes; a tile's sums change hands through shared memory so that a row's 128 words lie with 8 neighbouring lanes, and a CTA
// keeps its rows' largest values and sums from tile to tile.

#include "smat_loss.h"

#include <algorithm>

#include "smat_linear_tc.cuh"

namespace smat {
namespace loss {
namespace {

using namespace smat::lin;

constexpr int kChunk = 8, kLeastChunks = 3;  // slices of 64 that tensor memory adds up at most, and parts of a sum at least
constexpr int kWarps = 8, kLoad = kWarps, kMultiply = kWarps + 1;  // a narrow tile's: those that finish, and the two others
static_assert(kThreads == 32 * (kWarps + 2), "a narrow tile's threads");
constexpr int kBytesRows = kBM * kBK * 2;

struct Args {
  Logits p;
  int64_t tiles, tiles_r, tiles_c;
  int slices, chunk, chunks, width;  // chunks of `chunk` slices, the last one as long or shorter
  int* errors;
};

// The larger value; NaN if one is.
__device__ __forceinline__ float top_of(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ float top_of(float a, float b, float c) {
  float y;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// 16 columns of tensor memory added to 16 sums
__device__ __forceinline__ void add16(uint32_t at, float* v) {
  float x[16];
  take16(at, x);
#pragma unroll
  for (int t = 0; t < 16; ++t) v[t] += x[t];
}
// (m, s) joined with another's; parts of nothing have m = -infinity
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
  const float top = top_of(m, m2);
  if (top == -INFINITY) return;
  s = s * exp2_fast((m - top) * kLog2e) + s2 * exp2_fast((m2 - top) * kLog2e);
  m = top;
}
// The largest of N logits and the sum of exp(logit - largest); of nothing but -infinity: -infinity and 0. Those from `count` on
// are none.
template <int N>
__device__ __forceinline__ void reduce(float (&v)[N], int count, float& m, float& s) {
  if (count < N) {
#pragma unroll
    for (int t = 0; t < N; ++t) v[t] = t < count ? v[t] : -INFINITY;
  }
  float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
  for (int t = 0; t < N; t += 2) top[t / 2 % 4] = top_of(top[t / 2 % 4], v[t], v[t + 1]);
  m = top_of(top_of(top[0], top[1], top[2]), top[3]);
  s = 0.0f;
  if (m == -INFINITY) return;
  const float less = m * kLog2e;
  float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int t = 0; t < N; ++t) part[t % 4] += exp2_fast(fmaf(v[t], kLog2e, -less));
  s = (part[0] + part[1]) + (part[2] + part[3]);
}
// Logit number `at` of N
template <int N>
__device__ __forceinline__ float pick(const float (&v)[N], int at) {
  float x = v[0];
#pragma unroll
  for (int t = 1; t < N; ++t) x = t == at ? v[t] : x;
  return x;
}

// Whether all the threads that finish are to go on (`ok` of each): they meet here once a tile.
template <int THREADS>
__device__ __forceinline__ bool all_go_on(bool ok) {
  int all;
  asm volatile("{\n.reg .pred p, q;\nsetp.ne.s32 p, %1, 0;\nbarrier.red.and.pred q, 1, %2, p;\nselp.s32 %0, 1, 0, q;\n}"
               : "=r"(all)
               : "r"((int)ok), "n"(THREADS)
               : "memory");
  return all;
}

constexpr int kWideRows = 2 * kBM, kWideStages = 6, kWideStage = 2 * kBytesRows;
// Finishing warps, by fours: a quarter of a tile's words each, 64 sums a thread.
constexpr int kWideWarps = 16, kSides = kWideWarps / 4, kEach = 256 / kSides;
constexpr int kWideThreads = 32 * (kWideWarps + 2), kWideBytes = kWideStages * kWideStage + 1024;
constexpr int kSums = 256;
constexpr int kWideLoad = kWideWarps, kWideMultiply = kWideWarps + 1;

// See pair_kernel in smat_linear_tc.cu: the pair's first CTA ("leader") multiplies for both.
__global__ void __launch_bounds__(kWideThreads, 1)
    wide_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ Args a) {
  constexpr int kStages = kWideStages, kStage = kWideStage;
  extern __shared__ uint8_t raw[];
  __shared__ __align__(8) uint64_t bars[2 * kStages + 5];
  __shared__ float2 sides[2][kSides][kBM];
  __shared__ uint32_t tmem_at;
  __shared__ int dead_flag;
  uint8_t* ring = raw + ((1024 - (smem_address(raw) & 1023)) & 1023);
  volatile int* dead = &dead_flag;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t full = smem_address(bars), empty = full + 8 * kStages, sums_full = empty + 8 * kStages, sums_empty = sums_full + 16,
                 drained = sums_empty + 16;
  uint32_t rank;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const uint32_t member = rank & 1;
  const int64_t first_tile = blockIdx.x / 2, step = gridDim.x / 2;
  const int half_width = a.width / 2, chunks = a.chunks;

  if (warp == kWideLoad && lane == 0) {
    dead_flag = 0;
    for (int s = 0; s < kStages; ++s) {
      bar_init(full + 8 * s, 1);
      bar_init(empty + 8 * s, 1);
    }
    bar_init(drained, 1);
    for (int b = 0; b < 2; ++b) {
      bar_init(sums_full + 8 * b, 1);
      bar_init(sums_empty + 8 * b, 2 * kWideWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  if (warp == kWideMultiply) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_address(&tmem_at)), "r"(2 * kSums)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    fence_before();
  }
  __syncthreads();
  cluster_sync();  // the partner's barriers are there
  fence_after();
  const uint32_t tmem = tmem_at;

  if (warp == kWideLoad && lane == 0) {
    const uint32_t bytes = kBytesRows + half_width * kBK * 2;
    const uint32_t full_there = cluster_address_of(full, 0);
    uint32_t n = 0;  // slices fetched so far
    bool ok = true;
    for (int64_t tile = first_tile; ok && tile < a.tiles; tile += step) {
      int64_t tr, tc;
      tile_place<8>(a.tiles_r, a.tiles_c, tile, tr, tc);
      const int r0 = (int)(tr * kWideRows) + (int)member * kBM, c0 = (int)(tc * a.width) + (int)member * half_width;
      for (int k = 0; k < a.slices; ++k, ++n) {
        const uint32_t s = n % kStages;
        ok = bar_wait(empty + 8 * s, (n / kStages + 1) & 1, dead, a.errors);
        if (!ok) break;
        const uint32_t bar = full_there + 8 * s, to = smem_address(ring) + s * kStage;
        if (member == 0) bar_expect(full + 8 * s, 2 * bytes);
        tma_load_pair(to, &map_x, k * kBK, r0, bar);
        tma_load_pair(to + kBytesRows, &map_w, k * kBK, c0, bar);
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
  } else if (warp == kWideMultiply && lane == 0 && member == 0) {
    const uint32_t inst = kInstruction<false, false, 0, kWideRows> | (uint32_t)(a.width >> 3) << 17;
    const uint16_t both = 3u;
    uint32_t n = 0, made = 0;
    bool ok = true;
    for (int64_t tile = first_tile; ok && tile < a.tiles; tile += step) {
      for (int c = 0; ok && c < chunks; ++c, ++made) {
        const uint32_t half = made & 1, sums = tmem + half * kSums;
        ok = bar_wait(sums_empty + 8 * half, (made / 2 + 1) & 1, dead, a.errors);
        if (!ok) break;
        fence_after();
        const int end = min(a.chunk, a.slices - c * a.chunk);
        for (int k = 0; k < end; ++k, ++n) {
          const uint32_t s = n % kStages;
          ok = bar_wait(full + 8 * s, n / kStages & 1, dead, a.errors);
          if (!ok) break;
          fence_after();
          const uint32_t at = smem_address(ring) + s * kStage;
          const uint64_t da = descriptor<false>(at), db = descriptor<false>(at + kBytesRows);
#pragma unroll
          for (int t = 0; t < kBK / 16; ++t)
            mma_pair(sums, da + t * kStep16<false>, db + t * kStep16<false>, inst, k > 0 || t > 0);
          mma_commit_pair(empty + 8 * s, both);
        }
        if (ok) mma_commit_pair(sums_full + 8 * half, both);
      }
    }
    if (!ok) {  // products in flight end before the CTAs do
      mma_commit_pair(drained, 1);
      bar_drain(drained, 0);
    }
  } else if (warp < kWideWarps) {
    const int quarter = warp % 4, side = warp / 4;  // the 32 rows of tensor memory that this warp may read; its part of the words
    const int each = a.width / kSides;
    const uint32_t sums_empty_there = cluster_address_of(sums_empty, 0);
    uint32_t made = 0;
    bool ok = true;
    int turn = 0;
    for (int64_t tile = first_tile; tile < a.tiles; tile += step, turn ^= 1) {
      int64_t tr, tc;
      tile_place<8>(a.tiles_r, a.tiles_c, tile, tr, tc);
      const int64_t row = tr * kWideRows + (int)member * kBM + 32 * quarter + lane, col = tc * a.width + side * each;
      const int count = (int)max((int64_t)0, min((int64_t)each, a.p.cols - col));  // words of this thread
      int target = -1;  // among them
      if (row < a.p.rows) {
        const int64_t at = a.p.targets[row] - a.p.first_col - col;
        if (at >= 0 && at < count) target = (int)at;
      }
      float v[kEach];
#pragma unroll
      for (int t = 0; t < kEach; ++t) v[t] = 0.0f;
      for (int c = 0; c < chunks; ++c, ++made) {
        const uint32_t half = made & 1, sums = tmem + half * kSums + side * each + ((uint32_t)(32 * quarter) << 16);
        ok = bar_wait_warp(sums_full + 8 * half, made / 2 & 1, dead, a.errors);
        if (!ok) break;
        fence_after();
#pragma unroll
        for (int b = 0; b < kEach / 16; ++b)
          if (16 * b < each) add16(sums + 16 * b, v + 16 * b);
        fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive_there(sums_empty_there + 8 * half);
      }
      if (ok && target >= 0) a.p.picked[row] = pick<kEach>(v, target);
      float m, s;
      reduce<kEach>(v, count, m, s);
      // the sides' parts of a row are joined by the first one's threads; the next tile's go to the other place
      sides[turn][side][32 * quarter + lane] = make_float2(m, s);
      ok = all_go_on<32 * kWideWarps>(ok);
      if (!ok) break;
      if (side == 0 && row < a.p.rows) {
#pragma unroll
        for (int t = 1; t < kSides; ++t) {
          const float2 o = sides[turn][t][32 * quarter + lane];
          join(m, s, o.x, o.y);
        }
        a.p.partials[tc * a.p.rows + row] = make_float2(m, s);
      }
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  cluster_meet();  // the partner's multiplications read this CTA's shared memory, and its arrivals write it
  if (warp == kWideMultiply)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * kSums));
}

// Two CTAs per SM, so that one's start and end lie beside the other's copies; with 128 rows one, with as much on its way.
template <int BN>
struct Ring {
  static constexpr int kStages = BN == 32 ? 4 : BN == 64 ? 3 : 6, kCtas = BN == 128 ? 1 : 2;
  static constexpr int kStage = kBytesRows + BN * kBK * 2;
  static constexpr int kBytes = kStages * kStage + 1024;
};
constexpr int kHand = 32, kHandPad = 132;  // rows that change hands at a time, and a row's 128 words there

template <int BN>
__global__ void __launch_bounds__(kThreads, Ring<BN>::kCtas)
    narrow_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ Args a) {
  constexpr int kStages = Ring<BN>::kStages, kStage = Ring<BN>::kStage, kMine = BN / 2, kTurns = BN / kHand;
  extern __shared__ uint8_t raw[];
  __shared__ __align__(8) uint64_t bars[2 * kStages + 5];
  __shared__ __align__(16) float hand[kHand * kHandPad];
  __shared__ uint32_t tmem_at;
  __shared__ int dead_flag;
  uint8_t* ring = raw + ((1024 - (smem_address(raw) & 1023)) & 1023);
  volatile int* dead = &dead_flag;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t full = smem_address(bars), empty = full + 8 * kStages, sums_full = empty + 8 * kStages, sums_empty = sums_full + 16,
                 drained = sums_empty + 16;
  const int chunks = a.chunks;

  if (warp == kLoad && lane == 0) {
    dead_flag = 0;
    for (int s = 0; s < kStages; ++s) {
      bar_init(full + 8 * s, 1);
      bar_init(empty + 8 * s, 1);
    }
    bar_init(drained, 1);
    for (int b = 0; b < 2; ++b) {
      bar_init(sums_full + 8 * b, 1);
      bar_init(sums_empty + 8 * b, kWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  if (warp == kMultiply) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_address(&tmem_at)), "r"(2 * BN)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    fence_before();
  }
  __syncthreads();
  fence_after();
  const uint32_t tmem = tmem_at;

  if (warp == kLoad && lane == 0) {
    uint32_t n = 0;
    bool ok = true;
    for (int64_t tile = blockIdx.x; ok && tile < a.tiles; tile += gridDim.x)
      for (int k = 0; k < a.slices; ++k, ++n) {
        const uint32_t s = n % kStages;
        ok = bar_wait(empty + 8 * s, (n / kStages + 1) & 1, dead, a.errors);
        if (!ok) break;
        const uint32_t bar = full + 8 * s, to = smem_address(ring) + s * kStage;
        bar_expect(bar, kStage);
        tma_load(to, &map_w, k * kBK, (int)(tile * kBM), bar);
        tma_load(to + kBytesRows, &map_x, k * kBK, 0, bar);
      }
    if (!ok)  // copies in flight land before the CTA ends
      for (uint32_t s = 0; s < kStages && s < n; ++s) {
        const uint32_t last = n - 1 - s;
        bar_drain(full + 8 * (last % kStages), last / kStages & 1);
      }
  } else if (warp == kMultiply && lane == 0) {
    constexpr uint32_t kInst = kInstruction<false, false, BN>;
    uint32_t n = 0, made = 0;
    bool ok = true;
    for (int64_t tile = blockIdx.x; ok && tile < a.tiles; tile += gridDim.x)
      for (int c = 0; ok && c < chunks; ++c, ++made) {
        const uint32_t half = made & 1, sums = tmem + half * BN;
        ok = bar_wait(sums_empty + 8 * half, (made / 2 + 1) & 1, dead, a.errors);
        if (!ok) break;
        fence_after();
        const int end = min(a.chunk, a.slices - c * a.chunk);
        for (int k = 0; k < end; ++k, ++n) {
          const uint32_t s = n % kStages;
          ok = bar_wait(full + 8 * s, n / kStages & 1, dead, a.errors);
          if (!ok) break;
          fence_after();
          const uint32_t at = smem_address(ring) + s * kStage;
          const uint64_t da = descriptor<false>(at), db = descriptor<false>(at + kBytesRows);
#pragma unroll
          for (int t = 0; t < kBK / 16; ++t) mma(sums, da + t * kStep16<false>, db + t * kStep16<false>, kInst, k > 0 || t > 0);
          mma_commit(empty + 8 * s);
        }
        if (ok) mma_commit(sums_full + 8 * half);
      }
    if (!ok) {  // products in flight end before the CTA does
      mma_commit(drained);
      bar_drain(drained, 0);
    }
  } else if (warp < kWarps) {
    const int quarter = warp % 4, side = warp / 4;  // 32 of the tile's words; half of the rows
    const int mine = threadIdx.x / 8, part = threadIdx.x % 8;  // of the rows that change hands; of their words, 16
    float m[kTurns], s[kTurns];
    int64_t target[kTurns];
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
      // turn t hands over rows 16 t .. 16 t + 15 of either side
      const int64_t row = mine / 16 * kMine + 16 * t + mine % 16;
      m[t] = -INFINITY, s[t] = 0.0f;
      target[t] = row < a.p.rows ? a.p.targets[row] - a.p.first_col : -1;
    }
    uint32_t made = 0;
    bool ok = true;
    for (int64_t tile = blockIdx.x; ok && tile < a.tiles; tile += gridDim.x) {
      float v[kMine];
#pragma unroll
      for (int t = 0; t < kMine; ++t) v[t] = 0.0f;
      for (int c = 0; c < chunks; ++c, ++made) {
        const uint32_t half = made & 1, sums = tmem + half * BN + side * kMine + ((uint32_t)(32 * quarter) << 16);
        ok = bar_wait_warp(sums_full + 8 * half, made / 2 & 1, dead, a.errors);
        if (!ok) break;
        fence_after();
#pragma unroll
        for (int b = 0; b < kMine / 16; ++b) add16(sums + 16 * b, v + 16 * b);
        fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(sums_empty + 8 * half);
      }
      ok = all_go_on<32 * kWarps>(ok);
      if (!ok) break;
#pragma unroll
      for (int t = 0; t < kTurns; ++t) {
        if (t > 0) asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory");  // the last rows have been read
#pragma unroll
        for (int i = 0; i < 16; ++i) hand[(16 * side + i) * kHandPad + 32 * quarter + lane] = v[16 * t + i];
        asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory");
        float x[16];
        const float4* from = reinterpret_cast<const float4*>(hand + mine * kHandPad + 16 * part);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 f = from[i];
          x[4 * i] = f.x, x[4 * i + 1] = f.y, x[4 * i + 2] = f.z, x[4 * i + 3] = f.w;
        }
        const int64_t col = tile * kBM + 16 * part;
        const int count = (int)max((int64_t)0, min((int64_t)16, a.p.cols - col));
        const int64_t at = target[t] - col;
        if (at >= 0 && at < count) a.p.picked[mine / 16 * kMine + 16 * t + mine % 16] = pick<16>(x, (int)at);
        float m2, s2;
        reduce<16>(x, count, m2, s2);
        join(m[t], s[t], m2, s2);
      }
      asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory");
    }
    if (ok) {
#pragma unroll
      for (int t = 0; t < kTurns; ++t) {
#pragma unroll
        for (int d = 1; d < 8; d *= 2) {
          const float m2 = __shfl_xor_sync(0xFFFFFFFFu, m[t], d), s2 = __shfl_xor_sync(0xFFFFFFFFu, s[t], d);
          join(m[t], s[t], m2, s2);
        }
        const int64_t row = mine / 16 * kMine + 16 * t + mine % 16;
        if (part == 0 && row < a.p.rows) a.p.partials[(int64_t)blockIdx.x * a.p.rows + row] = make_float2(m[t], s[t]);
      }
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  if (warp == kMultiply) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * BN));
}

// ---- host side ----

struct Plan {
  int64_t tiles_r, tiles_c, ctas, slots;
  int width;
};

template <int BN>
cudaError_t plan_narrow(const Logits& p, int sms, Plan* plan) {
  static std::atomic<uint64_t> allowed;
  const cudaError_t e = allow_shared(narrow_kernel<BN>, Ring<BN>::kBytes, allowed);
  const int64_t tiles = (p.cols + kBM - 1) / kBM, room = (int64_t)Ring<BN>::kCtas * sms;
  const int64_t ctas = tiles < room ? tiles : room;
  *plan = {1, tiles, ctas, ctas, BN};
  return e;
}

// The width by an estimate of the time, as plan_pair of the linear layers has it.
cudaError_t plan_wide(const Logits& p, Plan* plan) {
  static std::atomic<uint64_t> allowed;
  static std::atomic<int> clusters[64][9];
  const cudaError_t e = allow_shared(wide_kernel, kWideBytes, allowed);
  if (e != cudaSuccess) return e;
  const int64_t at_once = clusters_at_once(wide_kernel, 2, kWideThreads, kWideBytes, clusters);
  const int64_t tiles_r = (p.rows + kWideRows - 1) / kWideRows, slices = (p.k + kBK - 1) / kBK;
  double least = 0;
  Plan best = {};
  for (int width = 256; width >= 64; width -= 64) {
    const int64_t tiles_c = (p.cols + width - 1) / width, tiles = tiles_r * tiles_c;
    const double rounds = (double)((tiles + at_once - 1) / at_once);
    const double slice = 2.0 * width > 256.0 + width ? 2.0 * width : 256.0 + width;
    const double products = slices * slice, finish = 16.0 * width;
    const double time = rounds * (products > finish ? products : finish) + finish + 400.0 * rounds;
    if (best.width == 0 || time < least) {
      least = time;
      best = {tiles_r, tiles_c, 2 * (tiles < at_once ? tiles : at_once), tiles_c, width};
    }
  }
  *plan = best;
  return cudaSuccess;
}

cudaError_t plan_of(const Logits& p, int sms, Plan* plan) {
  if (p.rows <= 32) return plan_narrow<32>(p, sms, plan);
  if (p.rows <= 64) return plan_narrow<64>(p, sms, plan);
  if (p.rows <= 128) return plan_narrow<128>(p, sms, plan);
  return plan_wide(p, plan);
}

}  // namespace

cudaError_t logit_slots(const Logits& p, int sms, int64_t* slots) {
  Plan g = {};
  const cudaError_t e = plan_of(p, sms, &g);
  *slots = g.slots;
  return e;
}

cudaError_t launch_logits(const Logits& p, int sms, cudaStream_t s) {
  Plan g = {};
  cudaError_t e = plan_of(p, sms, &g);
  Args a = {};
  a.p = p;
  a.tiles_r = g.tiles_r, a.tiles_c = g.tiles_c, a.tiles = g.tiles_r * g.tiles_c;
  a.slices = (int)((p.k + kBK - 1) / kBK), a.width = g.width;
  const int parts = std::max((a.slices + kChunk - 1) / kChunk, std::min(a.slices, kLeastChunks));
  a.chunk = parts ? (a.slices + parts - 1) / parts : 0;
  a.chunks = parts ? (a.slices + a.chunk - 1) / a.chunk : 0;
  if (e == cudaSuccess) e = error_word(&a.errors);
  if (e != cudaSuccess) return e;
  const bool wide = p.rows > 128;
  CUtensorMap mx = {}, mw = {};  // not read where the sum is over nothing
  if (p.k > 0 && !(encode(&mx, p.x, p.k, p.rows, p.ldx, wide ? kBM : g.width) &&
                   encode(&mw, p.w, p.k, p.cols, p.ldw, wide ? g.width / 2 : kBM)))
    return cudaErrorNotSupported;
  if (wide) return launch(wide_kernel, g.ctas, 2, kWideThreads, kWideBytes, s, mx, mw, a);
  if (g.width == 32) return launch(narrow_kernel<32>, g.ctas, 1, kThreads, Ring<32>::kBytes, s, mx, mw, a);
  if (g.width == 64) return launch(narrow_kernel<64>, g.ctas, 1, kThreads, Ring<64>::kBytes, s, mx, mw, a);
  return launch(narrow_kernel<128>, g.ctas, 1, kThreads, Ring<128>::kBytes, s, mx, mw, a);
}

}  // namespace loss
}  // namespace smat
