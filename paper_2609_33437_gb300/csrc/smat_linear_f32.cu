// The linear layers' products of fp32 matrices, to fp32 accuracy (smat_linear.h, Product; include/smat.h).
//
// Large ones run on the tensor cores. A first kernel cuts every fp32 value into three bf16 values, hi + mid + lo, each the
// nearest to what is left: exactly the value (from 2^-110 on; below, lo's last bits fall under bf16's smallest number, 2^-133).
// mid is at most 2^-8 and lo 2^-17 of the value's power of two (twice that next to the largest fp32 number), so the three of
// nine products that are left out, mid lo, lo mid and lo lo, are below 2^-24 (1 + 2^-9) of the whole, like one rounding, and of
// either sign. The product then is the other six, for a slice of 64 of the sum at a time and the small ones first, so that what
// an addition in tensor memory cuts off is cut off sums that are small yet (the last four additions of a slice cut off up to 2^-23 of it each); eight warps add the
// slices' sums in registers, rounding to nearest. Measured: 4096 x 4096 x 4096 576 us, 239 TFLOP/s of fp32 products where the
// fp32 units reach 75 at most; 515 x 896 x 4864 37 us, 10 of them to cut 19 MB, the rest bound by the copies into shared memory
// (110 KB for 1,920 cycles of multiplications). Its error against 64 bits there is 1.5e-7, a plain fp32 product's 6.2e-7.
//
// An infinity times a part that is 0 would give NaN, and the parts of an operand whose largest value is below 2^-86 miss bits
// that matter. So the first kernel says what it met, and in those cases the second one makes its tiles on the fp32 units
// instead. (Beside larger values those below 2^-110 are off by up to 2^-134.)
//
// Products of at most 16 rows read a weight once and wait for it: rows_kernel multiplies it as it comes, in registers.
//
// Other small ones run on the fp32 units too: the cutting would cost more than it gains. A CTA of 256 threads makes a
// tile of BM x 128 sums, BM / 16 x 8 of them in each thread's registers as packed pairs (one instruction multiplies and
// adds two). Slices along l go through shared memory, the next one loaded to registers while one is multiplied. Where the
// tiles are fewer than the SMs, l is cut among the CTAs of a cluster; each leaves its
// sums in its own shared memory and then adds up and finishes its share of the rows, in the cluster's order: no atomics,
// the same result every time.

#include "smat_linear.h"
#include "smat_linear_tc.cuh"

namespace smat {
namespace lin {
namespace {

constexpr int kUnits = 256;  // threads that make a tile on the fp32 units
constexpr int kBN = 128, kPad = 4;
// Slices along the sum: what is on its way from memory per CTA. Tiles of 32 rows wait for it, so theirs are long
// (100 x 200 x 300: 11.3 us, with tiles of 128 rows and slices of 16 17.7).
template <int BM>
constexpr int kSimtK = BM == 32 ? 64 : 16;

// In shared memory four neighbours of a slice [K][R + kPad] lie at a place that changes with every four rows, so that the
// stores of a slice that arrives along the sum meet in few banks.
__device__ __forceinline__ int place(int k, int i) { return i ^ ((k >> 2 & 7) << 2); }

// A barrier of the first kUnits threads (both kernels' warps 0 to 7).
__device__ __forceinline__ void units_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

struct Args {
  Product p;
  bool va, vb;    // operands whose rows may be read 16 bytes at a time
  bool vr, vo;    // residual, out likewise
  int64_t share;  // of the sum, per CTA of a cluster
};

// four values of a row, `count` of them there
__device__ __forceinline__ float4 load4(const float* p, int64_t count, bool vec) {
  if (vec && count >= 4) return *reinterpret_cast<const float4*>(p);
  return make_float4(count > 0 ? p[0] : 0.0f, count > 1 ? p[1] : 0.0f, count > 2 ? p[2] : 0.0f, count > 3 ? p[3] : 0.0f);
}

// One operand's slice [R][K] into registers, then into shared memory as [K][R + kPad].
template <int R, bool MN, int K>
struct Slice {
  static constexpr int kVecs = R * K / 4, kSteps = (kVecs + kUnits - 1) / kUnits;
  float4 v[kSteps];

  __device__ __forceinline__ void load(const float* p, int64_t ld, int64_t first, int64_t end, int64_t l, int64_t l_end,
                                       bool vec) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int at = threadIdx.x + s * kUnits;
      v[s] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (kVecs % kUnits && at >= kVecs) continue;
      if (MN) {
        const int64_t k = l + at / (R / 4), i = first + at % (R / 4) * 4;
        if (k < l_end) v[s] = load4(p + k * ld + i, end - i, vec);
      } else {
        const int64_t i = first + at / (K / 4), k = l + at % (K / 4) * 4;
        if (i < end) v[s] = load4(p + i * ld + k, l_end - k, vec);
      }
    }
  }

  __device__ __forceinline__ void store(float (*to)[R + kPad]) const {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int at = threadIdx.x + s * kUnits;
      if (kVecs % kUnits && at >= kVecs) continue;
      if (MN) {
        const int k = at / (R / 4);
        *reinterpret_cast<float4*>(&to[k][place(k, at % (R / 4) * 4)]) = v[s];
      } else {
        const int k = at % (K / 4) * 4, i = place(k, at / (K / 4));
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

__device__ __forceinline__ void store4(float* p, int64_t count, bool vec, const float (&v)[4]) {
  if (vec && count >= 4) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < count) p[i] = v[i];
}

// Four sums (i, j .. j + 3) to what the call returns. The 8 lanes that share a group of 32 columns call it together.
__device__ __forceinline__ void finish4(const Args& a, int64_t i, int64_t j, float (&v)[4]) {
  const Product& p = a.p;
  const int64_t count = i < p.I ? p.J - j : 0;
  float* out = (float*)p.out + i * p.ldo + j;
  if (p.mode == kForward) {
    if (p.bias) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (t < count) v[t] += ((const float*)p.bias)[j + t];
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
    SMAT_WITH_ACT(p.act, _Pragma("unroll") for (int t = 0; t < 4; ++t) v[t] = act_value<ACT, float>(v[t]))
    if (p.residual) {
      const float4 r = load4((const float*)p.residual + i * p.ldr + j, count, a.vr);
      v[0] += r.x, v[1] += r.y, v[2] += r.z, v[3] += r.w;
    }
  } else {
    if (count <= 0) return;
    if (p.mode == kGradInput && p.act != SMAT_ACT_NONE) {
      const float scale = unpack_scale(p.e[i * p.lde + j / kGroup]);
      SMAT_WITH_ACT(p.act, _Pragma("unroll") for (int t = 0; t < 4; ++t) if (t < count) v[t] *=
                    act_slope<ACT, float>((float)p.q[i * p.ldq + j + t] * scale))
    }
    if (p.accumulate) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (t < count) v[t] += out[t];
    }
  }
  store4(out, count, a.vo, v);
}

// ------------------------------------------------------------- fp32 units ---

template <int BM>
constexpr int kSlicesBytes = 2 * kSimtK<BM> * (BM + kPad + kBN + kPad) * 4;
template <int BM>
constexpr int kSimtBytes = kSlicesBytes<BM> > BM * kBN * 4 ? kSlicesBytes<BM> : BM * kBN * 4;

// The sums of BM x 128 from (i0, j0) over l0 .. l1, left in `shared` as [BM][128]; threads 0 to 255.
template <int BM, bool A_MN, bool B_MN>
__device__ __forceinline__ void simt_sums(const Args& a, float* shared, int64_t i0, int64_t j0, int64_t l0, int64_t l1) {
  constexpr int TM = BM / 16, K = kSimtK<BM>;  // consecutive rows per thread; a slice
  static_assert(TM == 8 || TM == 2, "");
  float (*sa)[K][BM + kPad] = reinterpret_cast<float (*)[K][BM + kPad]>(shared);
  float (*sb)[K][kBN + kPad] = reinterpret_cast<float (*)[K][kBN + kPad]>(shared + 2 * K * (BM + kPad));
  float (*sums)[kBN] = reinterpret_cast<float (*)[kBN]>(shared);  // afterwards

  const Product& p = a.p;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  uint64_t acc[TM][4];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0;

  Slice<BM, A_MN, K> na;
  Slice<kBN, B_MN, K> nb;
  const float *pa = (const float*)p.a, *pb = (const float*)p.b;
  if (l0 < l1) {
    na.load(pa, p.lda, i0, p.I, l0, l1, a.va);
    nb.load(pb, p.ldb, j0, p.J, l0, l1, a.vb);
    na.store(sa[0]);
    nb.store(sb[0]);
  }
  units_sync();
  int at = 0;
  for (int64_t l = l0; l < l1; l += K, at ^= 1) {
    const bool more = l + K < l1;
    if (more) {
      na.load(pa, p.lda, i0, p.I, l + K, l1, a.va);
      nb.load(pb, p.ldb, j0, p.J, l + K, l1, a.vb);
    }
#pragma unroll 16
    for (int k = 0; k < K; ++k) {
      const ulonglong2 b01 = *reinterpret_cast<const ulonglong2*>(&sb[at][k][place(k, tx * 4)]);
      const ulonglong2 b23 = *reinterpret_cast<const ulonglong2*>(&sb[at][k][place(k, 64 + tx * 4)]);
      float x[TM];
      if constexpr (TM == 8) {
        *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(&sa[at][k][place(k, ty * TM)]);
        *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(&sa[at][k][place(k, ty * TM + 4)]);
      } else {
        *reinterpret_cast<float2*>(x) = *reinterpret_cast<const float2*>(&sa[at][k][place(k, ty * TM)]);
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
    units_sync();
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    *reinterpret_cast<ulonglong2*>(&sums[ty * TM + i][tx * 4]) = make_ulonglong2(acc[i][0], acc[i][1]);
    *reinterpret_cast<ulonglong2*>(&sums[ty * TM + i][64 + tx * 4]) = make_ulonglong2(acc[i][2], acc[i][3]);
  }
}

template <int BM, bool A_MN, bool B_MN>
__global__ void __launch_bounds__(kUnits, 2) simt_kernel(const Args a) {
  extern __shared__ __align__(16) float shared[];
  const Product& p = a.p;
  const int64_t i0 = (int64_t)blockIdx.x * BM, j0 = (int64_t)blockIdx.y * kBN;
  const int64_t l0 = (int64_t)blockIdx.z * a.share, l1 = l0 + a.share < p.L ? l0 + a.share : p.L;
  simt_sums<BM, A_MN, B_MN>(a, shared, i0, j0, l0, l1);
  const int shares = gridDim.z;
  if (shares > 1)
    cluster_sync();
  else
    __syncthreads();
  // the rows go around among the CTAs of the cluster and their warps; a warp finishes a row of 128
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  for (int row = (int)blockIdx.z * 8 + warp; row < BM && i0 + row < p.I; row += 8 * shares) {
    const float* at = shared + row * kBN + lane * 4;
    float v[4] = {};
    if (shares == 1) {
      const float4 t = *reinterpret_cast<const float4*>(at);
      v[0] = t.x, v[1] = t.y, v[2] = t.z, v[3] = t.w;
    } else {
      for (int s = 0; s < shares; ++s) {
        const float4 t = cluster_load4(cluster_address(at, (uint32_t)s));
        v[0] += t.x, v[1] += t.y, v[2] += t.z, v[3] += t.w;
      }
    }
    finish4(a, i0 + row, j0 + lane * 4, v);
  }
  if (shares > 1) cluster_sync();  // nobody leaves while its sums are read
}

// ----------------------------------------------------------------- few rows ---

// Column j of rows i .. i + N - 1 to what the call returns; the warp holds 32 neighbouring columns from a multiple of 32 on.
// What the rows read is asked for first, all of it.
template <int N>
__device__ __forceinline__ void finish_column(const Args& a, int64_t i, int64_t j, float (&v)[N]) {
  const Product& p = a.p;
  if (i >= p.I) return;
  const bool there = j < p.J;
  const int mine = there ? (int)(p.I - i < N ? p.I - i : N) : 0;
  float* out = (float*)p.out + i * p.ldo + j;
  const bool forward = p.mode == kForward, slope = p.mode == kGradInput && p.act != SMAT_ACT_NONE;
  const float* from = forward ? (const float*)p.residual : p.accumulate ? (const float*)p.out : nullptr;
  const int64_t ld = forward ? p.ldr : p.ldo;
  float x[N];
  if (from) {
#pragma unroll
    for (int t = 0; t < N; ++t) x[t] = t < mine ? from[(i + t) * ld + j] : 0.0f;
  }
  if (slope) {
    int qs[N];
    uint32_t es[N];
#pragma unroll
    for (int t = 0; t < N; ++t) {
      qs[t] = t < mine ? p.q[(i + t) * p.ldq + j] : 0;
      es[t] = t < mine ? p.e[(i + t) * p.lde + j / kGroup] : 0;
    }
#pragma unroll
    for (int t = 0; t < N; ++t) x[t] = (float)qs[t] * unpack_scale(es[t]);
    SMAT_WITH_ACT(p.act, _Pragma("unroll") for (int t = 0; t < N; ++t) v[t] *= act_slope<ACT, float>(x[t]))
  }
  if (forward) {
    const float bias = p.bias && there ? ((const float*)p.bias)[j] : 0.0f;
#pragma unroll
    for (int t = 0; t < N; ++t) v[t] += bias;
    if (p.q) {
#pragma unroll
      for (int t = 0; t < N; ++t) {
        const uint32_t ex = pack_exponent(__reduce_max_sync(0xFFFFFFFFu, there ? __float_as_uint(fabsf(v[t])) : 0u));
        if (t < mine) {
          p.q[(i + t) * p.ldq + j] = (int8_t)pack_one(v[t], ex);
          if (j % kGroup == 0) p.e[(i + t) * p.lde + j / kGroup] = (uint8_t)ex;
        }
      }
    }
    SMAT_WITH_ACT(p.act, _Pragma("unroll") for (int t = 0; t < N; ++t) v[t] = act_value<ACT, float>(v[t]))
  }
  if (from) {
#pragma unroll
    for (int t = 0; t < N; ++t) v[t] += x[t];
  }
#pragma unroll
  for (int t = 0; t < N; ++t)
    if (t < mine) out[t * p.ldo] = v[t];
}

constexpr int kRowWarps = 8;
// Rows up to which it is taken. 4096 x 4096 with a weight that is not in L2, forward and back: one row 14.0 and 15.3 us (4.8
// and 4.4 TB/s; on the fp32 units' tiles 52 and 49), 16 rows 38 and 31 us (cut for the tensor cores 54 and 52). With other
// operands every call 8 rows of a 4864 x 896 weight take 11.2 and 25.7 us (24.6 and 36.4 otherwise), of 11008 x 4096 100 and 67
// (149 and 130), of 1024 x 1024 5.3 and 9.8 (10.2 and 10.1); 16 rows 12.8 and 30.7 (20.2 and 25.6), 125 and 74 (149 and 130),
// 5.7 and 10.8 (10.4 and 10.0). So back through smaller weights it is the slower one towards 16 rows, by 8 to 20%, and through
// 256 x 256 from 8 rows on (8.9 and 6.4): forward it is the faster one at all of these.
constexpr int kFewRows = 16;

// A product of at most R rows with a weight that is read once, where the copies bound it (rows 1 of 4096 x 4096: 67 MB).
// The sum is cut among the CTAs of a cluster; each leaves its share in shared memory, the cluster adds the shares in order.
//
// Forward: y(i, j) sums along W's row j. A CTA has 32 rows of W, a warp four of them; a lane multiplies 4 neighbours of
// each with those of every row of x, which the warps share, and the lanes' sums are added at the end.
// grad_input: dx(i, j) sums down W's column j. A CTA has 128 columns, a lane four neighbours; its warps take every eighth
// row of W, whose factors dy(i, l) are the same for all lanes, and their sums are added at the end.
template <int MODE, int R, bool VEC>
__global__ void __launch_bounds__(32 * kRowWarps, 2) rows_kernel(const Args a) {
  constexpr int kCols = MODE == kForward ? 32 : 128;  // of the result, per CTA
  constexpr int kWays = 4, kAtOnce = R < 8 ? R : 8;  // how the warps' sums of grad_input meet, see below
  constexpr int kChunk = 256, kFactorRow = R < 4 ? 4 : R + (R > 4 ? 4 : 0);
  constexpr int kSpace = kWays * kAtOnce * kCols > kChunk * kFactorRow ? kWays * kAtOnce * kCols : kChunk * kFactorRow;
  __shared__ __align__(16) float share[R][kCols];
  __shared__ __align__(16) float space[MODE == kForward ? R * kChunk : kSpace];
  const Product& p = a.p;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int64_t j0 = (int64_t)blockIdx.x * kCols;
  const int64_t l0 = (int64_t)blockIdx.y * a.share, l1 = l0 + a.share < p.L ? l0 + a.share : p.L;
  const float *x = (const float*)p.a, *w = (const float*)p.b;
  uint32_t shares;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(shares));

  float acc[R][4];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int t = 0; t < 4; ++t) acc[i][t] = 0.0f;

  if constexpr (MODE == kForward) {
    const int64_t j = j0 + 4 * warp;
    if constexpr (R == 1) {  // x from L1: 7.7 us for 4096 x 4096 in L2, through shared memory 12.4
#pragma unroll 2
      for (int64_t l = l0 + 4 * lane; l < l1; l += 128) {
        float4 b[4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
          b[t] = j + t < p.J ? load4(w + (j + t) * p.ldb + l, l1 - l, VEC) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        const float4 f = load4(x + l, l1 - l, VEC);
#pragma unroll
        for (int t = 0; t < 4; ++t)
          acc[0][t] = fmaf(f.x, b[t].x, fmaf(f.y, b[t].y, fmaf(f.z, b[t].z, fmaf(f.w, b[t].w, acc[0][t]))));
      }
    }
    float (*rows)[kChunk] = reinterpret_cast<float (*)[kChunk]>(space);  // of x
    for (int64_t c0 = R == 1 ? l1 : l0; c0 < l1; c0 += kChunk) {
      // W's values first: they are on their way while x is put down
      float4 b[kChunk / 128][4];
#pragma unroll
      for (int h = 0; h < kChunk / 128; ++h)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int64_t l = c0 + 128 * h + 4 * lane;
          b[h][t] = j + t < p.J ? load4(w + (j + t) * p.ldb + l, l1 - l, VEC) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
      __syncthreads();
#pragma unroll 4
      for (int at = threadIdx.x; at < R * kChunk / 4; at += 32 * kRowWarps) {
        const int i = at / (kChunk / 4), n = at % (kChunk / 4) * 4;
        *reinterpret_cast<float4*>(&rows[i][n]) =
            i < p.I ? load4(x + i * p.lda + c0 + n, l1 - c0 - n, VEC) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      }
      __syncthreads();
#pragma unroll
      for (int h = 0; h < kChunk / 128; ++h)
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const float4 f = *reinterpret_cast<const float4*>(&rows[i][128 * h + 4 * lane]);
#pragma unroll
          for (int t = 0; t < 4; ++t)
            acc[i][t] = fmaf(f.x, b[h][t].x, fmaf(f.y, b[h][t].y, fmaf(f.z, b[h][t].z, fmaf(f.w, b[h][t].w, acc[i][t]))));
        }
    }
    // the lanes' sums: kSums at a time, each step halves what a lane still holds
    constexpr int kSums = 4 * R < 32 ? 4 * R : 32;
#pragma unroll
    for (int i0 = 0; i0 < R; i0 += kSums / 4) {
      float v[kSums];
#pragma unroll
      for (int t = 0; t < kSums; ++t) v[t] = acc[i0 + t / 4][t % 4];
#pragma unroll
      for (int d = 16; d >= kSums; d /= 2)
#pragma unroll
        for (int t = 0; t < kSums; ++t) v[t] += __shfl_xor_sync(0xFFFFFFFFu, v[t], d);
#pragma unroll
      for (int d = kSums / 2; d > 0; d /= 2) {
        const bool high = lane & d;
#pragma unroll
        for (int t = 0; t < d; ++t) {
          const float give = high ? v[t] : v[t + d], keep = high ? v[t + d] : v[t];
          v[t] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, d);
        }
      }
      if (lane < kSums) share[i0 + lane / 4][4 * warp + lane % 4] = v[0];
    }
  } else {
    const int64_t j = j0 + 4 * lane;
    constexpr int kAhead = 8;  // rows of W in flight per warp
    static_assert(kChunk % (kAhead * kRowWarps) == 0, "a step stays inside a chunk");
    // factors of kChunk rows of W, [row of W][row of dy]
    float (*factor)[kFactorRow] = reinterpret_cast<float (*)[kFactorRow]>(space);
    for (int64_t c0 = l0; c0 < l1; c0 += kChunk) {
      const int rows = (int)(l1 - c0 < kChunk ? l1 - c0 : kChunk);
      __syncthreads();
      for (int at = threadIdx.x; at < R * kChunk; at += 32 * kRowWarps) {
        const int i = at / kChunk, n = at % kChunk;
        factor[n][i] = i < p.I && n < rows ? x[i * p.lda + c0 + n] : 0.0f;
      }
      __syncthreads();
      for (int n0 = warp; n0 < rows; n0 += kAhead * kRowWarps) {
        float4 b[kAhead];
#pragma unroll
        for (int h = 0; h < kAhead; ++h) {
          const int n = n0 + h * kRowWarps;
          b[h] = n < rows ? load4(w + (c0 + n) * p.ldb + j, p.J - j, VEC) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
#pragma unroll
        for (int h = 0; h < kAhead; ++h) {
          const int n = n0 + h * kRowWarps;  // below kChunk, of whose steps it is a whole number; past the rows 0 times 0
          float f[R < 4 ? 4 : R];
#pragma unroll
          for (int i = 0; i < R; i += 4) *reinterpret_cast<float4*>(f + i) = *reinterpret_cast<const float4*>(&factor[n][i]);
#pragma unroll
          for (int i = 0; i < R; ++i) {
            acc[i][0] = fmaf(f[i], b[h].x, acc[i][0]), acc[i][1] = fmaf(f[i], b[h].y, acc[i][1]);
            acc[i][2] = fmaf(f[i], b[h].z, acc[i][2]), acc[i][3] = fmaf(f[i], b[h].w, acc[i][3]);
          }
        }
      }
    }
    float (*more)[kAtOnce][kCols] = reinterpret_cast<float (*)[kAtOnce][kCols]>(space);
    // the warps' sums, up to 8 rows at a time: a first half of the warps leaves its sums, the other adds its own; then
    // they are added up in order
#pragma unroll
    for (int i0 = 0; i0 < R; i0 += kAtOnce) {
      __syncthreads();
      if (warp < kWays)
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
          *reinterpret_cast<float4*>(&more[warp][i][4 * lane]) =
              make_float4(acc[i0 + i][0], acc[i0 + i][1], acc[i0 + i][2], acc[i0 + i][3]);
      __syncthreads();
      if (warp >= kWays)
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          float4* at = reinterpret_cast<float4*>(&more[warp - kWays][i][4 * lane]);
          const float4 t = *at;
          *at = make_float4(t.x + acc[i0 + i][0], t.y + acc[i0 + i][1], t.z + acc[i0 + i][2], t.w + acc[i0 + i][3]);
        }
      __syncthreads();
      for (int at = threadIdx.x; at < kAtOnce * kCols; at += 32 * kRowWarps) {
        float v = 0.0f;
#pragma unroll
        for (int h = 0; h < kWays; ++h) v += more[h][at / kCols][at % kCols];
        share[i0 + at / kCols][at % kCols] = v;
      }
    }
  }
  if (shares > 1)
    cluster_sync();
  else
    __syncthreads();
  // blocks of 32 columns of a row go around among the cluster's CTAs and their warps
  constexpr int kBlocks = kCols / 32;
  for (int at = (int)blockIdx.y * kRowWarps + warp; at < (int)p.I * kBlocks; at += (int)shares * kRowWarps) {
    const int i = at / kBlocks, c = at % kBlocks * 32 + lane;
    float v[1] = {0.0f};
    if (shares == 1) {
      v[0] = share[i][c];
    } else {
#pragma unroll 8
      for (uint32_t s = 0; s < shares; ++s) v[0] += cluster_load(&share[i][c], s);
    }
    finish_column(a, i, j0 + c, v);
  }
  if (shares > 1) cluster_sync();  // nobody leaves while its sums are read
}

// ------------------------------------------------------------ tensor cores ---

// A tile has 128 columns j of the result along tensor memory's rows and `width` of its rows i along the columns, 32 to 160:
// the sums of 160 take 80 registers of each of the 256 threads that add them up. A warp then holds 32 neighbouring columns of
// a row, 128 bytes.
constexpr int kPart = kBM * kBK * 2;  // a slice of one part of the operand along the tile's rows
constexpr int kMostWidth = 160, kStages = 2;
constexpr int kBlock = 16, kMostBlocks = kMostWidth / kBlock / 2;  // of a warp's sums
// a part of the columns' operand; 64 columns at a time, the last 64 reach past 160
constexpr int kMostPartB = kMostWidth * kBK * 2;
constexpr int kStage = kParts * (kPart + kMostPartB);
constexpr int kTcBytes = kStages * kStage + 1024;
constexpr int kSums = 256;  // columns of tensor memory apart
static_assert(kSimtBytes<128> <= kStages * kStage, "a tile on the fp32 units takes the ring's place");

// One operand to cut: fp32 [rows, cols] to parts [3][rows][ldp] of bf16.
struct Cut {
  const float* from;
  uint16_t* to;
  int64_t rows, cols, ld, ldp;
  bool vec;          // rows on 16 bytes
  const int* count;  // or NULL: on the device, the rows there are; those up to the next multiple of 64 are cut too
};

// Both operands of a product; flags[CTA]: flag_of what it met. A thread cuts 8 neighbours of a row: 32 bytes in, 3 x 16 out.
__global__ void __launch_bounds__(256) cut_kernel(const Cut a, const Cut b, int ctas_a, uint32_t* flags) {
  __shared__ uint32_t tops[8];
  const bool first = (int)blockIdx.x < ctas_a;
  const Cut& c = first ? a : b;
  const int64_t ctas = first ? ctas_a : gridDim.x - ctas_a, cta = first ? blockIdx.x : blockIdx.x - ctas_a;
  const int64_t units = c.ldp / 8, plane = c.rows * c.ldp;
  const int64_t rows = c.count ? min(c.rows, (*c.count + (int64_t)63) / 64 * 64) : c.rows;
  uint32_t top = 0;
  // a CTA's rows one after another, its threads side by side along a row (a short row's threads share out rows)
  const int wide = (int)(units < 256 ? units : 256), high = 256 / wide;
  const int tx = threadIdx.x % wide, ty = threadIdx.x / wide;
  if (ty < high)
    for (int64_t r = cta * high + ty; r < rows; r += ctas * high)
      for (int64_t u = tx; u < units; u += wide) {
        const int64_t at = 8 * u;
        const float* p = c.from + r * c.ld + at;
        const float4 x = load4(p, c.cols - at, c.vec), y = load4(p + 4, c.cols - at - 4, c.vec);
        const float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        uint32_t w[3][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          uint32_t parts[3];
          cut2(v[2 * t], v[2 * t + 1], parts, top);
          w[0][t] = parts[0], w[1][t] = parts[1], w[2][t] = parts[2];
        }
#pragma unroll
        for (int t = 0; t < 3; ++t)
          *reinterpret_cast<uint4*>(c.to + t * plane + r * c.ldp + at) = make_uint4(w[t][0], w[t][1], w[t][2], w[t][3]);
      }
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  if (threadIdx.x % 32 == 0) tops[threadIdx.x / 32] = top;
  __syncthreads();
  if (threadIdx.x < 8) {
    top = __reduce_max_sync(0xFFu, tops[threadIdx.x]);
    if (threadIdx.x == 0) flags[blockIdx.x] = flag_of(top);
  }
}

struct TcArgs {
  Args f;
  int64_t tiles, tiles_r, tiles_c;  // of 128 columns j, of `width` rows i
  int width;
  int slices, share;  // slices of 64, and those of a CTA of a cluster
  float* parts;       // shares of sums
  const uint32_t *flags_a, *flags_b;
  int n_flags_a, n_flags;  // of the first operand, of both
  int* errors;
};

// The six products of a slice, small ones first: (part of the rows' operand, part of the columns')
__device__ constexpr int kOrder[6][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};

// A: the operand of j (the product's b), B: that of i (its a). COUNTED: the rows i, or of a weight's gradient the terms of the sum,
// are those that the device counts (p.count).
template <bool A_MN, bool B_MN, bool COUNTED>
__global__ void __launch_bounds__(kThreads, 1)
    f32_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
               const __grid_constant__ TcArgs a) {
  extern __shared__ uint8_t raw[];
  __shared__ __align__(8) uint64_t bars[2 * kStages + 5];
  __shared__ uint32_t tmem_at, met_here[kThreads / 32];
  __shared__ int dead_flag;
  uint8_t* ring = raw + ((1024 - (smem_address(raw) & 1023)) & 1023);
  volatile int* dead = &dead_flag;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t full = smem_address(bars), empty = full + 8 * kStages, sums_full = empty + 8 * kStages,
                 sums_empty = sums_full + 16, drained = sums_empty + 16;
  const Product& p = a.f.p;

  uint32_t shares, rank;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(shares));
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  int64_t tiles_c = a.tiles_c, tiles = a.tiles, I = p.I, L = p.L;
  int slices_there = a.slices;
  if (COUNTED && A_MN && B_MN) {
    L = min(L, (int64_t)*p.count);
    slices_there = (int)((L + kBK - 1) / kBK);
  } else if (COUNTED) {
    I = min(I, (int64_t)*p.count);
    tiles_c = (I + a.width - 1) / a.width;
    tiles = a.tiles_r * tiles_c;
  }
  const int slice0 = (int)rank * a.share;
  const int slices = max(0, min(a.share, slices_there - slice0));
  const int64_t first_tile = blockIdx.x / shares, step = gridDim.x / shares;

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
  }
  __syncwarp();
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_address(&tmem_at)),
                 "r"(2 * kSums)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    fence_before();
  }
  uint32_t met = 0;  // the second operand's flags from bit 8 on
  for (int i = threadIdx.x; i < a.n_flags; i += kThreads) met |= i < a.n_flags_a ? a.flags_a[i] : a.flags_b[i - a.n_flags_a] << 8;
  met = __reduce_or_sync(0xFFFFFFFFu, met);
  if (lane == 0) met_here[warp] = met;
  __syncthreads();
  fence_after();
  const uint32_t tmem = tmem_at;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) met |= met_here[w];
  auto uncut = [](uint32_t f) { return (f & kOdd) || (f & (kSmall | kLarge)) == kSmall; };
  const bool odd = uncut(met) || uncut(met >> 8);

  if (odd) {
    // an operand whose parts do not stand for it: all CTAs make tiles of 128 x 128 on the fp32 units
    if (warp < kEpiWarps) {
      float* sums = reinterpret_cast<float*>(ring);
      const int64_t ti = (I + kBM - 1) / kBM, tj = (p.J + kBN - 1) / kBN;
      for (int64_t tile = blockIdx.x; tile < ti * tj; tile += gridDim.x) {
        const int64_t i0 = tile % ti * kBM, j0 = tile / ti * kBN;
        simt_sums<128, B_MN, A_MN>(a.f, sums, i0, j0, 0, L);
        units_sync();
        for (int row = warp; row < kBM && i0 + row < I; row += 8) {
          const float4 t = *reinterpret_cast<const float4*>(sums + row * kBN + lane * 4);
          float v[4] = {t.x, t.y, t.z, t.w};
          finish4(a.f, i0 + row, j0 + lane * 4, v);
        }
        units_sync();
      }
    }
  } else if (warp == kTmaWarp && lane == 0) {
    // a part of the columns' operand: rows of the tile's width, or 64 columns of it at a time
    const int blocks_b = B_MN ? (a.width + 63) / 64 : 1;
    const int part_b = B_MN ? blocks_b * 8192 : a.width * kBK * 2;
    uint32_t n = 0;
    bool ok = true;
    for (int64_t tile = first_tile; ok && tile < tiles; tile += step) {
      int64_t tr, tc;
      tile_place<16>(a.tiles_r, tiles_c, tile, tr, tc);
      const int r0 = (int)(tr * kBM), c0 = (int)(tc * a.width);
      for (int k = 0; k < slices; ++k, ++n) {
        const uint32_t s = n % kStages;
        ok = bar_wait(empty + 8 * s, (n / kStages + 1) & 1, dead, a.errors);
        if (!ok) break;
        const int l = (slice0 + k) * kBK;
        const uint32_t bar = full + 8 * s, to = smem_address(ring) + s * kStage;
        bar_expect(bar, kParts * (kPart + part_b));
#pragma unroll
        for (int q = 0; q < kParts; ++q) {
          const uint32_t to_a = to + q * kPart, to_b = to + kParts * kPart + q * kMostPartB;
          if (A_MN) {
            tma_load3(to_a, &map_a, r0, l, q, bar);
            tma_load3(to_a + 8192, &map_a, r0 + 64, l, q, bar);
          } else {
            tma_load3(to_a, &map_a, l, r0, q, bar);
          }
          if (B_MN) {
            for (int b = 0; b < blocks_b; ++b) tma_load3(to_b + 8192 * b, &map_b, c0 + 64 * b, l, q, bar);
          } else {
            tma_load3(to_b, &map_b, l, c0, q, bar);
          }
        }
      }
    }
    if (!ok)  // copies in flight land before the CTA ends
      for (uint32_t s = 0; s < kStages && s < n; ++s) {
        const uint32_t last = n - 1 - s;
        bar_drain(full + 8 * (last % kStages), last / kStages & 1);
      }
  } else if (warp == kMmaWarp && lane == 0) {
    const uint32_t inst = kInstruction<A_MN, B_MN, 0> | (uint32_t)(a.width >> 3) << 17;
    uint32_t n = 0;
    bool ok = true;
    for (int64_t tile = first_tile; ok && tile < tiles; tile += step)
      for (int k = 0; k < slices; ++k, ++n) {
        const uint32_t s = n % kStages, half = n & 1, sums = tmem + half * kSums;
        ok = bar_wait(sums_empty + 8 * half, (n / 2 + 1) & 1, dead, a.errors) &&
             bar_wait(full + 8 * s, n / kStages & 1, dead, a.errors);
        if (!ok) break;
        fence_after();
        const uint32_t at = smem_address(ring) + s * kStage;
#pragma unroll
        for (int o = 0; o < 6; ++o) {
          const uint64_t da = descriptor<A_MN>(at + kOrder[o][0] * kPart);
          const uint64_t db = descriptor<B_MN>(at + kParts * kPart + kOrder[o][1] * kMostPartB);
#pragma unroll
          for (int t = 0; t < kBK / 16; ++t)
            mma(sums, da + t * kStep16<A_MN>, db + t * kStep16<B_MN>, inst, o > 0 || t > 0);
        }
        mma_commit(empty + 8 * s);
        mma_commit(sums_full + 8 * half);
      }
    if (!ok) {  // products in flight end before the CTA does
      mma_commit(drained);
      bar_drain(drained, 0);
    }
  } else if (warp < kEpiWarps) {
    // this warp's sums: 32 rows and half the columns of the tile, 16 columns at a time
    const int quarter = warp % 4, blocks = a.width / kBlock / 2, first = warp / 4 * blocks;
    uint32_t n = 0;
    bool ok = true;
    for (int64_t tile = first_tile; ok && tile < tiles; tile += step) {
      int64_t tr, tc;
      tile_place<16>(a.tiles_r, tiles_c, tile, tr, tc);
      float acc[kMostBlocks][kBlock];
#pragma unroll
      for (int b = 0; b < kMostBlocks; ++b)
#pragma unroll
        for (int t = 0; t < kBlock; ++t) acc[b][t] = 0.0f;
      for (int k = 0; k < slices; ++k, ++n) {
        const uint32_t half = n & 1;
        ok = bar_wait_warp(sums_full + 8 * half, n / 2 & 1, dead, a.errors);
        if (!ok) break;
        fence_after();
#pragma unroll
        for (int b = 0; b < kMostBlocks; ++b)
          if (b < blocks) {
            float v[kBlock];
            take16(tmem + half * kSums + kBlock * (first + b) + ((uint32_t)(32 * quarter) << 16), v);
#pragma unroll
            for (int t = 0; t < kBlock; ++t) acc[b][t] += v[t];
          }
        fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(sums_empty + 8 * half);
      }
      const int64_t j = tr * kBM + 32 * quarter, i0 = tc * a.width;
      if (shares > 1) {
        float* part = a.parts + ((size_t)first_tile * shares + rank) * a.width * kBM + 32 * quarter + lane;
#pragma unroll
        for (int b = 0; b < kMostBlocks; ++b)
          if (b < blocks) put_part(part + kBlock * (first + b) * kBM, acc[b]);
      } else if (ok && j < p.J) {
        // one block's code for all, the next one's sums moved to its place: five copies of it are 30 KB, which come from
        // memory at a first call (515 x 896 x 4864 through silu with nothing in L2 46.8 us, as copies 61.6)
#pragma unroll 1
        for (int b = 0; b < blocks; ++b) {
          finish_column(a.f, i0 + kBlock * (first + b), j + lane, acc[0]);
#pragma unroll
          for (int n = 1; n < kMostBlocks; ++n)
#pragma unroll
            for (int t = 0; t < kBlock; ++t) acc[n - 1][t] = acc[n][t];
        }
      }
    }
  }
  __syncwarp();
  if (shares > 1) {
    __syncthreads();
    cluster_sync();
    if (!odd && warp < kEpiWarps && first_tile < tiles && !__any_sync(0xFFFFFFFFu, *dead)) {
      int64_t tr, tc;
      tile_place<16>(a.tiles_r, tiles_c, first_tile, tr, tc);
      const int quarter = warp % 4;
      const int64_t j = tr * kBM + 32 * quarter, i0 = tc * a.width;
      const float* part = a.parts + (size_t)first_tile * shares * a.width * kBM + 32 * quarter + lane;
      for (int b = (int)rank + (int)shares * (warp / 4); b < a.width / kBlock && i0 + kBlock * b < p.I && j < p.J;
           b += 2 * (int)shares) {
        float v[kBlock];
        add_parts(shares, v, [&](uint32_t s, int t) { return __ldcg(part + ((size_t)s * a.width + kBlock * b + t) * kBM); });
        finish_column(a.f, i0 + kBlock * b, j + lane, v);
      }
    }
    cluster_meet();
  }
  fence_before();
  __syncthreads();
  if (warp == kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * kSums));
}

// ------------------------------------------------------------- host side ---

bool can(const void* p, int64_t ld) { return (uintptr_t)p % 16 == 0 && ld % 4 == 0; }

Args args_of(const Product& p) {
  Args a = {};
  a.p = p;
  a.va = can(p.a, p.lda);
  a.vb = can(p.b, p.ldb);
  a.vr = can(p.residual, p.ldr);
  a.vo = can(p.out, p.ldo);
  return a;
}

cudaLaunchConfig_t config(dim3 grid, int threads, int bytes, dim3 cluster, cudaLaunchAttribute* at, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = s;
  at->id = cudaLaunchAttributeClusterDimension;
  at->val.clusterDim = {cluster.x, cluster.y, cluster.z};
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cfg;
}

template <int BM, bool A_MN, bool B_MN>
cudaError_t launch_simt_tile(Args a, int sms, cudaStream_t s) {
  static std::atomic<uint64_t> allowed;
  auto* f = simt_kernel<BM, A_MN, B_MN>;
  const cudaError_t e = allow_shared(f, kSimtBytes<BM>, allowed);
  if (e != cudaSuccess) return e;
  const int64_t ti = (a.p.I + BM - 1) / BM, tj = (a.p.J + kBN - 1) / kBN;
  int shares = 1;
  // two CTAs fit on an SM; a share is at least 64 long
  while (shares < 8 && ti * tj * shares * 2 <= 2 * sms && a.p.L >= (int64_t)shares * 2 * 64) shares *= 2;
  constexpr int K = kSimtK<BM>;
  a.share = (a.p.L + shares * K - 1) / (shares * K) * K;
  cudaLaunchAttribute at;
  const cudaLaunchConfig_t cfg = config(dim3((unsigned)ti, (unsigned)tj, (unsigned)shares), kUnits, kSimtBytes<BM>,
                                        dim3(1, 1, (unsigned)shares), &at, s);
  return cudaLaunchKernelEx(&cfg, f, a);
}

template <int MODE, int R, bool VEC>
cudaError_t launch_rows_as(Args a, int sms, cudaStream_t s) {
  constexpr int kCols = MODE == kForward ? 32 : 128;
  const int64_t tiles = (a.p.J + kCols - 1) / kCols;
  // four CTAs' worth of warps per SM, a share at least 256 long
  int shares = 1;
  while (shares < 8 && tiles * shares * 2 <= 4 * sms && a.p.L >= (int64_t)shares * 2 * 256) shares *= 2;
  a.share = (a.p.L + shares * 128 - 1) / (shares * 128) * 128;
  cudaLaunchAttribute at;
  const cudaLaunchConfig_t cfg = config(dim3((unsigned)tiles, (unsigned)shares), 32 * kRowWarps, 0,
                                        dim3(1, (unsigned)shares, 1), &at, s);
  return cudaLaunchKernelEx(&cfg, rows_kernel<MODE, R, VEC>, a);
}
template <int MODE, int R>
cudaError_t launch_rows_of(const Args& a, int sms, cudaStream_t s) {
  return (MODE == kForward ? a.va && a.vb : a.vb) ? launch_rows_as<MODE, R, true>(a, sms, s)
                                                  : launch_rows_as<MODE, R, false>(a, sms, s);
}
template <int MODE>
cudaError_t launch_rows(const Product& p, int sms, cudaStream_t s) {
  const Args a = args_of(p);
  if (p.I <= 1) return launch_rows_of<MODE, 1>(a, sms, s);
  if (p.I <= 4) return launch_rows_of<MODE, 4>(a, sms, s);
  return launch_rows_of<MODE, 16>(a, sms, s);
}

template <bool A_MN, bool B_MN>
cudaError_t launch_simt(const Product& p, int sms, cudaStream_t s) {
  const Args a = args_of(p);
  return launch_simt_tile<32, A_MN, B_MN>(a, sms, s);
}

// What a product on the tensor cores needs: an operand's parts, flags, shares of sums.
struct Plan {
  int64_t tiles_r, tiles_c, ctas;
  int slices, share, shares, width, cuts_a, cuts_b;
  int64_t rows_a, cols_a, ldp_a, rows_b, cols_b, ldp_b;
  size_t bytes_a, bytes_b, bytes_flags, bytes_parts;
  size_t bytes() const { return bytes_a + bytes_b + bytes_flags + bytes_parts; }
};

constexpr size_t up(size_t x) { return (x + 255) / 256 * 256; }

// CTAs that cut an operand: two rounds of eight CTAs per SM at most
int cuts_of(int64_t rows, int64_t ldp, int sms) {
  const int64_t units = rows * (ldp / 8), ctas = (units + 511) / 512;
  return (int)(ctas < 8 * sms ? (ctas < 1 ? 1 : ctas) : 8 * sms);
}

template <bool A_MN, bool B_MN, bool COUNTED = false>
cudaError_t plan_tc(const Product& p, int sms, Plan* plan) {
  static std::atomic<uint64_t> allowed;
  static std::atomic<int> clusters[64][9];
  auto* f = f32_kernel<A_MN, B_MN, COUNTED>;
  const cudaError_t e = allow_shared(f, kTcBytes, allowed);
  if (e != cudaSuccess) return e;
  Plan g = {};
  g.slices = (int)((p.L + kBK - 1) / kBK);
  g.tiles_r = (p.J + kBM - 1) / kBM;
  // Width and shares of the sum by the least estimate in cycles: a slice takes the longer of its multiplications (12 per
  // column) and its copies (48 KB and 384 bytes per column at 45 bytes a cycle, as measured with two slices in flight);
  // shares are written and read through L2. All clusters of a shared sum run at once.
  double least = 0;
  for (int width = kMostWidth; width >= 32; width -= 32) {
    if (B_MN && width == kMostWidth) continue;  // its third 64 columns would not fit
    const int64_t tiles_c = (p.I + width - 1) / width, tiles = g.tiles_r * tiles_c;
    for (int shares = 1; shares <= 8; ++shares) {
      if (shares > 1 && (tiles * shares > sms || g.slices < 3 * shares ||
                         tiles > clusters_at_once(f, shares, kThreads, kTcBytes, clusters)))
        break;
      const int share = (g.slices + shares - 1) / shares;
      const double rounds = shares > 1 ? 1.0 : (double)((tiles + sms - 1) / sms);
      const double copies = (49152.0 + 384.0 * width) / 45.0, slice = 12.0 * width > copies ? 12.0 * width : copies;
      const double time = rounds * (share * slice + 1000.0 + 20.0 * width) + (shares > 1 ? 3000.0 + 14.0 * width : 0.0);
      if (g.width == 0 || time < least) {
        least = time;
        g.width = width;
        g.tiles_c = tiles_c;
        g.share = share;
        g.shares = shares > 1 ? (g.slices + share - 1) / share : 1;
        g.ctas = g.shares > 1 ? tiles * g.shares : (tiles < sms ? tiles : sms);
        g.bytes_parts = g.shares > 1 ? (size_t)tiles * g.shares * width * kBM * sizeof(float) : 0;
      }
    }
  }
  g.rows_a = A_MN ? p.L : p.J, g.cols_a = A_MN ? p.J : p.L;
  g.rows_b = B_MN ? p.L : p.I, g.cols_b = B_MN ? p.I : p.L;
  g.ldp_a = (g.cols_a + 31) / 32 * 32, g.ldp_b = (g.cols_b + 31) / 32 * 32;
  g.cuts_a = cuts_of(g.rows_a, g.ldp_a, sms), g.cuts_b = cuts_of(g.rows_b, g.ldp_b, sms);
  g.bytes_a = up((size_t)kParts * g.rows_a * g.ldp_a * 2);
  g.bytes_b = up((size_t)kParts * g.rows_b * g.ldp_b * 2);
  g.bytes_flags = up(sizeof(uint32_t) * (g.cuts_a + g.cuts_b));
  *plan = g;
  return cudaSuccess;
}

// Parts [3][rows][ldp] of `cols` columns in boxes of 64 x `box` of one part; what lies outside reads as 0.
bool encode_parts(CUtensorMap* map, const void* p, int64_t cols, int64_t rows, int64_t ldp, int box) {
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)kParts};
  const cuuint64_t strides[2] = {(cuuint64_t)ldp * 2, (cuuint64_t)rows * ldp * 2};
  const cuuint32_t boxes[3] = {64, (cuuint32_t)box, 1}, ones[3] = {1, 1, 1};
  const Encode f = encoder();
  return f && f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(p), dims, strides, boxes, ones,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The product of operands that are cut: a's parts and flags are those of p.b, b's of p.a.
template <bool A_MN, bool B_MN, bool COUNTED>
cudaError_t launch_parts(const Product& p, const Plan& g, const Parts& pa, const Parts& pb, float* sums, cudaStream_t s) {
  TcArgs a = {};
  const cudaError_t e = error_word(&a.errors);
  if (e != cudaSuccess) return e;
  a.f = args_of(p);
  a.flags_a = pa.flags, a.flags_b = pb.flags;
  a.n_flags_a = pa.n_flags, a.n_flags = pa.n_flags + pb.n_flags;
  a.parts = sums;
  a.tiles_r = g.tiles_r, a.tiles_c = g.tiles_c, a.tiles = g.tiles_r * g.tiles_c;
  a.slices = g.slices, a.share = g.share, a.width = g.width;
  CUtensorMap ma, mb;
  if (!encode_parts(&ma, pa.p, g.cols_a, g.rows_a, g.ldp_a, A_MN ? kBK : kBM) ||
      !encode_parts(&mb, pb.p, g.cols_b, g.rows_b, g.ldp_b, B_MN ? kBK : g.width))
    return cudaErrorNotSupported;
  cudaLaunchAttribute at;
  const cudaLaunchConfig_t cfg =
      config(dim3((unsigned)g.ctas), kThreads, kTcBytes, dim3((unsigned)g.shares, 1, 1), &at, s);
  return cudaLaunchKernelEx(&cfg, f32_kernel<A_MN, B_MN, COUNTED>, ma, mb, a);
}

template <bool A_MN, bool B_MN>
cudaError_t launch_tc32(const Product& p, int sms, char* workspace, cudaStream_t s) {
  Plan g;
  const cudaError_t e = plan_tc<A_MN, B_MN>(p, sms, &g);
  if (e != cudaSuccess) return e;
  char *pa = workspace, *pb = pa + g.bytes_a, *pf = pb + g.bytes_b;
  uint32_t* flags = (uint32_t*)pf;
  const Cut ca = {(const float*)p.b, (uint16_t*)pa, g.rows_a, g.cols_a, p.ldb, g.ldp_a, can(p.b, p.ldb), nullptr};
  const Cut cb = {(const float*)p.a, (uint16_t*)pb, g.rows_b, g.cols_b, p.lda, g.ldp_b, can(p.a, p.lda), nullptr};
  cut_kernel<<<g.cuts_a + g.cuts_b, 256, 0, s>>>(ca, cb, g.cuts_a, flags);
  const cudaError_t f = cudaGetLastError();
  if (f != cudaSuccess) return f;
  return launch_parts<A_MN, B_MN, false>(p, g, {pa, flags, g.cuts_a}, {pb, flags + g.cuts_a, g.cuts_b},
                                         (float*)(pf + g.bytes_flags), s);
}

// Whether cutting the operands pays: not for few rows (rows_kernel), nor for products that start and end as fast as they
// run. Call after call with other operands, cut and as they are: 64 x 1024 x 1024 (gradient of a weight) 9.6 and 8.2 us,
// 256 x 512 x 512 12.7 and 9.9, 384 x 512 x 512 13.2 and 15.3, 17 x 2048 x 2048 (gradient of a weight) 15.7 and 23.6.
bool on_tensor_cores(const Product& p) {
  return p.L > 0 && (p.I > kFewRows || p.mode == kGradWeight) && (double)p.I * (double)p.J * (double)p.L > 1 << 26;
}

}  // namespace

cudaError_t f32_workspace(const Product& p, int sms, size_t* bytes) {
  *bytes = 0;
  if (!on_tensor_cores(p)) return cudaSuccess;
  Plan g;
  const cudaError_t e = p.mode == kForward     ? plan_tc<false, false>(p, sms, &g)
                        : p.mode == kGradInput ? plan_tc<true, false>(p, sms, &g)
                                               : plan_tc<true, true>(p, sms, &g);
  if (e == cudaSuccess) *bytes = g.bytes();
  return e;
}

cudaError_t launch_f32(const Product& p, int sms, void* workspace, cudaStream_t s) {
  const bool tc = on_tensor_cores(p);
  char* w = (char*)workspace;
  if (p.mode == kForward) {
    if (p.I <= kFewRows) return launch_rows<kForward>(p, sms, s);
    return tc ? launch_tc32<false, false>(p, sms, w, s) : launch_simt<false, false>(p, sms, s);
  }
  if (p.mode == kGradInput) {
    if (p.I <= kFewRows) return launch_rows<kGradInput>(p, sms, s);
    return tc ? launch_tc32<true, false>(p, sms, w, s) : launch_simt<false, true>(p, sms, s);
  }
  return tc ? launch_tc32<true, true>(p, sms, w, s) : launch_simt<true, true>(p, sms, s);
}

bool f32_on_tensor_cores(const Product& p) { return on_tensor_cores(p) && (p.mode == kGradWeight || p.I > kFewRows); }

int64_t parts_ld(int64_t cols) { return (cols + 31) / 32 * 32; }
size_t parts_bytes(int64_t rows, int64_t cols) { return up((size_t)kParts * (size_t)rows * (size_t)parts_ld(cols) * 2); }
int parts_flags(int64_t rows, int64_t cols, int sms) { return cuts_of(rows, parts_ld(cols), sms); }

cudaError_t launch_cut(const Uncut& a, const Uncut& b, int sms, cudaStream_t s) {
  auto job = [](const Uncut& u) {
    return Cut{u.from, (uint16_t*)u.to.p, u.rows, u.cols, u.ld, parts_ld(u.cols), can(u.from, u.ld), u.count};
  };
  // flags of both lie side by side only by chance: a launch for each
  for (const Uncut* u : {&a, &b}) {
    if (!u->from) continue;
    cut_kernel<<<u->to.n_flags, 256, 0, s>>>(job(*u), job(*u), u->to.n_flags, u->to.flags);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t f32_parts_workspace(const Product& p, int sms, size_t* bytes) {
  Plan g = {};
  const cudaError_t e = p.mode == kForward     ? plan_tc<false, false, true>(p, sms, &g)
                        : p.mode == kGradInput ? plan_tc<true, false, true>(p, sms, &g)
                                               : plan_tc<true, true, true>(p, sms, &g);
  *bytes = e == cudaSuccess ? g.bytes_parts : 0;
  return e;
}

cudaError_t launch_f32_parts(const Product& p, const Parts& of_b, const Parts& of_a, int sms, void* workspace, cudaStream_t s) {
  Plan g;
  float* sums = (float*)workspace;
  cudaError_t e;
  if (p.mode == kForward) {
    e = plan_tc<false, false, true>(p, sms, &g);
    return e == cudaSuccess ? launch_parts<false, false, true>(p, g, of_b, of_a, sums, s) : e;
  }
  if (p.mode == kGradInput) {
    e = plan_tc<true, false, true>(p, sms, &g);
    return e == cudaSuccess ? launch_parts<true, false, true>(p, g, of_b, of_a, sums, s) : e;
  }
  e = plan_tc<true, true, true>(p, sms, &g);
  return e == cudaSuccess ? launch_parts<true, true, true>(p, g, of_b, of_a, sums, s) : e;
}

}  // namespace lin
}  // namespace smat
