// What the host side of the linear layers (smat_linear_host.cpp) and their kernels share.
#pragma once

#include <atomic>
#include <cstdint>

#include <cuda_runtime.h>

#include "smat.h"

namespace smat {
namespace lin {

// Allows a kernel its dynamic shared memory, once per kernel and device.
template <class F>
cudaError_t allow_shared(F* f, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
  if (e != cudaSuccess || (done.load(std::memory_order_relaxed) & bit)) return e;
  e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// What happens to a product's sums on their way out. The last three are bf16 products of the loss over a vocabulary
// (smat_loss.h): logits that leave as their gradient, an input's gradient in fp32, stored or added to what is there, and a
// weight's gradient over rows that the device counts.
enum Mode : int { kForward = 0, kGradInput = 1, kGradWeight = 2, kLogitGrad = 3, kGradInputSum = 4, kGradWeightRows = 5 };

// A row of a logits' gradient: g (exp2(log2(e) logit - lse2) - [column = target]).
struct LossRow {
  float lse2;  // log2(e) lse
  float g;
  int target;  // or -1
  float own;   // fp32: lse; bf16: the target's own gradient, see gather_kernel in smat_loss.cu
};

// One product: out(i, j) from sum over l of A(i, l) B(j, l), i < I, j < J, l < L. An operand with the sum running
// along its rows ("K-major") has A(i, l) at a[i * lda + l]; one with the sum running down its columns ("MN-major")
// at a[l * lda + i]:
//   forward      A = x [rows, k]   B = W [n, k]   both K-major
//   grad_input   A = dy [rows, n]  K-major, B = W [n, k] MN-major, j runs over k
//   grad_weight  A = dy [rows, n]  B = x [rows, k] both MN-major, i over n and j over k
struct Product {
  int mode;  // Mode
  int dtype;
  const void* a;
  const void* b;
  int64_t lda, ldb;
  int64_t I, J, L;
  // the epilogue
  const void* bias;      // [J]
  const void* residual;  // [I, J]
  void* out;             // [I, J]
  int8_t* q;             // [I, J]: written by the forward, read by grad_input
  uint8_t* e;
  int64_t ldr, ldo, ldq, lde;
  int act;
  int accumulate;  // grad_weight: add to what out holds
  // bf16 grad_weight: db [I] from shares of its sums, [sum_shares][I]; db NULL: none
  const float* sums;
  void* db;
  int sum_shares, add_db;
  // the loss's products
  const int* count;         // kLogitGrad and on, launch_f32_parts; on the device: how many rows there are, at most I (or L)
  const LossRow* loss_rows; // kLogitGrad: [I]
  int64_t first_col;        // kLogitGrad: the first column's place in the vocabulary
  int splits;               // kGradInputSum: parts of the sum that other clusters make, each `slab` rows after the last (0: one)
  int64_t slab;             // a multiple of 256
  int halves;               // kLogitGrad: rows from count / 2 on are what the same rows before them lose by their rounding
};

// fp32 (smat_linear_f32.cu): any size, stride and alignment. `workspace`: f32_workspace() bytes, which go by mode, I, J
// and L alone.
cudaError_t f32_workspace(const Product& p, int sms, size_t* bytes);
cudaError_t launch_f32(const Product& p, int sms, void* workspace, cudaStream_t s);

// The same in steps, for operands that several products share and rows that the device counts (p.count: the rows i, for a weight's
// gradient the terms of the sum). An operand [rows, cols] is cut into parts of bf16, [3][rows][parts_ld(cols)], and flags that say
// whether they stand for it. Only for products that f32_on_tensor_cores() names.
struct Parts {
  void* p;  // parts_bytes(rows, cols)
  uint32_t* flags;
  int n_flags;  // parts_flags(rows, cols), where launch_cut makes them
};
struct Uncut {
  const float* from;  // or NULL: nothing to cut
  int64_t rows, cols, ld;
  const int* count;  // or NULL: on the device, the rows there are; those behind them up to a multiple of 64 hold zeros
  Parts to;
};
bool f32_on_tensor_cores(const Product& p);
int64_t parts_ld(int64_t cols);
size_t parts_bytes(int64_t rows, int64_t cols);
int parts_flags(int64_t rows, int64_t cols, int sms);
cudaError_t launch_cut(const Uncut& a, const Uncut& b, int sms, cudaStream_t s);
cudaError_t f32_parts_workspace(const Product& p, int sms, size_t* bytes);
cudaError_t launch_f32_parts(const Product& p, const Parts& of_b, const Parts& of_a, int sms, void* workspace, cudaStream_t s);

// bf16 on the tensor cores (smat_linear_tc.cu): a and b on 16-byte boundaries, lda and ldb multiples of 8.
// `workspace`: tc_workspace() bytes, which go by mode, I, J and L alone.
cudaError_t tc_workspace(const Product& p, int sms, size_t* bytes);
cudaError_t launch_tc(const Product& p, int sms, void* workspace, cudaStream_t s);
// kGradInputSum: into how many parts its sum is best cut, for few rows.
cudaError_t grad_input_splits(const Product& p, int* splits);
// The tensor-core products' error bits of the current device; read and cleared (waits for the stream).
cudaError_t error_word(int** at);
cudaError_t read_errors(int* out, cudaStream_t s);

// smat_pack8.cu; `dy` NULL: out = act(h^), else dy * act'(h^)
cudaError_t launch_pack8(const void* x, int64_t ldx, int8_t* q, int64_t ldq, uint8_t* e, int64_t lde, int64_t rows,
                         int64_t cols, int dtype, int sms, cudaStream_t s);
cudaError_t launch_unpack8(const int8_t* q, int64_t ldq, const uint8_t* e, int64_t lde, const void* dy, int64_t lddy,
                           void* out, int64_t ldout, int64_t rows, int64_t cols, int dtype, int act, int sms,
                           cudaStream_t s);
// db[n] = sum over rows of dy[rows, n], or added to db
cudaError_t launch_row_sums(const void* dy, int64_t lddy, void* db, int64_t rows, int64_t cols, int dtype, bool add,
                            int sms, cudaStream_t s);

// A weight gradient over 1 to kOuterRows rows (smat_linear_outer.cu): x, or q and e read through act; db may be NULL. Up to
// these many it is faster than the products' tiles (4096 x 4096, call after call: bf16 one row 7.0 us against 18, 8 rows 17.6
// against 18.1, with rows off 16 bytes 18 against 37; fp32 one row 12 us against 80, 16 rows 37 against 38; with nothing in L2
// 14 against 26, 25.6 against 26.1, 24 against 92, 50 against 61). With other operands every call, bf16 8 and fp32 16 rows: 128 x
// 64 3.3 us against 5.2 and 3.1 against 5.7, 512 x 512 3.2 and 5.4, 3.5 and 5.7, 896 x 4864 9.1 and 11.2, 16.2 and 16.8, 4096 x
// 1024 9.2 and 10.3, 16.2 and 24.9; 11008 x 4096 39.2 and 38.1, 91.5 and 86.5, where it no longer is, by 3 and 6%.
constexpr int64_t kOuterRows = 16, kOuterRowsBf16 = 8;
struct Outer {
  const void* dy;
  const void* x;
  const int8_t* q;
  const uint8_t* e;
  void* dw;
  void* db;
  int64_t rows, k, n, lddy, ldx, ldq, lde, lddw;
  int act;
  bool add_dw, add_db;
};
cudaError_t launch_outer(const Outer& a, int dtype, int sms, cudaStream_t s);

// What a bf16 product needs done before it: nothing for a job whose first pointer (sums: `to`) is NULL. Rows written
// start on 32 bytes.
struct Prepare {
  struct Copy {
    const void* from;
    void* to;
    int64_t rows, cols, ld, ldto;
    int ctas;
  } copy[2];
  struct Unpack {  // act(h^)
    const int8_t* q;
    const uint8_t* e;
    void* to;
    int64_t rows, cols, ldq, lde, ldto;
    int ctas;
    bool whole;  // q's rows start on 16 bytes
  } unpack;
  struct Sums {  // [shares][cols]: of every column over the rows of a share
    const void* dy;
    float* to;
    int64_t rows, cols, lddy;
    int shares;
    bool vec;
  } sums;
};
int sum_shares(int64_t rows);
cudaError_t launch_prepare(Prepare a, int act, int sms, cudaStream_t s);

}  // namespace lin
}  // namespace smat
