// What the host side of the loss over a vocabulary (smat_loss_host.cpp) and its kernels (smat_loss.cu; the products are the
// linear layers') share.
#pragma once

#include <cstdint>

#include <cuda_runtime.h>

#include "smat_linear.h"

namespace smat {
namespace loss {

using lin::LossRow;

// bf16 logits x W^T of a piece of the vocabulary (smat_loss_tc.cu): x and w on 16-byte boundaries, row strides multiples of 8.
struct Logits {
  const void* x;
  const void* w;
  const int64_t* targets;
  float2* partials;  // [slots][rows]: largest logit and sum of exponentials of what is left, of a part of the words
  float* picked;     // [rows]: the target's logit, where the target is one of the words
  int64_t rows, k, cols, ldx, ldw;
  int64_t first_col;  // the first word's place in the vocabulary
};
// The parts that a row's words come in: by rows, k and cols alone.
cudaError_t logit_slots(const Logits& p, int sms, int64_t* slots);
cudaError_t launch_logits(const Logits& p, int sms, cudaStream_t s);

// The rows that count (their target is not `ignore`) by number: place[row] or -1, and *count. twice: every one a second time, at
// place + *count / 2.
struct Index {
  const int64_t* targets;
  const float* g;
  const float* lse;
  const void* w;  // as the call has it
  int64_t ldw;
  int64_t rows, n, ignore;
  int* place;
  LossRow* info;
  int* count;
  bool twice;
};
cudaError_t launch_index(const Index& a, cudaStream_t s);
// x's rows that count and their info, at their places; rows of zeros behind them up to the next multiple of 64, or to the
// end.
cudaError_t launch_gather(const Index& a, const void* x, int64_t ldx, void* to, int64_t ldto, int64_t k, int dtype, bool to_end,
                          int sms, cudaStream_t s);
// dx's sums, in `splits` parts that lie `apart` floats after one another.
struct Sums {
  const float* at;
  int64_t ld;
  int splits;
  int64_t apart;
};
// dx from the sums at the rows' places (both of them); 0 for a row that has none.
cudaError_t launch_scatter(const Sums& from, const Index& a, void* dx, int64_t lddx, int64_t k, int dtype, int sms, cudaStream_t s);
// A row's parts [slots][rows] (largest logit, sum of exponentials) joined.
struct Join {
  const float2* partials;
  const float* picked;
  const int64_t* targets;
  float* loss;
  float* lse;
  int64_t rows, slots, n, ignore;
};
cudaError_t launch_join(const Join& a, int sms, cudaStream_t s);
// fp32 logits of a piece of the vocabulary, [rows, cols]: their part of each row, and their gradient in their place (rows behind
// the last one that counts: 0).
cudaError_t launch_row_part(const float* z, int64_t ldz, int64_t rows, int64_t cols, int64_t first_col, const int64_t* targets,
                            float2* part, float* picked, int sms, cudaStream_t s);
cudaError_t launch_row_grad(float* z, int64_t ldz, int64_t rows, int64_t cols, int64_t first_col, const LossRow* info,
                            const int* count, int sms, cudaStream_t s);
// The same for rows that count, and those behind them up to a multiple of 64, with the gradient's parts for the tensor cores beside
// it (flags: one of each CTA, parts.n_flags of them).
cudaError_t launch_row_grad_cut(float* z, int64_t ldz, int64_t rows, int64_t cols, int64_t first_col, const LossRow* info,
                                const int* count, const lin::Parts& parts, cudaStream_t s);
// to += from, [rows, cols] both, row stride ld
cudaError_t launch_add(float* to, const float* from, int64_t ld, int64_t rows, int64_t cols, int sms, cudaStream_t s);

}  // namespace loss
}  // namespace smat
