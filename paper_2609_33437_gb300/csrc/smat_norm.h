// What the host side of the norms (smat_norm_host.cpp) and their kernels (smat_norm.cu) share.
#pragma once

#include <cstdint>

#include <cuda_runtime.h>

#include "smat.h"

namespace smat {
namespace norm {

struct Forward {
  const void* x;
  const void* r;  // residual or NULL; then h is written
  const void* w;  // weight, bias: or NULL
  const void* b;
  void* h;
  void* y;
  float* stats;  // or NULL: [2][rows] (mean, 1 / deviation), rms [1][rows]
  int64_t rows, cols, ldx, ldr, ldh, ldy;
  float eps;
  bool rms;
};

struct Backward {
  const void* dy;
  const void* h;
  const float* stats;
  const void* w;   // or NULL
  const void* dh;  // or NULL
  void* dx;        // or NULL
  void* dw;        // or NULL
  void* db;        // or NULL
  int64_t rows, cols, lddy, ldh, lddh, lddx;
  bool rms, accumulate;
  float* parts;  // [shares][dw, db as they are wanted][cols]
  int shares;
};

cudaError_t launch_forward(const Forward& a, int dtype, int weight_dtype, int sms, cudaStream_t s);
// The shares of the rows that a weight's gradient is summed in: a call's workspace is shares * wanted * cols floats.
int backward_shares(int64_t rows, int64_t cols, int dtype, int sms);
cudaError_t launch_backward(const Backward& a, int dtype, int weight_dtype, int sms, cudaStream_t s);

}  // namespace norm
}  // namespace smat
