// What the host side of the AdamW step over many tensors (smat_adamw_host.cpp) and its kernels (smat_adamw.cu) share.
#pragma once

#include <cmath>
#include <cstdint>

#include <cuda_runtime.h>

#include "smat.h"

namespace smat {
namespace adamw {

constexpr int kGroup = SMAT_ADAMW_GROUP;

// A tensor of a launch: `first` of its groups in the list (from the launch's first one on), and what its last group lacks.
struct Entry {
  void* p;
  const void* g;
  uint32_t first;
  uint16_t lacks;  // 0 .. 255
  uint16_t whole;  // both start on 32 bytes: whole groups are read and written 8 elements at a time
};

struct Constants {  // computed in double, rounded once
  float b1, omb1, b2, omb2, eps;
  float decay, step, bc2, inv_bc2;  // 1 - lr wd, lr / (1 - b1^t), sqrt(1 - b2^t) and one over it
};
// 1 - beta^t (the logarithm of 0 is -infinity: its power is 0)
inline double correction(double beta, double t) { return -std::expm1(t * std::log(beta)); }
inline Constants constants_of(double lr, double beta1, double beta2, double eps, double weight_decay, double bc1, double bc2) {
  return {(float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)eps, (float)(1.0 - lr * weight_decay),
          (float)(lr / bc1), (float)std::sqrt(bc2), (float)(1.0 / std::sqrt(bc2))};
}
inline bool within(double v, double low, double high) { return v >= low && v < high; }  // false for NaN
// What is wrong with the hyperparameters, or NULL.
inline const char* refuse(double lr, double beta1, double beta2, double eps, double weight_decay) {
  const double huge = 3e38;  // finite in fp32
  if (!within(lr, 0.0, huge)) return "lr must be finite and 0 or more";
  if (!within(beta1, 0.0, 1.0) || !within(beta2, 0.0, 1.0)) return "betas must be in [0, 1)";
  if (!within(eps, 1.1754944e-38, huge)) return "eps must be finite and at least 2^-126";
  if (!within(weight_decay, 0.0, huge)) return "weight_decay must be finite and 0 or more";
  return nullptr;
}
inline bool step_fits(int64_t t) { return t >= 1 && t < int64_t(1) << 31; }

struct Call {
  Constants c;
  float scale;
  const float* scale_at;   // or NULL
  const float* lr_at;      // or NULL: the device's lr
  const int64_t* step_at;  // or NULL: the device's t
  double lr, bc1, log_b1, log_b2, weight_decay;  // for those two (bc1: 1 - b1^t)
  uint32_t seed_key;       // of the seed, before the step
  uint32_t key;            // with the step
  void* m1;                // of the launch's first group on
  void* m2;
  uint8_t* e1;
  uint8_t* e2;
  int64_t place;           // of the launch's first element in the list
  uint32_t groups;
  int32_t n;
};

// As many tensors as fit beside a Call in a launch's parameters (32,764 bytes).
constexpr int kMaxEntries = 1300;

constexpr uint32_t kMix1 = 0x85EBCA6Bu, kMix2 = 0xC2B2AE35u;
__host__ __device__ inline uint32_t mix(uint32_t h) {  // the 32-bit finaliser of MurmurHash3 (A. Appleby)
  h ^= h >> 16;
  h *= kMix1;
  h ^= h >> 13;
  h *= kMix2;
  return h ^ h >> 16;
}

cudaError_t launch_step(const Call& c, const Entry* entries, int dtype, int grad_dtype, int bits, int sms, cudaStream_t s);
cudaError_t launch_values(const uint8_t* q1, const uint8_t* e1, const uint8_t* q2, const uint8_t* e2, void* m1, void* r,
                          int64_t places, int sms, cudaStream_t s);

}  // namespace adamw
}  // namespace smat
