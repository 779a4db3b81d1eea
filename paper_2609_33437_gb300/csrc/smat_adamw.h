// What the host side of the AdamW step over many tensors (smat_adamw_host.cpp) and its kernels (smat_adamw.cu) share.
#pragma once

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
