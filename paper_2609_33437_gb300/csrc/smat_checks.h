// What the host sides of the operators share: messages, checks of matrices and workspaces, the device's SM count.
#pragma once

#include <atomic>
#include <cstdarg>
#include <cstdio>

#include <cuda_runtime.h>

#include "smat.h"
#include "smat_internal.h"

namespace smat {
namespace lin {

inline smat_status lfail(smat_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  return (smat_status)record_error_code(st, buf);
}

inline smat_status cuda_status(cudaError_t e, const char* what) {
  if (e == cudaSuccess) return SMAT_OK;
  return lfail(SMAT_ERR_CUDA, "%s: %s (%s)", what, cudaGetErrorName(e), cudaGetErrorString(e));
}

inline size_t elem_of(int32_t dtype) { return dtype == SMAT_BF16 ? 2 : 4; }

// One matrix argument; `cols` 0 or `rows` 0: nothing is read.
struct Mat {
  const char* name;
  const void* p;
  int64_t rows, cols, ld;
  size_t elem;
  bool written;
  bool empty() const { return rows == 0 || cols == 0; }
  uintptr_t begin() const { return (uintptr_t)p; }
  uintptr_t end() const { return begin() + ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) * elem; }
};

// Whether two matrices share an element. Views of one buffer with one row stride whose columns lie apart (the
// slices of a joint projection) do not.
inline bool overlap(const Mat& a, const Mat& b) {
  if (a.empty() || b.empty() || a.end() <= b.begin() || b.end() <= a.begin()) return false;
  const uintptr_t stride = (uintptr_t)a.ld * a.elem;
  if (stride != (uintptr_t)b.ld * b.elem || stride == 0) return true;
  const Mat &lo = a.begin() <= b.begin() ? a : b, &hi = a.begin() <= b.begin() ? b : a;
  const uintptr_t off = (hi.begin() - lo.begin()) % stride;
  return off < (uintptr_t)lo.cols * lo.elem || off + (uintptr_t)hi.cols * hi.elem > stride;
}

// `same`: two matrices that may be one and the same (or -1)
inline smat_status check_mats(const Mat* m, int count, int same_a, int same_b) {
  for (int i = 0; i < count; ++i) {
    if (m[i].empty()) continue;
    if (!m[i].p) return lfail(SMAT_ERR_INVALID_ARG, "%s is NULL", m[i].name);
    if (m[i].ld < m[i].cols || m[i].ld > (int64_t(1) << 40))
      return lfail(SMAT_ERR_INVALID_ARG, "%s: row stride %lld for %lld columns", m[i].name, (long long)m[i].ld,
                   (long long)m[i].cols);
    if ((uintptr_t)m[i].p % m[i].elem)
      return lfail(SMAT_ERR_ALIGNMENT, "%s: not aligned to %zu bytes", m[i].name, m[i].elem);
  }
  for (int i = 0; i < count; ++i) {
    if (!m[i].written) continue;
    for (int j = 0; j < count; ++j) {
      if (i == j || (m[j].written && j < i)) continue;
      if ((i == same_a && j == same_b) && m[i].p == m[j].p && m[i].ld == m[j].ld) continue;
      if (overlap(m[i], m[j]))
        return lfail(SMAT_ERR_INVALID_ARG, "%s overlaps %s", m[i].name, m[j].name);
    }
  }
  GpuAccess access;
  for (int i = 0; i < count; ++i) {
    if (m[i].empty()) continue;
    const int ok = access.check(m[i].p);
    if (ok < 0) return lfail(SMAT_ERR_CUDA, "no current CUDA device or pointer attributes unavailable");
    if (!ok) return lfail(SMAT_ERR_INVALID_ARG, "%s is not accessible from the GPU", m[i].name);
  }
  return SMAT_OK;
}

// The current device's SM count, asked for once per device.
inline smat_status device_sms(int* sms) {
  static std::atomic<int> known[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && dev < 64 && (*sms = known[dev].load(std::memory_order_relaxed)) > 0) return SMAT_OK;
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess && dev < 64) known[dev].store(*sms, std::memory_order_relaxed);
  return cuda_status(e, "device query");
}

constexpr size_t kWsAlign = 256;
inline size_t up(size_t x) { return (x + kWsAlign - 1) / kWsAlign * kWsAlign; }

inline smat_status check_workspace(const void* d_workspace, size_t bytes, size_t needed) {
  if (needed == 0) return SMAT_OK;
  if (!d_workspace) return lfail(SMAT_ERR_WORKSPACE, "workspace is NULL");
  if ((uintptr_t)d_workspace % kWsAlign) return lfail(SMAT_ERR_WORKSPACE, "workspace not 256-byte aligned");
  if (bytes < needed) return lfail(SMAT_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", bytes, needed);
  return SMAT_OK;
}

// The tensor-core products read bf16 operands whose rows start on 16 bytes. One that does not is copied to the
// workspace first: rows of ld_of(cols) elements.
inline int64_t ld_of(int64_t cols) { return (cols + 31) / 32 * 32; }
inline size_t copy_bytes(int64_t rows, int64_t cols, size_t elem) { return up((size_t)rows * (size_t)ld_of(cols) * elem); }

struct Operand {
  const void* p;
  int64_t rows, cols, ld;
  bool copied;
};
inline Operand operand(const void* p, int64_t rows, int64_t cols, int64_t ld, int32_t dtype) {
  Operand o = {p, rows, cols, ld, false};
  if (dtype != SMAT_BF16 || rows == 0 || cols == 0) return o;
  if (rows == 1) o.ld = ld_of(cols);  // any stride will do
  o.copied = (uintptr_t)p % 16 || o.ld % 8;
  return o;
}
inline size_t operand_bytes(const Operand& o) { return o.copied ? copy_bytes(o.rows, o.cols, 2) : 0; }

// An exception (the host's memory running out) is a status like any other failure.
template <class F>
smat_status guarded(F&& f) {
  try {
    return f();
  } catch (...) {
    return SMAT_ERR_CUDA;
  }
}

}  // namespace lin
}  // namespace smat
