// Host side of the norms (include/smat.h, "norms"): argument checks, workspace, launches.

#include <cuda_runtime.h>

#include "smat.h"
#include "smat_checks.h"
#include "smat_norm.h"

using namespace smat;
using namespace smat::lin;

namespace {

// Sizes below 2^31 - 2^16: columns are counted in 32 bits with a tile's worth to spare.
constexpr int64_t kMaxSize = (int64_t(1) << 31) - (1 << 16);

smat_status check_norm(int64_t rows, int64_t cols, int32_t dtype, int32_t weight_dtype, int32_t kind) {
  if (rows < 0 || rows > kMaxSize) return lfail(SMAT_ERR_INVALID_ARG, "rows %lld out of range", (long long)rows);
  if (cols < 1 || cols > kMaxSize) return lfail(SMAT_ERR_INVALID_ARG, "cols %lld out of range", (long long)cols);
  if (dtype != SMAT_F32 && dtype != SMAT_BF16) return lfail(SMAT_ERR_UNSUPPORTED, "dtype %d not supported", dtype);
  if (weight_dtype != dtype && weight_dtype != SMAT_F32)
    return lfail(SMAT_ERR_UNSUPPORTED, "weights of dtype %d beside dtype %d", weight_dtype, dtype);
  if (kind != SMAT_NORM_LAYER && kind != SMAT_NORM_RMS) return lfail(SMAT_ERR_UNSUPPORTED, "kind %d not supported", kind);
  return SMAT_OK;
}

int64_t stats_of(int64_t rows, int32_t kind) { return kind == SMAT_NORM_LAYER ? 2 * rows : rows; }

smat_status norm_forward(const smat_norm_args* a, cudaStream_t stream) {
  if (!a) return lfail(SMAT_ERR_INVALID_ARG, "args is NULL");
  smat_status st = check_norm(a->rows, a->cols, a->dtype, a->weight_dtype, a->kind);
  if (st != SMAT_OK) return st;
  if (!(a->eps >= 0.0f)) return lfail(SMAT_ERR_INVALID_ARG, "eps must be 0 or more");
  const int64_t m = a->rows, n = a->cols;
  if (m > 0 && !a->residual != !a->h) return lfail(SMAT_ERR_INVALID_ARG, "residual and h: give both or neither");
  const size_t es = elem_of(a->dtype), ew = elem_of(a->weight_dtype);
  const Mat mats[] = {
      {"h", a->h, a->residual ? m : 0, n, a->ldh, es, true},
      {"y", a->y, m, n, a->ldy, es, true},
      {"stats", a->stats, a->stats ? 1 : 0, stats_of(m, a->kind), stats_of(m, a->kind), 4, true},
      {"x", a->x, m, n, a->ldx, es, false},
      {"residual", a->residual, a->residual ? m : 0, n, a->ldr, es, false},
      {"w", a->w, m && a->w ? 1 : 0, n, n, ew, false},
      {"b", a->b, m && a->b ? 1 : 0, n, n, ew, false},
  };
  st = check_mats(mats, 7, 0, 4);
  if (st != SMAT_OK || m == 0) return st;
  int sms = 1;
  st = device_sms(&sms);
  if (st != SMAT_OK) return st;
  const norm::Forward f = {a->x, a->residual, a->w, a->b, a->h, a->y, a->stats, m, n, a->ldx, a->ldr, a->ldh, a->ldy,
                           a->eps, a->kind == SMAT_NORM_RMS};
  return cuda_status(norm::launch_forward(f, a->dtype, a->weight_dtype, sms, stream), "norm launch");
}

// The bytes of the shares' sums; `shares`: how many there are.
size_t grad_bytes(const smat_norm_grad_args* a, int* shares) {
  int sms = 0;
  *shares = 0;
  if (a->rows == 0 || (!a->dw && !a->db) || device_sms(&sms) != SMAT_OK) return 0;
  *shares = norm::backward_shares(a->rows, a->cols, a->dtype, sms);
  return up((size_t)*shares * ((a->dw != nullptr) + (a->db != nullptr)) * (size_t)a->cols * sizeof(float));
}

smat_status norm_backward(const smat_norm_grad_args* a, void* d_workspace, size_t workspace_bytes, cudaStream_t stream) {
  if (!a) return lfail(SMAT_ERR_INVALID_ARG, "args is NULL");
  smat_status st = check_norm(a->rows, a->cols, a->dtype, a->weight_dtype, a->kind);
  if (st != SMAT_OK) return st;
  if (a->accumulate != 0 && a->accumulate != 1)
    return lfail(SMAT_ERR_UNSUPPORTED, "unknown accumulate value %d", a->accumulate);
  const int64_t m = a->rows, n = a->cols;
  const size_t es = elem_of(a->dtype), ew = elem_of(a->weight_dtype);
  const Mat mats[] = {
      {"dx", a->dx, a->dx ? m : 0, n, a->lddx, es, true},
      {"dw", a->dw, a->dw ? 1 : 0, n, n, ew, true},
      {"db", a->db, a->db ? 1 : 0, n, n, ew, true},
      {"dy", a->dy, m, n, a->lddy, es, false},
      {"h", a->h, m, n, a->ldh, es, false},
      {"stats", a->stats, m ? 1 : 0, stats_of(m, a->kind), stats_of(m, a->kind), 4, false},
      {"w", a->w, m && a->w ? 1 : 0, n, n, ew, false},
      {"dh", a->dh, a->dh && a->dx ? m : 0, n, a->lddh, es, false},
  };
  st = check_mats(mats, 8, 0, 7);
  if (st != SMAT_OK || (!a->dx && !a->dw && !a->db)) return st;
  int sms = 1, shares = 0;
  const size_t bytes = grad_bytes(a, &shares);
  st = check_workspace(d_workspace, workspace_bytes, bytes);
  if (st == SMAT_OK) st = device_sms(&sms);
  if (st != SMAT_OK) return st;
  const norm::Backward b = {a->dy, a->h, a->stats, a->w, a->dh, a->dx, a->dw, a->db, m, n, a->lddy, a->ldh, a->lddh,
                            a->lddx, a->kind == SMAT_NORM_RMS, a->accumulate != 0, (float*)d_workspace, shares};
  return cuda_status(norm::launch_backward(b, a->dtype, a->weight_dtype, sms, stream), "norm gradient launch");
}

}  // namespace

extern "C" {

smat_status smat_norm(const smat_norm_args* args, smat_stream_t stream) {
  return guarded([&] { return norm_forward(args, (cudaStream_t)stream); });
}

size_t smat_norm_grad_workspace_bytes(const smat_norm_grad_args* a) {
  int shares;
  if (!a || a->rows < 0 || a->rows > kMaxSize || a->cols < 1 || a->cols > kMaxSize) return 0;
  return grad_bytes(a, &shares);
}

smat_status smat_norm_grad(const smat_norm_grad_args* args, void* d_workspace, size_t workspace_bytes,
                           smat_stream_t stream) {
  return guarded([&] { return norm_backward(args, d_workspace, workspace_bytes, (cudaStream_t)stream); });
}

}  // extern "C"
