// Host side of the linear layers (include/smat.h): argument checks, workspace, launches.

#include <atomic>
#include <cstdarg>
#include <cstdio>

#include <cuda_runtime.h>

#include "smat.h"
#include "smat_internal.h"
#include "smat_linear.h"

using namespace smat;
using namespace smat::lin;

namespace {

smat_status lfail(smat_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  return (smat_status)record_error_code(st, buf);
}

smat_status cuda_status(cudaError_t e, const char* what) {
  if (e == cudaSuccess) return SMAT_OK;
  return lfail(SMAT_ERR_CUDA, "%s: %s (%s)", what, cudaGetErrorName(e), cudaGetErrorString(e));
}

// Sizes are below 2^31 - 2^16, so that kernels can round them up and count in 32 bits (offsets are 64 bits wide).
// The second size of a result (n of linear and grad_weight, k of grad_input) is cut into at most 65535 tiles.
constexpr int64_t kMaxSize = (int64_t(1) << 31) - (1 << 16);
constexpr int64_t kMaxCols = int64_t(65535) * 64;

size_t elem_of(int32_t dtype) { return dtype == SMAT_BF16 ? 2 : 4; }

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
bool overlap(const Mat& a, const Mat& b) {
  if (a.empty() || b.empty() || a.end() <= b.begin() || b.end() <= a.begin()) return false;
  const uintptr_t stride = (uintptr_t)a.ld * a.elem;
  if (stride != (uintptr_t)b.ld * b.elem || stride == 0) return true;
  const Mat &lo = a.begin() <= b.begin() ? a : b, &hi = a.begin() <= b.begin() ? b : a;
  const uintptr_t off = (hi.begin() - lo.begin()) % stride;
  return off < (uintptr_t)lo.cols * lo.elem || off + (uintptr_t)hi.cols * hi.elem > stride;
}

smat_status check_sizes(int64_t rows, int64_t k, int64_t n, int32_t dtype, int32_t act) {
  const int64_t sizes[3] = {rows, k, n};
  const char* names[3] = {"rows", "k", "n"};
  for (int i = 0; i < 3; ++i)
    if (sizes[i] < 0 || sizes[i] > (i == 0 ? kMaxSize : kMaxCols))
      return lfail(SMAT_ERR_INVALID_ARG, "%s %lld out of range", names[i], (long long)sizes[i]);
  if (dtype != SMAT_F32 && dtype != SMAT_BF16) return lfail(SMAT_ERR_UNSUPPORTED, "dtype %d not supported", dtype);
  if (act < SMAT_ACT_NONE || act > SMAT_ACT_SILU) return lfail(SMAT_ERR_UNSUPPORTED, "activation %d not supported", act);
  return SMAT_OK;
}

// `same`: two matrices that may be one and the same (or -1)
smat_status check_mats(const Mat* m, int count, int same_a, int same_b) {
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
smat_status device_sms(int* sms) {
  static std::atomic<int> known[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && dev < 64 && (*sms = known[dev].load(std::memory_order_relaxed)) > 0) return SMAT_OK;
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess && dev < 64) known[dev].store(*sms, std::memory_order_relaxed);
  return cuda_status(e, "device query");
}

int64_t groups_of(int64_t cols) { return (cols + SMAT_PACK8_GROUP - 1) / SMAT_PACK8_GROUP; }

constexpr size_t kWsAlign = 256;
size_t up(size_t x) { return (x + kWsAlign - 1) / kWsAlign * kWsAlign; }

smat_status check_workspace(const void* d_workspace, size_t bytes, size_t needed) {
  if (needed == 0) return SMAT_OK;
  if (!d_workspace) return lfail(SMAT_ERR_WORKSPACE, "workspace is NULL");
  if ((uintptr_t)d_workspace % kWsAlign) return lfail(SMAT_ERR_WORKSPACE, "workspace not 256-byte aligned");
  if (bytes < needed) return lfail(SMAT_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", bytes, needed);
  return SMAT_OK;
}

// The tensor-core products read bf16 operands whose rows start on 16 bytes. One that does not is copied to the
// workspace first: rows of ld_of(cols) elements.
int64_t ld_of(int64_t cols) { return (cols + 31) / 32 * 32; }
size_t copy_bytes(int64_t rows, int64_t cols, size_t elem) { return up((size_t)rows * (size_t)ld_of(cols) * elem); }

struct Operand {
  const void* p;
  int64_t rows, cols, ld;
  bool copied;
};
Operand operand(const void* p, int64_t rows, int64_t cols, int64_t ld, int32_t dtype) {
  Operand o = {p, rows, cols, ld, false};
  if (dtype != SMAT_BF16 || rows == 0 || cols == 0) return o;
  if (rows == 1) o.ld = ld_of(cols);  // any stride will do
  o.copied = (uintptr_t)p % 16 || o.ld % 8;
  return o;
}
size_t operand_bytes(const Operand& o) { return o.copied ? copy_bytes(o.rows, o.cols, 2) : 0; }

// The operands of the three products, rows and columns as they lie in memory; of grad_weight's x^ in 8 bits, the
// values it is read back to.
struct Operands {
  Operand a, b;
  size_t values;  // bytes of grad_weight's x^
  size_t parts;   // bytes of the product's own
  size_t sums;    // bytes of the shares of db's sums
  size_t bytes() const { return values + operand_bytes(a) + operand_bytes(b) + sums + parts; }
};

size_t parts_of(int mode, int32_t dtype, int64_t I, int64_t J, int64_t L) {
  int sms = 0;
  size_t bytes = 0;
  if (device_sms(&sms) != SMAT_OK) return 0;
  Product p = {};
  p.mode = mode, p.I = I, p.J = J, p.L = L;
  const cudaError_t e = dtype == SMAT_BF16 ? tc_workspace(p, sms, &bytes) : f32_workspace(p, sms, &bytes);
  return e == cudaSuccess ? up(bytes) : 0;
}

Operands operands(const smat_linear_args* g) {
  if (g->n == 0 || g->rows == 0) return {};
  return {operand(g->x, g->rows, g->k, g->ldx, g->dtype), operand(g->w, g->n, g->k, g->ldw, g->dtype), 0,
          parts_of(kForward, g->dtype, g->rows, g->n, g->k)};
}
Operands operands(const smat_grad_input_args* g) {
  if (g->k == 0 || g->rows == 0) return {};
  return {operand(g->dy, g->rows, g->n, g->lddy, g->dtype), operand(g->w, g->n, g->k, g->ldw, g->dtype), 0,
          parts_of(kGradInput, g->dtype, g->rows, g->k, g->n)};
}
// Whether a weight gradient is written row by row of it, without a product's tiles (at least one row of dy).
bool few_rows(const smat_grad_weight_args* g) {
  return g->rows >= 1 && g->rows <= (g->dtype == SMAT_BF16 ? kOuterRowsBf16 : kOuterRows);
}
Operands operands(const smat_grad_weight_args* g) {
  if (g->k == 0 || g->n == 0 || g->rows == 0 || few_rows(g)) return {};
  Operands o = {operand(g->dy, g->rows, g->n, g->lddy, g->dtype), {}, 0,
                parts_of(kGradWeight, g->dtype, g->n, g->k, g->rows)};
  if (g->q)
    o.values = copy_bytes(g->rows, g->k, elem_of(g->dtype));
  else
    o.b = operand(g->x, g->rows, g->k, g->ldx, g->dtype);
  if (g->db && g->dtype == SMAT_BF16) o.sums = up(sizeof(float) * (size_t)sum_shares(g->rows) * (size_t)g->n);
  return o;
}

// What has to be done first (`first`: grad_weight's x^ and sums, where it is bf16), then the product.
smat_status run_product(Product& p, const Operands& o, Prepare& first, char* d_workspace, int act, int sms, cudaStream_t s,
                        const char* what) {
  const Operand* in[2] = {&o.a, &o.b};
  const void** to[2] = {&p.a, &p.b};
  int64_t* ld[2] = {&p.lda, &p.ldb};
  for (int i = 0; i < 2; ++i) {
    if (!in[i]->p) continue;
    *to[i] = in[i]->p;
    *ld[i] = in[i]->ld;
    if (!in[i]->copied) continue;
    *to[i] = d_workspace;
    *ld[i] = ld_of(in[i]->cols);
    first.copy[i] = {in[i]->p, d_workspace, in[i]->rows, in[i]->cols, in[i]->ld, *ld[i], 0};
    d_workspace += operand_bytes(*in[i]);
  }
  if (first.sums.to) {
    p.sums = first.sums.to = (float*)d_workspace;
    p.sum_shares = first.sums.shares;
    d_workspace += o.sums;
  }
  if (p.dtype == SMAT_BF16) {
    const smat_status st = cuda_status(launch_prepare(first, act, sms, s), "preparing launch");
    if (st != SMAT_OK) return st;
  }
  return cuda_status(p.dtype == SMAT_BF16 ? launch_tc(p, sms, d_workspace, s)
                                            : launch_f32(p, sms, d_workspace, s),
                     what);
}

// A call's size check without its message: what the size queries return 0 for.
bool sizes_fit(int64_t rows, int64_t k, int64_t n) {
  return rows >= 0 && rows <= kMaxSize && k >= 0 && k <= kMaxCols && n >= 0 && n <= kMaxCols;
}

// An exception (the host's memory running out) is a status like any other failure.
template <class F>
smat_status guarded(F&& f) {
  try {
    return f();
  } catch (...) {
    return SMAT_ERR_CUDA;
  }
}

template <class A>
size_t workspace_of(const A* a) {
  return a && sizes_fit(a->rows, a->k, a->n) ? operands(a).bytes() : 0;
}

}  // namespace

extern "C" {

size_t smat_linear_workspace_bytes(const smat_linear_args* a) { return workspace_of(a); }
size_t smat_grad_input_workspace_bytes(const smat_grad_input_args* a) { return workspace_of(a); }
size_t smat_grad_weight_workspace_bytes(const smat_grad_weight_args* a) { return workspace_of(a); }

static smat_status linear(const smat_linear_args* a, void* d_workspace, size_t workspace_bytes,
                          smat_stream_t stream) {
  if (!a) return lfail(SMAT_ERR_INVALID_ARG, "args is NULL");
  smat_status st = check_sizes(a->rows, a->k, a->n, a->dtype, a->act);
  if (st != SMAT_OK) return st;
  if (!a->q != !a->e) return lfail(SMAT_ERR_INVALID_ARG, "q and e: give both or neither");
  const size_t es = elem_of(a->dtype);
  const int64_t m = a->rows, k = a->k, n = a->n;
  const Mat mats[] = {
      {"y", a->y, m, n, a->ldy, es, true},
      {"q", a->q, a->q ? m : 0, n, a->ldq, 1, true},
      {"e", a->e, a->e ? m : 0, groups_of(n), a->lde, 1, true},
      {"x", a->x, n ? m : 0, k, a->ldx, es, false},
      {"w", a->w, m ? n : 0, k, a->ldw, es, false},
      {"bias", a->bias, m && a->bias ? 1 : 0, n, n, es, false},
      {"residual", a->residual, a->residual ? m : 0, n, a->ldr, es, false},
  };
  st = check_mats(mats, 7, 0, 6);
  if (st != SMAT_OK || m == 0 || n == 0) return st;
  const Operands ops = operands(a);
  st = check_workspace(d_workspace, workspace_bytes, ops.bytes());
  if (st != SMAT_OK) return st;
  int sms = 1;
  st = device_sms(&sms);
  if (st != SMAT_OK) return st;
  Product p = {};
  p.mode = kForward;
  p.dtype = a->dtype;
  p.I = m, p.J = n, p.L = k;
  p.bias = a->bias, p.residual = a->residual, p.out = a->y, p.q = a->q, p.e = a->e;
  p.ldr = a->ldr, p.ldo = a->ldy, p.ldq = a->ldq, p.lde = a->lde;
  p.act = a->act;
  Prepare first = {};
  return run_product(p, ops, first, (char*)d_workspace, SMAT_ACT_NONE, sms, stream, "linear launch");
}

static smat_status grad_input(const smat_grad_input_args* a, void* d_workspace, size_t workspace_bytes,
                              smat_stream_t stream) {
  if (!a) return lfail(SMAT_ERR_INVALID_ARG, "args is NULL");
  smat_status st = check_sizes(a->rows, a->k, a->n, a->dtype, a->act);
  if (st != SMAT_OK) return st;
  const bool act = a->act != SMAT_ACT_NONE;
  const int64_t m = a->rows, k = a->k, n = a->n;
  const bool read = act && m > 0 && k > 0;  // of nothing q and e may be NULL, as memory of no bytes often is
  if ((read && (!a->q || !a->e)) || (!act && (a->q || a->e)))
    return lfail(SMAT_ERR_INVALID_ARG, "q and e: give both with an activation, neither without");
  const size_t es = elem_of(a->dtype);
  const Mat mats[] = {
      {"dx", a->dx, m, k, a->lddx, es, true},
      {"dy", a->dy, k ? m : 0, n, a->lddy, es, false},
      {"w", a->w, m ? n : 0, k, a->ldw, es, false},
      {"q", a->q, act ? m : 0, k, a->ldq, 1, false},
      {"e", a->e, act ? m : 0, groups_of(k), a->lde, 1, false},
  };
  st = check_mats(mats, 5, -1, -1);
  if (st != SMAT_OK || m == 0 || k == 0) return st;
  const Operands ops = operands(a);
  st = check_workspace(d_workspace, workspace_bytes, ops.bytes());
  if (st != SMAT_OK) return st;
  int sms = 1;
  st = device_sms(&sms);
  if (st != SMAT_OK) return st;
  Product p = {};
  p.mode = kGradInput;
  p.dtype = a->dtype;
  p.I = m, p.J = k, p.L = n;
  p.out = a->dx, p.q = const_cast<int8_t*>(a->q), p.e = const_cast<uint8_t*>(a->e);
  p.ldo = a->lddx, p.ldq = a->ldq, p.lde = a->lde;
  p.act = a->act;
  Prepare first = {};
  return run_product(p, ops, first, (char*)d_workspace, SMAT_ACT_NONE, sms, stream, "grad_input launch");
}

static smat_status grad_weight(const smat_grad_weight_args* a, void* d_workspace, size_t workspace_bytes,
                               smat_stream_t stream) {
  if (!a) return lfail(SMAT_ERR_INVALID_ARG, "args is NULL");
  smat_status st = check_sizes(a->rows, a->k, a->n, a->dtype, a->act);
  if (st != SMAT_OK) return st;
  if (!a->q != !a->e) return lfail(SMAT_ERR_INVALID_ARG, "q and e: give both or neither");
  const int64_t m = a->rows, k = a->k, n = a->n;
  const bool some = m > 0 && k > 0 && n > 0;
  if (some && !a->x == !a->q) return lfail(SMAT_ERR_INVALID_ARG, "give x, or q and e, not both");
  if (!a->q && a->act != SMAT_ACT_NONE && (some || a->x))  // of nothing q may be NULL
    return lfail(SMAT_ERR_INVALID_ARG, "an activation is applied to x in 8 bits only");
  if ((a->accumulate & ~(SMAT_ACCUMULATE_DW | SMAT_ACCUMULATE_DB)) || a->reserved)
    return lfail(SMAT_ERR_UNSUPPORTED, "unknown accumulate flags 0x%x", a->accumulate);
  const size_t es = elem_of(a->dtype);
  const Mat mats[] = {
      {"dw", a->dw, n, k, a->lddw, es, true},
      {"db", a->db, a->db ? 1 : 0, n, n, es, true},
      {"dy", a->dy, m, n, a->lddy, es, false},
      {"x", a->x, n && a->x ? m : 0, k, a->ldx, es, false},
      {"q", a->q, n && a->q ? m : 0, k, a->ldq, 1, false},
      {"e", a->e, n && a->e ? m : 0, groups_of(k), a->lde, 1, false},
  };
  st = check_mats(mats, 6, -1, -1);
  if (st != SMAT_OK || n == 0) return st;
  const Operands ops = operands(a);
  st = check_workspace(d_workspace, workspace_bytes, ops.bytes());
  if (st != SMAT_OK) return st;
  int sms = 1;
  st = device_sms(&sms);
  if (st != SMAT_OK) return st;
  if (k > 0 && few_rows(a)) {
    const Outer o = {a->dy, a->x, a->q, a->e, a->dw, a->db, m, k, n, a->lddy, a->ldx, a->ldq, a->lde, a->lddw, a->act,
                     (a->accumulate & SMAT_ACCUMULATE_DW) != 0, (a->accumulate & SMAT_ACCUMULATE_DB) != 0};
    return cuda_status(launch_outer(o, a->dtype, sms, stream), "grad_weight launch");
  }
  const bool bf16 = a->dtype == SMAT_BF16;
  Prepare first = {};
  Product p = {};
  p.mode = kGradWeight;
  p.dtype = a->dtype;
  p.b = d_workspace, p.ldb = ld_of(k);  // x^ in 8 bits: its values
  p.I = n, p.J = k, p.L = m;
  p.out = a->dw, p.ldo = a->lddw;
  p.accumulate = a->accumulate & SMAT_ACCUMULATE_DW;
  if (a->db && bf16 && ops.sums) {
    first.sums = {a->dy, (float*)d_workspace, m, n, a->lddy, sum_shares(m), false};
    p.db = a->db;
    p.add_db = a->accumulate & SMAT_ACCUMULATE_DB;
  } else if (a->db) {
    st = cuda_status(launch_row_sums(a->dy, a->lddy, a->db, m, n, a->dtype, a->accumulate & SMAT_ACCUMULATE_DB, sms,
                                     stream), "row sums launch");
    if (st != SMAT_OK) return st;
  }
  if (k == 0) return SMAT_OK;
  if (ops.values && bf16) {
    first.unpack = {a->q, a->e, d_workspace, m, k, a->ldq, a->lde, ld_of(k), 0, false};
  } else if (ops.values) {
    st = cuda_status(launch_unpack8(a->q, a->ldq, a->e, a->lde, nullptr, 0, d_workspace, ld_of(k), m, k, a->dtype,
                                    a->act, sms, stream), "unpack launch");
    if (st != SMAT_OK) return st;
  }
  return run_product(p, ops, first, (char*)d_workspace + ops.values, a->act, sms, stream, "grad_weight launch");
}

smat_status smat_linear(const smat_linear_args* a, void* d_workspace, size_t workspace_bytes, smat_stream_t stream) {
  return guarded([&] { return linear(a, d_workspace, workspace_bytes, stream); });
}
smat_status smat_grad_input(const smat_grad_input_args* a, void* d_workspace, size_t workspace_bytes,
                            smat_stream_t stream) {
  return guarded([&] { return grad_input(a, d_workspace, workspace_bytes, stream); });
}
smat_status smat_grad_weight(const smat_grad_weight_args* a, void* d_workspace, size_t workspace_bytes,
                             smat_stream_t stream) {
  return guarded([&] { return grad_weight(a, d_workspace, workspace_bytes, stream); });
}

smat_status smat_linear_poll_errors(smat_stream_t stream, int32_t* errors_out) {
  if (!errors_out) return lfail(SMAT_ERR_INVALID_ARG, "errors_out is NULL");
  int v = 0;
  const smat_status st = cuda_status(read_errors(&v, stream), "error flag read");
  if (st == SMAT_OK) *errors_out = v;
  return st;
}

static smat_status elementwise(const char* what, const void* dy, int64_t lddy, const int8_t* q, int64_t ldq,
                               const uint8_t* e, int64_t lde, void* out, int64_t ldout, int64_t rows, int64_t cols,
                               int32_t dtype, int32_t act, bool pack, bool slope, smat_stream_t stream) {
  smat_status st = check_sizes(rows, cols, 0, dtype, act);
  if (st != SMAT_OK) return st;
  const size_t es = elem_of(dtype);
  const Mat mats[] = {
      {pack ? "x" : "out", out, rows, cols, ldout, es, !pack},
      {"q", q, rows, cols, ldq, 1, pack},
      {"e", e, rows, groups_of(cols), lde, 1, pack},
      {"dy", dy, slope ? rows : 0, cols, lddy, es, false},
  };
  st = check_mats(mats, 4, -1, -1);
  if (st != SMAT_OK || rows == 0 || cols == 0) return st;
  int sms = 1;
  st = device_sms(&sms);
  if (st != SMAT_OK) return st;
  return cuda_status(pack ? launch_pack8(out, ldout, const_cast<int8_t*>(q), ldq, const_cast<uint8_t*>(e), lde, rows,
                                         cols, dtype, sms, stream)
                          : launch_unpack8(q, ldq, e, lde, dy, lddy, out, ldout, rows, cols, dtype, act, sms, stream),
                     what);
}

smat_status smat_pack8(const void* x, int64_t ldx, int8_t* q, int64_t ldq, uint8_t* e, int64_t lde, int64_t rows,
                       int64_t cols, int32_t dtype, smat_stream_t stream) {
  return guarded([&] { return elementwise("pack8 launch", nullptr, 0, q, ldq, e, lde, const_cast<void*>(x), ldx, rows, cols, dtype,
                     SMAT_ACT_NONE, true, false, stream); });
}

smat_status smat_unpack8(const int8_t* q, int64_t ldq, const uint8_t* e, int64_t lde, void* out, int64_t ldout,
                         int64_t rows, int64_t cols, int32_t dtype, int32_t act, smat_stream_t stream) {
  return guarded([&] { return elementwise("unpack8 launch", nullptr, 0, q, ldq, e, lde, out, ldout, rows, cols, dtype, act, false, false,
                     stream); });
}

smat_status smat_act_grad8(const void* dy, int64_t lddy, const int8_t* q, int64_t ldq, const uint8_t* e, int64_t lde,
                           void* out, int64_t ldout, int64_t rows, int64_t cols, int32_t dtype, int32_t act,
                           smat_stream_t stream) {
  return guarded([&] { return elementwise("act_grad8 launch", dy, lddy, q, ldq, e, lde, out, ldout, rows, cols, dtype, act, false, true,
                     stream); });
}

}  // extern "C"
