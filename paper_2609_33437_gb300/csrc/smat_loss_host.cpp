// Host side of the loss over a vocabulary (include/smat.h): argument checks, pieces of the vocabulary, workspace, launches.
//
// bf16, forward: the logits' product reduces each of its tiles to a row's largest value and sum of exponentials, a last kernel
// joins these. Back: a piece of the logits is made again and leaves its product as d in bf16 (pieces of kPieceBytes), which the
// products of dx (summed over the pieces in fp32) and of dW's rows then read. fp32 logits are written a piece at a time, and
// kernels of their own read them.

#include <algorithm>

#include <cuda_runtime.h>

#include "smat.h"
#include "smat_checks.h"
#include "smat_loss.h"

using namespace smat;
using namespace smat::lin;

namespace {

// As the linear layers: the vocabulary is cut into at most 65535 tiles of 64 or more columns.
constexpr int64_t kMaxSize = (int64_t(1) << 31) - (1 << 16);
constexpr int64_t kMaxCols = int64_t(65535) * 64;

// A piece of the vocabulary: as many columns as d's bytes allow, at least kPieceCols.
constexpr int64_t kPieceBytes = int64_t(192) << 20, kPieceCols = 2048;
// A piece of W that is copied because its rows do not start on 16 bytes.
constexpr int64_t kCopyBytes = int64_t(64) << 20;
// A piece of W cut for the tensor cores (fp32), which with few rows takes more space than d: 64 x 4096 of 151936 words 3.7 GB
// beside 38 MB if taken whole. Smaller pieces cost more at their ends (384 MiB: 515 x 4096 x 32000 forward 955 us for 824).
constexpr int64_t kCutBytes = int64_t(1) << 30;

bool sizes_fit(int64_t rows, int64_t k, int64_t n) {
  return rows >= 0 && rows <= kMaxSize && k >= 0 && k <= kMaxCols && n >= 1 && n <= kMaxCols;
}

smat_status check_sizes(int64_t rows, int64_t k, int64_t n, int32_t dtype) {
  if (!sizes_fit(rows, k, n))
    return lfail(SMAT_ERR_INVALID_ARG, "sizes out of range: %lld rows, k %lld, n %lld", (long long)rows, (long long)k,
                 (long long)n);
  if (dtype != SMAT_F32 && dtype != SMAT_BF16) return lfail(SMAT_ERR_UNSUPPORTED, "dtype %d not supported", dtype);
  return SMAT_OK;
}

// n in pieces of one length (the last may be shorter), a multiple of 256, of at most `most` columns where that is not below
// kPieceCols.
int64_t piece_of(int64_t n, int64_t most) {
  if (most < kPieceCols) most = kPieceCols;
  if (n <= most) return n;
  const int64_t pieces = (n + most - 1) / most;
  return std::min(n, ((n + pieces - 1) / pieces + 255) / 256 * 256);
}

// The most columns of a piece whose d, or fp32 logits, have `rows` rows.
int64_t most_of(int64_t rows, int64_t k, int64_t n, int32_t dtype, const Operand& w) {
  int64_t most = kPieceBytes / ((int64_t)elem_of(dtype) * rows);
  if (w.copied) most = std::min(most, kCopyBytes / (2 * ld_of(k)));
  Product p = {};
  p.mode = kForward, p.dtype = dtype, p.I = rows, p.J = n, p.L = k;
  if (dtype == SMAT_F32 && f32_on_tensor_cores(p)) most = std::min(most, kCutBytes / (6 * parts_ld(k)));
  return most;
}

// Places in the workspace, in turn.
struct Space {
  size_t at = 0;
  size_t take(size_t bytes) {
    const size_t was = at;
    at += up(bytes);
    return was;
  }
};

size_t product_bytes(const Product& p, int sms) {
  size_t bytes = 0;
  const cudaError_t e = p.dtype == SMAT_BF16 ? tc_workspace(p, sms, &bytes) : f32_workspace(p, sms, &bytes);
  return e == cudaSuccess ? bytes : 0;
}
cudaError_t launch_product(const Product& p, int sms, void* workspace, cudaStream_t s) {
  return p.dtype == SMAT_BF16 ? launch_tc(p, sms, workspace, s) : launch_f32(p, sms, workspace, s);
}

Product product(int mode, int dtype, int64_t I, int64_t J, int64_t L) {
  Product p = {};
  p.mode = mode, p.dtype = dtype, p.I = I, p.J = J, p.L = L;
  return p;
}

// W's rows from `first` on as a product reads them: where they are, or their copy.
struct Rows {
  const void* p;
  int64_t ld;
};
cudaError_t rows_of(const void* w, int64_t ldw, const Operand& o, int64_t first, int64_t count, int64_t k, size_t elem, void* copy,
                    int sms, cudaStream_t s, Rows* out) {
  const char* from = (const char*)w + (size_t)first * (size_t)ldw * elem;
  if (!o.copied) {
    *out = {from, o.ld};
    return cudaSuccess;
  }
  *out = {copy, ld_of(k)};
  Prepare first_of = {};
  first_of.copy[0] = {from, copy, count, k, ldw, ld_of(k), 0};
  return launch_prepare(first_of, SMAT_ACT_NONE, sms, s);
}

// ---- forward ----

struct ForwardPlan {
  Operand x, w;
  int64_t piece, slots;                    // slots: of every piece but the last, or 1
  size_t partials, picked, xcopy, wcopy, z, parts, bytes;
};

loss::Logits logits(const smat_token_loss_args* a, int64_t cols) {
  loss::Logits p = {};
  p.rows = a->rows, p.k = a->k, p.cols = cols;
  return p;
}

smat_status plan(const smat_token_loss_args* a, int sms, ForwardPlan* out) {
  ForwardPlan f = {};
  const bool bf = a->dtype == SMAT_BF16;
  const int64_t m = a->rows, k = a->k, n = a->n;
  f.x = operand(a->x, m, k, a->ldx, a->dtype);
  f.w = operand(a->w, n, k, a->ldw, a->dtype);
  f.piece = n;
  if (!bf)
    f.piece = piece_of(n, most_of(m, k, n, a->dtype, f.w));
  else if (f.w.copied)
    f.piece = piece_of(n, kCopyBytes / (2 * ld_of(k)));
  const int64_t pieces = (n + f.piece - 1) / f.piece, last = n - (pieces - 1) * f.piece;
  int64_t last_slots = 1;
  f.slots = 1;
  if (bf) {
    cudaError_t e = loss::logit_slots(logits(a, f.piece), sms, &f.slots);
    if (e == cudaSuccess) e = loss::logit_slots(logits(a, last), sms, &last_slots);
    if (e != cudaSuccess) return cuda_status(e, "plan of the logits' product");
  }
  Space s;
  f.partials = s.take(sizeof(float2) * (size_t)m * (size_t)((pieces - 1) * f.slots + last_slots));
  f.picked = s.take(sizeof(float) * (size_t)m);
  f.xcopy = s.take(operand_bytes(f.x));
  f.wcopy = s.take(f.w.copied ? copy_bytes(f.piece, k, 2) : 0);
  f.z = s.take(bf ? 0 : copy_bytes(m, f.piece, 4));
  if (!bf)
    f.parts = s.take(std::max(product_bytes(product(kForward, a->dtype, m, f.piece, k), sms),
                              product_bytes(product(kForward, a->dtype, m, last, k), sms)));
  f.bytes = s.at;
  *out = f;
  return SMAT_OK;
}

smat_status forward(const smat_token_loss_args* a, void* d_workspace, size_t workspace_bytes, cudaStream_t s) {
  if (!a) return lfail(SMAT_ERR_INVALID_ARG, "args is NULL");
  smat_status st = check_sizes(a->rows, a->k, a->n, a->dtype);
  if (st != SMAT_OK) return st;
  if (a->reserved) return lfail(SMAT_ERR_UNSUPPORTED, "reserved must be 0");
  const int64_t m = a->rows, k = a->k, n = a->n;
  const size_t es = elem_of(a->dtype);
  const Mat mats[] = {
      {"loss", a->loss, m ? 1 : 0, m, m, 4, true},
      {"lse", a->lse, m ? 1 : 0, m, m, 4, true},
      {"x", a->x, m, k, a->ldx, es, false},
      {"w", a->w, m ? n : 0, k, a->ldw, es, false},
      {"targets", a->targets, m ? 1 : 0, m, m, 8, false},
  };
  st = check_mats(mats, 5, -1, -1);
  if (st != SMAT_OK || m == 0) return st;
  int sms = 1;
  st = device_sms(&sms);
  if (st != SMAT_OK) return st;
  ForwardPlan f;
  st = plan(a, sms, &f);
  if (st == SMAT_OK) st = check_workspace(d_workspace, workspace_bytes, f.bytes);
  if (st != SMAT_OK) return st;
  char* ws = (char*)d_workspace;
  const bool bf = a->dtype == SMAT_BF16;
  float2* partials = (float2*)(ws + f.partials);
  float* picked = (float*)(ws + f.picked);
  Rows x;
  cudaError_t e = rows_of(a->x, a->ldx, f.x, 0, m, k, es, ws + f.xcopy, sms, s, &x);
  int64_t slots = 0;
  for (int64_t c = 0; e == cudaSuccess && c < n; c += f.piece) {
    const int64_t cols = std::min(f.piece, n - c);
    Rows w;
    e = rows_of(a->w, a->ldw, f.w, c, cols, k, es, ws + f.wcopy, sms, s, &w);
    if (e != cudaSuccess) break;
    if (bf) {
      loss::Logits p = logits(a, cols);
      p.x = x.p, p.ldx = x.ld, p.w = w.p, p.ldw = w.ld;
      p.targets = a->targets, p.partials = partials + slots * m, p.picked = picked, p.first_col = c;
      int64_t made = 0;
      e = loss::logit_slots(p, sms, &made);
      if (e == cudaSuccess) e = loss::launch_logits(p, sms, s);
      slots += made;
    } else {
      Product p = product(kForward, a->dtype, m, cols, k);
      p.a = x.p, p.lda = x.ld, p.b = w.p, p.ldb = w.ld, p.out = ws + f.z, p.ldo = ld_of(f.piece);
      e = launch_product(p, sms, ws + f.parts, s);
      if (e == cudaSuccess)
        e = loss::launch_row_part((const float*)p.out, p.ldo, m, cols, c, a->targets, partials + slots * m, picked, sms, s);
      ++slots;
    }
  }
  if (e == cudaSuccess) e = loss::launch_join({partials, picked, a->targets, a->loss, a->lse, m, slots, n, a->ignore}, sms, s);
  return cuda_status(e, "token_loss launch");
}

// ---- gradient ----

struct GradPlan {
  Operand w;
  int64_t piece;
  int splits;    // of dx's sum, bf16; each has `slab` rows of `sums`
  int64_t slab;
  bool cut;  // fp32: the products share operands that are cut for the tensor cores
  size_t count, place, info, x, d, sums, more, wcopy, cut_x, cut_w, cut_d, parts, bytes;
};

// bf16 with so few rows that all of them twice fit one tile of the products: d is kept as two bf16 numbers, its nearest and what that
// lacks, as rows of their own. Few rows' roundings of d do not cancel (one row: dx and dW off by up to 2^-8 beside their own
// rounding), and the second rows are free. From there on d is one bf16 number: 8192 x 4096 x 32000 dx and dW off by 0.0023 in
// the norm, 0.0017 of it their own rounding; a second one would double two of the four products.
constexpr int64_t kTwiceRows = 128;
int64_t rows_of_d(const smat_token_loss_grad_args* a) {
  return a->dtype == SMAT_BF16 && a->rows <= kTwiceRows ? 2 * a->rows : a->rows;
}

// The three products of a piece.
void products(const smat_token_loss_grad_args* a, const GradPlan& g, int64_t cols, Product* p) {
  const bool bf = a->dtype == SMAT_BF16;
  const int64_t rows = rows_of_d(a);
  p[0] = product(bf ? kLogitGrad : kForward, a->dtype, rows, cols, a->k);
  p[1] = product(bf ? kGradInputSum : kGradInput, a->dtype, rows, a->k, cols);
  p[1].splits = g.splits, p[1].slab = g.slab;
  p[2] = product(bf ? kGradWeightRows : kGradWeight, a->dtype, cols, a->k, rows);
}

smat_status plan(const smat_token_loss_grad_args* a, int sms, GradPlan* out) {
  GradPlan g = {};
  const bool bf = a->dtype == SMAT_BF16;
  const size_t es = elem_of(a->dtype);
  const int64_t m = rows_of_d(a), k = a->k, n = a->n;
  g.w = operand(a->w, n, k, a->ldw, a->dtype);
  g.piece = piece_of(n, most_of(m, k, n, a->dtype, g.w));
  const int64_t pieces = (n + g.piece - 1) / g.piece, last = n - (pieces - 1) * g.piece;
  g.splits = 1, g.slab = m;
  if (bf && a->dx) {
    const cudaError_t e = grad_input_splits(product(kGradInputSum, a->dtype, m, k, g.piece), &g.splits);
    if (e != cudaSuccess) return cuda_status(e, "plan of dx's product");
    if (g.splits > 1) g.slab = (m + 255) / 256 * 256;
  }
  Space s;
  g.count = s.take(sizeof(int));
  g.place = s.take(sizeof(int) * (size_t)m);
  g.info = s.take(sizeof(LossRow) * (size_t)m);
  g.x = s.take(copy_bytes(m, k, es));
  g.d = s.take(copy_bytes(m, g.piece, es));
  g.sums = s.take(a->dx ? copy_bytes(g.splits * g.slab, k, 4) : 0);
  g.more = s.take(a->dx && !bf && pieces > 1 ? copy_bytes(m, k, 4) : 0);
  g.wcopy = s.take(g.w.copied ? copy_bytes(g.piece, k, 2) : 0);
  size_t parts = 0;
  g.cut = !bf;
  for (int64_t cols : {g.piece, last}) {
    Product p[3];
    products(a, g, cols, p);
    for (const Product& q : p) g.cut = g.cut && f32_on_tensor_cores(q);
  }
  for (int64_t cols : {g.piece, last}) {
    Product p[3];
    products(a, g, cols, p);
    for (int i = 0; i < 3; ++i) {
      if (i > 0 && !(i == 1 ? a->dx : a->dw)) continue;
      size_t bytes = 0;
      if (!g.cut)
        bytes = product_bytes(p[i], sms);
      else if (f32_parts_workspace(p[i], sms, &bytes) != cudaSuccess)
        bytes = 0;
      parts = std::max(parts, bytes);
    }
  }
  if (g.cut) {
    auto cut = [&](int64_t rows, int64_t cols) {
      return s.take(parts_bytes(rows, cols) + up(sizeof(uint32_t) * (size_t)parts_flags(rows, cols, sms)));
    };
    g.cut_x = cut(m, k), g.cut_w = cut(g.piece, k), g.cut_d = cut(m, g.piece);
  }
  g.parts = s.take(parts);
  g.bytes = s.at;
  *out = g;
  return SMAT_OK;
}

smat_status backward(const smat_token_loss_grad_args* a, void* d_workspace, size_t workspace_bytes, cudaStream_t s) {
  if (!a) return lfail(SMAT_ERR_INVALID_ARG, "args is NULL");
  smat_status st = check_sizes(a->rows, a->k, a->n, a->dtype);
  if (st != SMAT_OK) return st;
  if (a->accumulate != 0 && a->accumulate != 1)
    return lfail(SMAT_ERR_UNSUPPORTED, "unknown accumulate value %d", a->accumulate);
  const int64_t m = a->rows, k = a->k, n = a->n;
  const size_t es = elem_of(a->dtype);
  const Mat mats[] = {
      {"dx", a->dx, a->dx ? m : 0, k, a->lddx, es, true},
      {"dw", a->dw, a->dw ? n : 0, k, a->lddw, es, true},
      {"g", a->g, m ? 1 : 0, m, m, 4, false},
      {"x", a->x, m, k, a->ldx, es, false},
      {"w", a->w, m ? n : 0, k, a->ldw, es, false},
      {"targets", a->targets, m ? 1 : 0, m, m, 8, false},
      {"lse", a->lse, m ? 1 : 0, m, m, 4, false},
  };
  st = check_mats(mats, 7, -1, -1);
  if (st != SMAT_OK || k == 0 || (!a->dx && !a->dw)) return st;
  int sms = 1;
  st = device_sms(&sms);
  if (st != SMAT_OK) return st;
  if (m == 0) {  // dw of no rows
    if (!a->dw || a->accumulate) return SMAT_OK;
    return cuda_status(cudaMemset2DAsync(a->dw, (size_t)a->lddw * es, 0, (size_t)k * es, (size_t)n, s), "token_loss_grad of no rows");
  }
  GradPlan f;
  st = plan(a, sms, &f);
  if (st == SMAT_OK) st = check_workspace(d_workspace, workspace_bytes, f.bytes);
  if (st != SMAT_OK) return st;
  char* ws = (char*)d_workspace;
  const bool bf = a->dtype == SMAT_BF16;
  int *count = (int*)(ws + f.count), *place = (int*)(ws + f.place);
  LossRow* info = (LossRow*)(ws + f.info);
  const int64_t ldk = ld_of(k), ldd = ld_of(f.piece);
  float *sums = (float*)(ws + f.sums), *more = (float*)(ws + f.more);
  const loss::Index index = {a->targets, a->g, a->lse, a->w, a->ldw, m, n, a->ignore, place, info, count, rows_of_d(a) > m};
  cudaError_t e = loss::launch_index(index, s);
  if (e == cudaSuccess) e = loss::launch_gather(index, a->x, a->ldx, ws + f.x, ldk, k, a->dtype, !bf && !f.cut, sms, s);
  auto parts_at = [&](size_t at, int64_t rows, int64_t cols) {
    return Parts{ws + at, (uint32_t*)(ws + at + parts_bytes(rows, cols)), parts_flags(rows, cols, sms)};
  };
  for (int64_t c = 0; e == cudaSuccess && c < n; c += f.piece) {
    const int64_t cols = std::min(f.piece, n - c);
    Rows w;
    e = rows_of(a->w, a->ldw, f.w, c, cols, k, es, ws + f.wcopy, sms, s, &w);
    if (e != cudaSuccess) break;
    Product p[3];
    products(a, f, cols, p);
    for (Product& q : p) q.count = count, q.loss_rows = info, q.first_col = c, q.halves = index.twice;
    p[0].a = ws + f.x, p[0].lda = ldk, p[0].b = w.p, p[0].ldb = w.ld, p[0].out = ws + f.d, p[0].ldo = ldd;
    p[1].a = ws + f.d, p[1].lda = ldd, p[1].b = w.p, p[1].ldb = w.ld, p[1].ldo = ldk;
    p[1].out = bf || c == 0 ? sums : more, p[1].accumulate = bf && c > 0;
    p[2].a = ws + f.d, p[2].lda = ldd, p[2].b = ws + f.x, p[2].ldb = ldk, p[2].ldo = a->lddw, p[2].accumulate = a->accumulate;
    p[2].out = a->dw ? (char*)a->dw + (size_t)c * (size_t)a->lddw * es : nullptr;
    if (f.cut) {
      const Parts px = parts_at(f.cut_x, m, k), pw = parts_at(f.cut_w, cols, k), pd = parts_at(f.cut_d, m, cols);
      const Uncut rows = {c == 0 ? (const float*)(ws + f.x) : nullptr, m, k, ldk, count, px};
      e = launch_cut(rows, {(const float*)w.p, cols, k, w.ld, nullptr, pw}, sms, s);
      if (e == cudaSuccess) e = launch_f32_parts(p[0], pw, px, sms, ws + f.parts, s);
      if (e == cudaSuccess) e = loss::launch_row_grad_cut((float*)(ws + f.d), ldd, m, cols, c, info, count, pd, s);
      if (e == cudaSuccess && a->dx) e = launch_f32_parts(p[1], pw, pd, sms, ws + f.parts, s);
      if (e == cudaSuccess && a->dx && c > 0) e = loss::launch_add(sums, more, ldk, m, k, sms, s);
      if (e == cudaSuccess && a->dw) e = launch_f32_parts(p[2], px, pd, sms, ws + f.parts, s);
      continue;
    }
    e = launch_product(p[0], sms, ws + f.parts, s);
    if (e == cudaSuccess && !bf) e = loss::launch_row_grad((float*)(ws + f.d), ldd, m, cols, c, info, count, sms, s);
    if (e == cudaSuccess && a->dx) e = launch_product(p[1], sms, ws + f.parts, s);
    if (e == cudaSuccess && a->dx && !bf && c > 0) e = loss::launch_add(sums, more, ldk, m, k, sms, s);
    if (e == cudaSuccess && a->dw) e = launch_product(p[2], sms, ws + f.parts, s);
  }
  if (e == cudaSuccess && a->dx)
    e = loss::launch_scatter({sums, ldk, f.splits, f.slab * ldk}, index, a->dx, a->lddx, k, a->dtype, sms, s);
  return cuda_status(e, "token_loss_grad launch");
}

// A size query: 0 for what the call itself refuses.
template <class Args, class Plan>
size_t workspace_of(const Args* a, Plan f) {
  int sms = 1;
  if (!a || !sizes_fit(a->rows, a->k, a->n) || a->rows == 0 || (a->dtype != SMAT_F32 && a->dtype != SMAT_BF16) ||
      device_sms(&sms) != SMAT_OK || plan(a, sms, &f) != SMAT_OK)
    return 0;
  return f.bytes;
}

}  // namespace

extern "C" {

size_t smat_token_loss_workspace_bytes(const smat_token_loss_args* a) { return workspace_of(a, ForwardPlan()); }
size_t smat_token_loss_grad_workspace_bytes(const smat_token_loss_grad_args* a) {
  return a && (a->k == 0 || (!a->dx && !a->dw)) ? 0 : workspace_of(a, GradPlan());
}

smat_status smat_token_loss(const smat_token_loss_args* args, void* d_workspace, size_t workspace_bytes, smat_stream_t stream) {
  return guarded([&] { return forward(args, d_workspace, workspace_bytes, (cudaStream_t)stream); });
}
smat_status smat_token_loss_grad(const smat_token_loss_grad_args* args, void* d_workspace, size_t workspace_bytes,
                                 smat_stream_t stream) {
  return guarded([&] { return backward(args, d_workspace, workspace_bytes, (cudaStream_t)stream); });
}

}  // extern "C"
