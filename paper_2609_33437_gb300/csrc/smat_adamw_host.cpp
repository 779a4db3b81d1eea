// Host side of the AdamW step over many tensors (include/smat.h, "AdamW"): argument checks, the launches' tables.

#include <algorithm>
#include <cmath>
#include <vector>

#include <cuda_runtime.h>

#include "smat.h"
#include "smat_adamw.h"
#include "smat_checks.h"

using namespace smat;
using namespace smat::lin;

namespace {

constexpr int64_t kMaxNumel = int64_t(1) << 40;
constexpr int32_t kMaxTensors = 1 << 20;

int64_t groups_of(int64_t numel) { return (numel + adamw::kGroup - 1) / adamw::kGroup; }

// -1: a size or their number is out of range
int64_t places_of(const int64_t* numels, int32_t n) {
  if (n < 0 || n > kMaxTensors || (n > 0 && !numels)) return -1;
  int64_t groups = 0;
  for (int32_t k = 0; k < n; ++k) {
    if (numels[k] < 0 || numels[k] > kMaxNumel) return -1;
    groups += groups_of(numels[k]);
  }
  return groups > (int64_t(1) << 40) ? -1 : groups * adamw::kGroup;
}

struct Range {
  uintptr_t begin, end;
  bool written;
  const char* name;
  int32_t index;  // or -1
  size_t elem;
};

smat_status say(const Range& r, smat_status st, const char* what) {
  if (r.index < 0) return lfail(st, "%s %s", r.name, what);
  return lfail(st, "%s[%d] %s", r.name, r.index, what);
}

smat_status check_ranges(std::vector<Range>& ranges) {
  for (const Range& r : ranges) {
    if (!r.begin) return say(r, SMAT_ERR_INVALID_ARG, "is NULL");
    if (r.begin % r.elem) return say(r, SMAT_ERR_ALIGNMENT, "is misaligned");
  }
  GpuAccess access;
  std::sort(ranges.begin(), ranges.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
  const Range *far = nullptr, *far_written = nullptr;  // of those before, the one that ends last
  for (const Range& r : ranges) {
    const Range* other = r.written ? far : far_written;
    if (other && other->end > r.begin) {
      char buf[96];
      std::snprintf(buf, sizeof(buf), "overlaps %s[%d]", other->name, other->index < 0 ? 0 : other->index);
      return say(r, SMAT_ERR_INVALID_ARG, buf);
    }
    if (!far || r.end > far->end) far = &r;
    if (r.written && (!far_written || r.end > far_written->end)) far_written = &r;
  }
  for (const Range& r : ranges) {
    const int ok = access.check((const void*)r.begin);
    if (ok < 0) return lfail(SMAT_ERR_CUDA, "no current CUDA device or pointer attributes unavailable");
    if (!ok) return say(r, SMAT_ERR_INVALID_ARG, "is not accessible from the GPU");
  }
  return SMAT_OK;
}

// What a step refuses; *any: whether it has anything to do.
smat_status check(const smat_adamw_args* a, bool* any) {
  *any = false;
  if (!a) return lfail(SMAT_ERR_INVALID_ARG, "args is NULL");
  if (a->dtype != SMAT_F32 && a->dtype != SMAT_BF16) return lfail(SMAT_ERR_UNSUPPORTED, "dtype %d not supported", a->dtype);
  if (a->grad_dtype != SMAT_F32 && a->grad_dtype != SMAT_BF16)
    return lfail(SMAT_ERR_UNSUPPORTED, "gradients' dtype %d not supported", a->grad_dtype);
  if (a->bits != 8 && a->bits != 32) return lfail(SMAT_ERR_UNSUPPORTED, "moments in %d bits not supported", a->bits);
  const double huge = 3e38;  // finite in fp32
  if (!a->scale_at && !adamw::within(a->scale, -huge, huge)) return lfail(SMAT_ERR_INVALID_ARG, "scale must be finite");
  if (const char* why = adamw::refuse(a->lr, a->beta1, a->beta2, a->eps, a->weight_decay))
    return lfail(SMAT_ERR_INVALID_ARG, "%s", why);
  if (!a->step_at && !adamw::step_fits(a->step))
    return lfail(SMAT_ERR_INVALID_ARG, "step %lld out of range", (long long)a->step);
  const int32_t n = a->n_tensors;
  const int64_t places = places_of(a->numels, n);
  if (places < 0) return lfail(SMAT_ERR_INVALID_ARG, "n_tensors or numels out of range");
  if (a->bits == 8 && places >= (int64_t(1) << 32))
    return lfail(SMAT_ERR_INVALID_ARG, "8 bits: %lld places, 2^32 and more are not numbered", (long long)places);
  if (n > 0 && (!a->params || !a->grads)) return lfail(SMAT_ERR_INVALID_ARG, "params or grads is NULL");
  if (a->bits == 32 && (a->e1 || a->e2)) return lfail(SMAT_ERR_INVALID_ARG, "e1 and e2: with 8 bits only");

  const size_t ep = elem_of(a->dtype), eg = elem_of(a->grad_dtype), em = a->bits == 8 ? 1 : 4;
  std::vector<Range> ranges;
  ranges.reserve(2 * (size_t)n + 8);
  auto add = [&](const char* name, int32_t i, const void* p, size_t bytes, bool written, size_t elem) {
    ranges.push_back({(uintptr_t)p, (uintptr_t)p + bytes, written, name, i, elem});
  };
  for (int32_t k = 0; k < n; ++k) {
    if (a->numels[k] == 0 || !a->grads[k]) continue;
    *any = true;
    add("params", k, a->params[k], (size_t)a->numels[k] * ep, true, ep);
    add("grads", k, a->grads[k], (size_t)a->numels[k] * eg, false, eg);
  }
  if (!*any) return SMAT_OK;
  add("m1", -1, a->m1, (size_t)places * em, true, 32);
  add("m2", -1, a->m2, (size_t)places * em, true, 32);
  if (a->bits == 8) {
    add("e1", -1, a->e1, (size_t)(places / adamw::kGroup), true, 1);
    add("e2", -1, a->e2, (size_t)(places / adamw::kGroup), true, 1);
  }
  if (a->scale_at) add("scale_at", -1, a->scale_at, 4, false, 4);
  if (a->lr_at) add("lr_at", -1, a->lr_at, 4, false, 4);
  if (a->step_at) add("step_at", -1, a->step_at, 8, false, 8);
  return check_ranges(ranges);
}

smat_status step(const smat_adamw_args* a, cudaStream_t stream) {
  bool any;
  smat_status st = check(a, &any);
  if (st != SMAT_OK || !any) return st;
  int sms = 1;
  st = device_sms(&sms);
  if (st != SMAT_OK) return st;
  const int32_t n = a->n_tensors;
  const size_t em = a->bits == 8 ? 1 : 4;

  adamw::Call c = {};
  const double t = (double)a->step;
  c.lr = a->lr, c.weight_decay = a->weight_decay;
  c.log_b1 = std::log(a->beta1), c.log_b2 = std::log(a->beta2);  // as `correction` has them
  const double bc2 = a->step_at ? 1.0 : adamw::correction(a->beta2, t);
  c.bc1 = a->step_at ? 1.0 : adamw::correction(a->beta1, t);
  c.c = adamw::constants_of(a->lr, a->beta1, a->beta2, a->eps, a->weight_decay, c.bc1, bc2);
  c.scale = (float)a->scale, c.scale_at = a->scale_at, c.lr_at = a->lr_at, c.step_at = a->step_at;
  c.seed_key = adamw::mix(adamw::mix((uint32_t)a->seed) ^ (uint32_t)(a->seed >> 32));
  c.key = adamw::mix(adamw::mix(c.seed_key ^ (uint32_t)a->step));

  // A launch takes what comes next of the list until its table is full or its groups would not be counted in 32 bits.
  std::vector<adamw::Entry> table;
  table.reserve(n < adamw::kMaxEntries ? n : adamw::kMaxEntries);
  int64_t group = 0, first = 0;  // of the list; the launch's first
  auto go = [&] {
    if (table.empty()) return SMAT_OK;
    c.n = (int32_t)table.size();
    c.place = first * adamw::kGroup;
    c.groups = (uint32_t)(group - first);
    c.m1 = (char*)a->m1 + (size_t)c.place * em;
    c.m2 = (char*)a->m2 + (size_t)c.place * em;
    if (a->bits == 8) c.e1 = a->e1 + first, c.e2 = a->e2 + first;
    const cudaError_t e = adamw::launch_step(c, table.data(), a->dtype, a->grad_dtype, a->bits, sms, stream);
    table.clear();
    return cuda_status(e, "AdamW launch");
  };
  for (int32_t k = 0; k < n; ++k) {
    const int64_t groups = groups_of(a->numels[k]);
    const bool there = groups > 0 && a->grads[k];
    // a tensor that is left out ends a launch: its groups belong to no entry
    if (!there && groups == 0) continue;
    if (!there || (int)table.size() == adamw::kMaxEntries || (!table.empty() && group - first + groups > UINT32_MAX)) {
      st = go();
      if (st != SMAT_OK) return st;
    }
    if (there) {
      if (table.empty()) first = group;
      const bool whole = (uintptr_t)a->params[k] % 32 == 0 && (uintptr_t)a->grads[k] % 32 == 0;
      table.push_back({a->params[k], a->grads[k], (uint32_t)(group - first),
                       (uint16_t)(groups * adamw::kGroup - a->numels[k]), (uint16_t)whole});
    }
    group += groups;
  }
  return go();
}

smat_status values(const uint8_t* q1, const uint8_t* e1, const uint8_t* q2, const uint8_t* e2, void* m1, void* r,
                   int64_t places, cudaStream_t stream) {
  if (places < 0 || places % adamw::kGroup || places > (int64_t(1) << 48))
    return lfail(SMAT_ERR_INVALID_ARG, "places %lld: a list has a multiple of %d", (long long)places, adamw::kGroup);
  if (places == 0) return SMAT_OK;
  const size_t n = (size_t)places, g = n / adamw::kGroup;
  std::vector<Range> ranges = {
      {(uintptr_t)q1, (uintptr_t)q1 + n, false, "q1", -1, 16},  {(uintptr_t)q2, (uintptr_t)q2 + n, false, "q2", -1, 16},
      {(uintptr_t)e1, (uintptr_t)e1 + g, false, "e1", -1, 1},   {(uintptr_t)e2, (uintptr_t)e2 + g, false, "e2", -1, 1},
      {(uintptr_t)m1, (uintptr_t)m1 + 2 * n, true, "m1", -1, 16}, {(uintptr_t)r, (uintptr_t)r + 2 * n, true, "r", -1, 16}};
  smat_status st = check_ranges(ranges);
  int sms = 1;
  if (st == SMAT_OK) st = device_sms(&sms);
  if (st != SMAT_OK) return st;
  return cuda_status(adamw::launch_values(q1, e1, q2, e2, m1, r, places, sms, stream), "AdamW values launch");
}

}  // namespace

extern "C" {

int64_t smat_adamw_places(const int64_t* numels, int32_t n_tensors) {
  const int64_t places = places_of(numels, n_tensors);
  return places < 0 ? 0 : places;
}

smat_status smat_adamw_check(const smat_adamw_args* args) {
  return guarded([&] {
    bool any;
    return check(args, &any);
  });
}

smat_status smat_adamw_step(const smat_adamw_args* args, smat_stream_t stream) {
  return guarded([&] { return step(args, (cudaStream_t)stream); });
}

smat_status smat_adamw_values(const uint8_t* q1, const uint8_t* e1, const uint8_t* q2, const uint8_t* e2, void* m1, void* r,
                              int64_t places, smat_stream_t stream) {
  return guarded([&] { return values(q1, e1, q2, e2, m1, r, places, (cudaStream_t)stream); });
}

}  // extern "C"
