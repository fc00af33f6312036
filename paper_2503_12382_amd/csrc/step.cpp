// C entry points of the step that follows a gradient: argument checks, then the
// launchers.  Nothing here touches the device before the checks have passed.

#include <algorithm>
#include <cmath>
#include <exception>
#include <limits>
#include <vector>

#include "step.h"

namespace {

using reno::fail_thread;

bool is_type(int64_t t) { return t == RENO_T_FP32 || t == RENO_T_BF16 || t == RENO_T_FP16; }
int64_t size_of(int64_t type) { return type == RENO_T_FP32 ? 4 : 2; }
bool aligned(const void* p, int64_t to) { return (uintptr_t)p % (uintptr_t)to == 0; }

// Memory that a call reads or writes.
struct Range {
  uintptr_t begin, end;
  bool written;
};

// Whether anything written lies in anything else.
bool overlap(std::vector<Range>& r) {
  std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
  uintptr_t any = 0, written = 0;   // ends of what began before
  for (const Range& x : r) {
    if (x.begin < (x.written ? any : written)) return true;
    any = std::max(any, x.end);
    if (x.written) written = std::max(written, x.end);
  }
  return false;
}

void add(std::vector<Range>& r, const void* p, int64_t bytes, bool written) {
  if (p && bytes) r.push_back({(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, written});
}

reno_status check_list(const void* list, int64_t count) {
  if (count < 0 || count > RENO_STEP_MAX_TENSORS)
    return fail_thread(RENO_E_INVALID, "count must be in [0, RENO_STEP_MAX_TENSORS]");
  if (!list && count) return fail_thread(RENO_E_INVALID, "null list");
  return RENO_OK;
}

reno_status check_grads(const reno_gradient* g, int64_t count) {
  const reno_status s = check_list(g, count);
  if (s != RENO_OK) return s;
  for (int64_t i = 0; i < count; ++i) {
    if (g[i].n < 0 || g[i].n >= (int64_t(1) << 40)) return fail_thread(RENO_E_INVALID, "n must be in [0, 2^40)");
    if (!is_type(g[i].type)) return fail_thread(RENO_E_INVALID, "type must be a reno_type");
    if (!g[i].grad && g[i].n) return fail_thread(RENO_E_INVALID, "null gradient");
    if (!aligned(g[i].grad, size_of(g[i].type)))
      return fail_thread(RENO_E_INVALID, "an operand is not aligned to its type");
  }
  return RENO_OK;
}

bool is_scale(double x) { return x > 0 && std::isfinite(x); }

reno_status done(hipError_t e) {
  return e == hipSuccess ? RENO_OK : fail_thread(RENO_E_HIP, hipGetErrorString(e));
}

// f(), with what it throws (host memory for the overlap check) as a status.
template <typename F>
reno_status guarded(const F& f) {
  try {
    return f();
  } catch (const std::exception&) {
    return fail_thread(RENO_E_NOMEM, "out of host memory");
  }
}

reno_status check_params(const reno_parameter* p, int64_t count) {
  const reno_status s = check_list(p, count);
  if (s != RENO_OK) return s;
  for (int64_t i = 0; i < count; ++i) {
    const reno_parameter& x = p[i];
    if (x.n < 0 || x.n >= (int64_t(1) << 40)) return fail_thread(RENO_E_INVALID, "n must be in [0, 2^40)");
    if (!is_type(x.type)) return fail_thread(RENO_E_INVALID, "type must be a reno_type");
    if (x.grad_type != x.type && x.grad_type != RENO_T_FP32)
      return fail_thread(RENO_E_INVALID, "grad_type must be type or RENO_T_FP32");
    if (x.master && x.type == RENO_T_FP32) return fail_thread(RENO_E_INVALID, "fp32 weights have no fp32 copy");
    if (x.n && (!x.param || !x.grad || !x.exp_avg || !x.exp_avg_sq)) return fail_thread(RENO_E_INVALID, "null operand");
    if (!aligned(x.param, size_of(x.type)) || !aligned(x.grad, size_of(x.grad_type)) || !aligned(x.master, 4) ||
        !aligned(x.exp_avg, 4) || !aligned(x.exp_avg_sq, 4))
      return fail_thread(RENO_E_INVALID, "an operand is not aligned to its type");
  }
  return RENO_OK;
}

}  // namespace

extern "C" {

reno_status reno_grad_workspace(const reno_gradient* g, int64_t count, int64_t* bytes_host) {
  const reno_status s = check_grads(g, count);
  if (s != RENO_OK) return s;
  if (!bytes_host) return fail_thread(RENO_E_INVALID, "null argument");
  *bytes_host = 8 * reno::norm_parts(g, count);
  return RENO_OK;
}

reno_status reno_grad_norm(const reno_gradient* g, int64_t count, double scale, float* norm, void* ws, int64_t bytes,
                           void* stream) {
  const reno_status s = check_grads(g, count);
  if (s != RENO_OK) return s;
  if (!is_scale(scale)) return fail_thread(RENO_E_INVALID, "scale must be positive and finite");
  if (!norm || !aligned(norm, 4)) return fail_thread(RENO_E_INVALID, "norm must be a float on the device");
  const int64_t need = 8 * reno::norm_parts(g, count);
  if (bytes < need) return fail_thread(RENO_E_INVALID, "workspace too small");
  if (need && (!ws || !aligned(ws, 256))) return fail_thread(RENO_E_INVALID, "workspace must be 256-byte aligned");
  return guarded([&] {
    std::vector<Range> r;
    add(r, norm, 4, true);
    add(r, ws, need, true);   // blocks would write partial sums over what others still read
    for (int64_t i = 0; i < count; ++i) add(r, g[i].grad, g[i].n * size_of(g[i].type), false);
    if (overlap(r)) return fail_thread(RENO_E_INVALID, "an output overlaps another operand");
    return done(reno::launch_norm(g, count, scale, norm, static_cast<double*>(ws), static_cast<hipStream_t>(stream)));
  });
}

reno_status reno_grad_clip(const reno_gradient* g, int64_t count, const float* norm, double scale, double max_norm,
                           void* stream) {
  const reno_status s = check_grads(g, count);
  if (s != RENO_OK) return s;
  if (!is_scale(scale)) return fail_thread(RENO_E_INVALID, "scale must be positive and finite");
  if (!(max_norm > 0)) return fail_thread(RENO_E_INVALID, "max_norm must be positive");
  if (!norm || !aligned(norm, 4)) return fail_thread(RENO_E_INVALID, "norm must be a float on the device");
  return guarded([&] {
    std::vector<Range> r;
    add(r, norm, 4, false);
    for (int64_t i = 0; i < count; ++i) {
      const int64_t n = g[i].n * size_of(g[i].type);
      if (!g[i].out && n) return fail_thread(RENO_E_INVALID, "null out");
      if (!aligned(g[i].out, size_of(g[i].type))) return fail_thread(RENO_E_INVALID, "an operand is not aligned to its type");
      add(r, g[i].out, n, true);
      if (g[i].out != g[i].grad) add(r, g[i].grad, n, false);
    }
    if (overlap(r)) return fail_thread(RENO_E_INVALID, "an output overlaps another operand");
    return done(reno::launch_clip(g, count, norm, scale, max_norm, static_cast<hipStream_t>(stream)));
  });
}

reno_status reno_adamw_step(const reno_parameter* p, int64_t count, const reno_adamw* how, void* stream) {
  const reno_status s = check_params(p, count);
  if (s != RENO_OK) return s;
  if (!how) return fail_thread(RENO_E_INVALID, "null argument");
  for (double x : {how->lr, how->weight_decay})
    if (!(x >= 0) || !std::isfinite((float)x)) return fail_thread(RENO_E_INVALID, "lr and weight_decay must be 0 or more and finite");
  for (double x : {how->beta1, how->beta2})
    if (!(x >= 0) || !((float)x < 1)) return fail_thread(RENO_E_INVALID, "betas must be in [0, 1)");
  if (!(how->eps > 0) || !std::isnormal((float)how->eps)) return fail_thread(RENO_E_INVALID, "eps must be a positive normal float");
  if (!is_scale(how->scale)) return fail_thread(RENO_E_INVALID, "scale must be positive and finite");
  if (!(how->max_norm > 0)) return fail_thread(RENO_E_INVALID, "max_norm must be positive");
  if (!how->steps || !aligned(how->steps, 4)) return fail_thread(RENO_E_INVALID, "steps must be two words on the device");
  if (!aligned(how->norm, 4) || !aligned(how->lr_factor, 4))
    return fail_thread(RENO_E_INVALID, "an operand is not aligned to its type");
  return guarded([&] {
    std::vector<Range> r;
    add(r, how->norm, 4, false);
    add(r, how->lr_factor, 4, false);
    add(r, how->steps, 8, true);
    for (int64_t i = 0; i < count; ++i) {
      const reno_parameter& x = p[i];
      add(r, x.param, x.n * size_of(x.type), true);
      add(r, x.grad, x.n * size_of(x.grad_type), false);
      add(r, x.master, x.n * 4, true);
      add(r, x.exp_avg, x.n * 4, true);
      add(r, x.exp_avg_sq, x.n * 4, true);
    }
    if (overlap(r)) return fail_thread(RENO_E_INVALID, "an output overlaps another operand");
    return done(reno::launch_adamw(p, count, *how, static_cast<hipStream_t>(stream)));
  });
}

}  // extern "C"
