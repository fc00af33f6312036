// C entry points of the head's training operators: argument checks, then the
// launchers.  Nothing here allocates or touches the device before the checks
// have passed.

#include <cmath>

#include "head.h"

namespace {

using reno::fail_thread;

reno_status check_head(const reno_head* p, int k) {
  if (!p) return fail_thread(RENO_E_INVALID, "null head");
  if (p->rows < 0 || p->rows >= (int64_t(1) << 31)) return fail_thread(RENO_E_INVALID, "rows must be in [0, 2^31)");
  if (p->channels < 1 || p->channels > RENO_HEAD_MAX_CHANNELS)
    return fail_thread(RENO_E_INVALID, "channels must be in [1, RENO_HEAD_MAX_CHANNELS]");
  if (p->symbols < 1 || p->symbols > RENO_HEAD_MAX_SYMBOLS)
    return fail_thread(RENO_E_INVALID, "symbols must be in [1, RENO_HEAD_MAX_SYMBOLS]");
  if (p->type != RENO_T_FP32 && p->type != RENO_T_BF16 && p->type != RENO_T_FP16)
    return fail_thread(RENO_E_INVALID, "type must be a reno_type");
  if (p->h_stride < p->channels || p->h_stride >= (int64_t(1) << 31))
    return fail_thread(RENO_E_INVALID, "h_stride must be in [channels, 2^31)");
  if (p->w_stride < p->symbols || p->w_stride >= (int64_t(1) << 31))
    return fail_thread(RENO_E_INVALID, "w_stride must be in [symbols, 2^31)");
  if (k < 1 || k > RENO_HEAD_MAX_TOP) return fail_thread(RENO_E_INVALID, "k must be in [1, RENO_HEAD_MAX_TOP]");
  return RENO_OK;
}

reno_status run(reno::HeadCall& c, const reno_head* p, const reno_head_data* d, void* ws, int64_t bytes, void* stream) {
  const reno_status s = check_head(p, c.k);
  if (s != RENO_OK) return s;
  if (!d) return fail_thread(RENO_E_INVALID, "null data");
  c.p = *p;
  c.d = *d;
  c.grad = d->dh || d->dw || d->db;
  if (!d->w) return fail_thread(RENO_E_INVALID, "null weights");
  if (p->rows > 0) {
    if (!d->h || !c.index) return fail_thread(RENO_E_INVALID, "null input");
    if (!d->bits) return fail_thread(RENO_E_INVALID, "null bits");
  }
  const uintptr_t size = p->type == RENO_T_FP32 ? 4 : 2;
  const void* typed[] = {d->h, d->w, d->b, d->dh, d->dw, d->db};
  const void* words[] = {d->row_weight, d->bits, d->lse, c.index, c.logit};
  for (const void* q : typed)
    if ((uintptr_t)q % size) return fail_thread(RENO_E_INVALID, "an operand is not aligned to its type");
  for (const void* q : words)
    if ((uintptr_t)q % 4) return fail_thread(RENO_E_INVALID, "an operand is not aligned to its type");
  if (bytes < reno::head_workspace(*p, c.k, c.grad)) return fail_thread(RENO_E_INVALID, "workspace too small");
  if (!ws || (uintptr_t)ws % 256) return fail_thread(RENO_E_INVALID, "workspace must be 256-byte aligned");
  c.ws = static_cast<char*>(ws);
  const hipError_t e = reno::launch_head(c, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail_thread(RENO_E_HIP, hipGetErrorString(e));
  return RENO_OK;
}

reno_status check_sample(const reno_sample* p) {
  if (!p) return fail_thread(RENO_E_INVALID, "null argument");
  if (p->rows < 0 || p->rows >= (int64_t(1) << 31)) return fail_thread(RENO_E_INVALID, "rows must be in [0, 2^31)");
  if (p->symbols < 1 || p->symbols > RENO_HEAD_MAX_SYMBOLS)
    return fail_thread(RENO_E_INVALID, "symbols must be in [1, RENO_HEAD_MAX_SYMBOLS]");
  if (p->type != RENO_T_FP32 && p->type != RENO_T_BF16 && p->type != RENO_T_FP16)
    return fail_thread(RENO_E_INVALID, "type must be a reno_type");
  if (p->row_stride < p->symbols || p->row_stride >= (int64_t(1) << 31))
    return fail_thread(RENO_E_INVALID, "row_stride must be in [symbols, 2^31)");
  if (!(p->temperature == 0.0 || (p->temperature >= 0x1p-126 && p->temperature <= 0x1p126)))
    return fail_thread(RENO_E_INVALID, "temperature must be 0 or in [2^-126, 2^126]");
  if (!(p->top_p >= 0.0 && p->top_p <= 1.0)) return fail_thread(RENO_E_INVALID, "top_p must be in [0, 1]");
  if (!(p->min_p >= 0.0 && p->min_p <= 1.0)) return fail_thread(RENO_E_INVALID, "min_p must be in [0, 1]");
  if (p->top_k < 0) return fail_thread(RENO_E_INVALID, "top_k must be 0 or more");
  if (p->allowed && p->allowed_stride != 0 && (p->allowed_stride < p->symbols || p->allowed_stride >= (int64_t(1) << 31)))
    return fail_thread(RENO_E_INVALID, "allowed_stride must be 0 or in [symbols, 2^31)");
  return RENO_OK;
}

}  // namespace

extern "C" {

reno_status reno_head_workspace(const reno_head* head, int top_k, int grad, int64_t* bytes_host) {
  const reno_status s = check_head(head, top_k);
  if (s != RENO_OK) return s;
  if (!bytes_host) return fail_thread(RENO_E_INVALID, "null argument");
  *bytes_host = reno::head_workspace(*head, top_k, grad != 0);
  return RENO_OK;
}

reno_status reno_head_code_length(const reno_head* head, const reno_head_data* data, const int32_t* symbol,
                                  void* workspace, int64_t workspace_bytes, void* hip_stream) {
  reno::HeadCall c;
  c.index = symbol;
  return run(c, head, data, workspace, workspace_bytes, hip_stream);
}

reno_status reno_head_distill(const reno_head* head, const reno_head_data* data, const int32_t* top_index,
                              const float* top_logit, int k, float temperature, void* workspace,
                              int64_t workspace_bytes, void* hip_stream) {
  // log2(e) / temperature, which logits are multiplied by, has to be a normal float
  if (!(temperature > 0.0f) || !std::isfinite(temperature) ||
      !std::isnormal((float)(1.4426950408889634 / (double)temperature)))
    return fail_thread(RENO_E_INVALID, "temperature must be positive and finite, and so log2(e) over it");
  if (!top_logit && head && head->rows > 0) return fail_thread(RENO_E_INVALID, "null input");
  reno::HeadCall c;
  c.k = k;
  c.index = top_index;
  // without rows nothing reads it; any value says that this is a distillation
  static const float none = 0.0f;
  c.logit = top_logit ? top_logit : &none;
  c.temperature = temperature;
  return run(c, head, data, workspace, workspace_bytes, hip_stream);
}

reno_status reno_top_logits(const void* logits, int type, int64_t rows, int symbols, int64_t row_stride, int k,
                            int32_t* index, float* value, float* lse, void* hip_stream) {
  if (rows < 0 || rows >= (int64_t(1) << 31)) return fail_thread(RENO_E_INVALID, "rows must be in [0, 2^31)");
  if (symbols < 1 || symbols > RENO_HEAD_MAX_SYMBOLS)
    return fail_thread(RENO_E_INVALID, "symbols must be in [1, RENO_HEAD_MAX_SYMBOLS]");
  if (type != RENO_T_FP32 && type != RENO_T_BF16 && type != RENO_T_FP16)
    return fail_thread(RENO_E_INVALID, "type must be a reno_type");
  if (row_stride < symbols || row_stride >= (int64_t(1) << 31))
    return fail_thread(RENO_E_INVALID, "row_stride must be in [symbols, 2^31)");
  if (k < 1 || k > RENO_HEAD_MAX_TOP) return fail_thread(RENO_E_INVALID, "k must be in [1, RENO_HEAD_MAX_TOP]");
  if (rows == 0) return RENO_OK;
  if (!logits || !index || !value) return fail_thread(RENO_E_INVALID, "null argument");
  if ((uintptr_t)logits % (type == RENO_T_FP32 ? 4 : 2) || (uintptr_t)index % 4 || (uintptr_t)value % 4 ||
      (uintptr_t)lse % 4)
    return fail_thread(RENO_E_INVALID, "an operand is not aligned to its type");
  const hipError_t e = reno::launch_top(logits, type, rows, symbols, row_stride, k, index, value, lse,
                                        static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return fail_thread(RENO_E_HIP, hipGetErrorString(e));
  return RENO_OK;
}

reno_status reno_sample_symbols(const reno_sample* how, const void* logits, const float* u, int32_t* symbol, float* bits,
                                void* hip_stream) {
  const reno_status s = check_sample(how);
  if (s != RENO_OK) return s;
  if (how->rows == 0) return RENO_OK;
  if (!logits || !u || !symbol || !bits) return fail_thread(RENO_E_INVALID, "null argument");
  const void* words[] = {u, symbol, bits, how->temperature_rows, how->top_p_rows, how->min_p_rows, how->top_k_rows};
  for (const void* q : words)
    if ((uintptr_t)q % 4) return fail_thread(RENO_E_INVALID, "an operand is not aligned to its type");
  if ((uintptr_t)logits % (how->type == RENO_T_FP32 ? 4 : 2))
    return fail_thread(RENO_E_INVALID, "an operand is not aligned to its type");
  const hipError_t e = reno::launch_sample(*how, logits, u, symbol, bits, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return fail_thread(RENO_E_HIP, hipGetErrorString(e));
  return RENO_OK;
}

}  // extern "C"
