/*
 * reno_step.h - the step that follows a gradient: the global norm of a model's
 * gradients, clipping by it, and the AdamW update of the weights.
 *
 * They take the gradients of the head's training operators (reno_head.h) or any
 * others: a list of arrays, one for each weight tensor, of a type each.
 *
 * Conventions: those of reno_head.h (no context, nothing allocated on the
 * device, kernels enqueued on hip_stream, status codes, nothing thrown or
 * aborted, calls may be captured into a graph), and
 *  - Lists are host arrays and read before the call returns; what their entries
 *    point to is on the device.  A captured graph keeps the pointers, and the
 *    scalars that are given by value.
 *  - Arrays are dense and may start anywhere that their type allows.  An entry of
 *    n = 0 may have null pointers.
 *  - What a call writes overlaps nothing else that it reads or writes (refused
 *    with RENO_E_INVALID), but an `out` that is its own `grad`.
 *  - Sums of squares are carried in 64 bits and joined in a fixed order; states
 *    and updates are fp32, each result is rounded once to its type.
 *  - The same call gives the same bits every time.
 */
#ifndef RENO_STEP_H
#define RENO_STEP_H

#include "reno_head.h"

#ifdef __cplusplus
extern "C" {
#endif

#define RENO_STEP_MAX_TENSORS (1 << 20)

/* One tensor's gradient. */
typedef struct {
  int64_t n;        /* elements, 0 <= n < 2^40 */
  int64_t type;     /* reno_type of grad and out */
  const void* grad; /* [n] */
  void* out;        /* [n] clipped gradient (reno_grad_clip; not read by reno_grad_norm) */
} reno_gradient;

/* One tensor of weights with its state. */
typedef struct {
  int64_t n;          /* elements, 0 <= n < 2^40 */
  int64_t type;       /* reno_type of param */
  int64_t grad_type;  /* reno_type of grad: that of param, or RENO_T_FP32 */
  void* param;        /* [n] weights, updated */
  const void* grad;   /* [n] */
  float* master;      /* [n] fp32 copy of weights of 16 bits, updated: then param is only written,
                         as its rounding.  NULL: none (fp32 weights have none); weights of 16 bits
                         then lose what is below their own rounding */
  float* exp_avg;     /* [n] first moment, updated */
  float* exp_avg_sq;  /* [n] second moment, updated */
} reno_parameter;

/* How a step is made. */
typedef struct {
  double lr, beta1, beta2, eps, weight_decay;
  double scale;           /* gradients are multiplied by it: one over a loss scale */
  double max_norm;        /* with norm: gradients are scaled down to it; +inf: never */
  const float* lr_factor; /* device, multiplies lr; NULL: 1 (a schedule for captured graphs) */
  const float* norm;      /* device, as reno_grad_norm left it (with the same scale); NULL: no
                             clipping, and the step is always made */
  int32_t* steps;         /* device [2], zero before the first call: steps made, and a word that the
                             calls share and leave zero */
} reno_adamw;

/* Bytes of workspace (into *bytes_host) of reno_grad_norm for the list. */
reno_status reno_grad_workspace(const reno_gradient* grads_host, int64_t count, int64_t* bytes_host);

/* NORM: *norm = scale sqrt(sum over all tensors of g^2), to fp32 (inf past its
 * range); 0 for an empty list, NaN or inf with a gradient that is.  scale:
 * positive and finite. */
reno_status reno_grad_norm(const reno_gradient* grads_host, int64_t count, double scale, float* norm, void* workspace,
                           int64_t workspace_bytes, void* hip_stream);

/* CLIPPING: out = g scale c, c = min(1, max_norm / norm) (c = max_norm / norm too
 * where the norm is NaN).  norm: device, as reno_grad_norm left it.  max_norm:
 * positive, +inf allowed. */
reno_status reno_grad_clip(const reno_gradient* grads_host, int64_t count, const float* norm, double scale,
                           double max_norm, void* hip_stream);

/* ADAMW, the t-th step (t = steps[0] + 1, left there), c as above:
 *   g' = g scale c
 *   exp_avg = beta1 exp_avg + (1 - beta1) g',  exp_avg_sq = beta2 exp_avg_sq + (1 - beta2) g'^2
 *   w -= lr (exp_avg / (1 - beta1^t) / (sqrt(exp_avg_sq / (1 - beta2^t)) + eps) + weight_decay w)
 * With a norm that is inf or NaN nothing is changed, steps neither.  lr and
 * weight_decay: 0 or more and finite; betas: in [0, 1); eps: a positive normal
 * float.  Where (1 - beta2) g'^2 exceeds fp32, exp_avg_sq becomes infinite and
 * stays so, and its weight moves by the decay alone, until it is set anew; a g'
 * that is infinite or NaN itself makes its weight NaN.  Calls that share `steps`
 * must not overlap, and each counts as a step: parameter groups have one each. */
reno_status reno_adamw_step(const reno_parameter* params_host, int64_t count, const reno_adamw* how, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* RENO_STEP_H */
