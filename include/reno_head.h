/*
 * reno_head.h - training operators of the codec's head: the ideal code length
 * of a linear head with its gradient, distillation of a head from a teacher's
 * top logits with its gradient, and the selection of those top logits.
 *
 * They stand beside reno_code_length and reno_predict_probs (reno.h), whose
 * head they train: z = w^T h + b (Eq. 10), bits = -log2 softmax(z)[symbol]
 * (Eq. 4).  The features may be the framework's own (reno_features) or any
 * others, and the alphabet any size.  Without gradients no logits are kept; with
 * them, those of one piece of rows at a time are, in the workspace: all of a call
 * of up to 2^28 (fp32: 2^27) logits or 256 rows, at most so many of a larger one.
 *
 * Conventions: those of reno.h (device pointers, status codes, nothing thrown
 * or aborted), and
 *  - The calls have no context and allocate nothing.  Scratch is the caller's
 *    workspace of at least the size reno_head_workspace gives, 256-byte
 *    aligned.  A call only enqueues kernels on hip_stream (a stream of the
 *    current device; NULL: the null stream), on whose device every pointer
 *    lies, and may be captured into a graph.  Calls that can overlap, replays
 *    of a captured graph among them, need workspaces and outputs of their own.
 *  - Argument errors return RENO_E_INVALID before anything is enqueued, launch
 *    errors RENO_E_HIP, with the message in reno_last_error(NULL).
 *  - Matrices are row-major; inputs may have rows further apart than their
 *    length, outputs are dense.  Element types are reno_type; sums, softmax
 *    statistics, bits and normalisers are fp32, gradients are rounded once to
 *    the type of what they belong to.
 *  - Outputs overlap neither each other nor inputs.
 *  - Logits are carried in powers of two over the temperature: a bias or logit of
 *    |z / T| log2(e) >= 2^128 counts as infinite.  A symbol whose logit is -inf has
 *    probability 0; a row all of whose logits are -inf has lse -inf and NaN bits.
 *    A row with a logit of +inf has lse +inf, bits of +inf, or NaN where the logit
 *    of a target is +inf itself, and may have NaN in every gradient it reaches.
 *    That is for biases: a weight that is infinite or NaN may make any gradient
 *    NaN, dh of rows that are left out too, and a bias of +inf or NaN dw and db of
 *    calls without any row taken.
 *  - The same call gives the same bits every time.
 */
#ifndef RENO_HEAD_H
#define RENO_HEAD_H

#include "reno.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  RENO_T_FP32 = 0, /* products of operands carried as three bf16 parts, cut off: 24 bits, down to
                      2^-133 (operands below 2^-110, in heads of up to 128 channels and 256
                      symbols g (p - q) too, keep fewer).  Of the nine products of parts six
                      are kept; the others are below 2^-21 of the whole together, 2^-24.6 on
                      average, and of its sign.  (Up to 4 rows without gradients, in wider heads:
                      plain fp32 sums.) */
  RENO_T_BF16 = 1, /* bf16 products, fp32 sums; logits' gradients are rounded to bf16 before
                      they meet h and w (kept until then to 2^-12 of the probability, and
                      as 0 below 2^-39 of the largest of 64 or 128 symbols), so that
                      gradients have two roundings, 1.4 times the error of one; calls of up
                      to 16 rows, where nothing averages, carry them in two parts and have one */
  RENO_T_FP16 = 2  /* the same in fp16, logits' gradients scaled by 2^14 over the largest
                      row weight so that none above 2^-38 of it is lost */
} reno_type;

#define RENO_HEAD_MAX_CHANNELS 16384
#define RENO_HEAD_MAX_SYMBOLS (1 << 20)
#define RENO_HEAD_MAX_TOP 128

/* A linear head over `symbols` classes applied to `rows` feature rows. */
typedef struct {
  int64_t rows;      /* N, 0 <= N < 2^31 */
  int channels;      /* C, 1 .. RENO_HEAD_MAX_CHANNELS */
  int symbols;       /* V, 1 .. RENO_HEAD_MAX_SYMBOLS */
  int type;          /* reno_type of h, w, b, dh, dw and db */
  int64_t h_stride;  /* elements from one row of h to the next, >= C */
  int64_t w_stride;  /* elements from one row of w to the next, >= V */
} reno_head;

/* Operands and results of one call. */
typedef struct {
  const void* h;           /* [N][C] features */
  const void* w;           /* [C][V] weights, the layout of reno_weights.head_w */
  const void* b;           /* [V] bias, or NULL: zero */
  const float* row_weight; /* [N] g: the gradients are those of sum_r g_r bits_r; NULL: 1 */
  float* bits;             /* [N] out */
  float* lse;              /* [N] out, or NULL: log sum_v exp(z_rv / temperature) (natural log) */
  void* dh;                /* [N][C] out, or NULL: not wanted */
  void* dw;                /* [C][V] out, or NULL */
  void* db;                /* [V] out, or NULL */
} reno_head_data;

/* Bytes of workspace (into *bytes_host) for a call on such a head with top_k
 * entries a row (reno_head_code_length: 1), with any gradient (grad != 0) or
 * none: every row's targets (8 top_k + 5 bytes a row), a copy of w as 16-bit
 * parts (reserved also for weights that turn out to be read in place), one piece
 * of rows (copies of h: 2^31 bytes or 256 rows at most) and, with gradients, its
 * logits (fp32 10 bytes each, fp16 6, bf16 2) and fp32 sums of dw.  No device work. */
reno_status reno_head_workspace(const reno_head* head, int top_k, int grad, int64_t* bytes_host);

/* CODE LENGTH of a head with its gradient (Eqs. 4, 10):
 *   bits_r = (lse_r - z_r[s_r]) / ln 2
 *   dz_rv = g_r / ln 2 (softmax(z_r)_v - [v = s_r]),  dh = dz w^T,  dw = h^T dz,  db = sum_r dz_r
 * symbol int32 [N].  A negative symbol leaves its row out: bits, lse and dh of
 * the row are 0, and nothing of the row (NaN and infinities in h or row_weight
 * included) reaches dw or db.  A symbol of V or more gives NaN bits, and NaN in
 * every gradient that the row reaches. */
reno_status reno_head_code_length(const reno_head* head, const reno_head_data* data, const int32_t* symbol,
                                  void* workspace, int64_t workspace_bytes, void* hip_stream);

/* DISTILLATION from a teacher's top logits: the row's k entries top_index
 * int32 [N][k], top_logit float [N][k] (RENO_HEAD_MAX_TOP at most; reno_top_logits
 * makes them) stand for the distribution q_r = softmax_j(top_logit_rj / T),
 * the student's is p_r = softmax(z_r / T) over all symbols:
 *   bits_r = sum_j q_rj log2(q_rj / p_r[top_index_rj])
 *   dz_rv = g_r / (T ln 2) (p_rv - q_r(v)),  q_r(v) = sum of q_rj with top_index_rj = v
 * An entry with a negative index is not there; one whose index occurs before
 * counts with it, as one entry of their summed probability.  A row without any
 * entry (or with logits of -inf only) is left out as above; an index of V or
 * more, or an entry's logit of +inf or NaN, gives NaN as above.  temperature:
 * positive and finite, 2^-127 to 2^126. */
reno_status reno_head_distill(const reno_head* head, const reno_head_data* data, const int32_t* top_index,
                              const float* top_logit, int k, float temperature, void* workspace,
                              int64_t workspace_bytes, void* hip_stream);

/* TOP LOGITS: the k largest of each row of logits [N][V] (type: reno_type,
 * rows row_stride >= V elements apart) in descending order, ties by ascending
 * index, NaN above everything: index int32 [N][k], value float [N][k]; with
 * k > V the entries from V on are -1 and -inf.  lse: NULL or float [N], the row's
 * log sum exp in natural log (+inf with a logit of +inf, NaN with one of NaN).
 * 1 <= k <= RENO_HEAD_MAX_TOP.  Needs no workspace. */
reno_status reno_top_logits(const void* logits, int type, int64_t rows, int symbols, int64_t row_stride, int k,
                            int32_t* index, float* value, float* lse, void* hip_stream);

/* FEATURES of a model scale (b0 < scale < B) that the head is applied to, as
 * the last reno_predict_probs of that scale left them (Sec. 3.2, h of the last
 * layer; two-stage: of the first head, the second's are h + Emb(S1)): fp32
 * [N_scale][C].  RENO_ALL_SCALES: every model scale, concatenated in order.
 * A channel that no weight reads (its rows of the head, of both heads, are all
 * zero; the full predictor's own layers read every channel) is not kept by the
 * model kernels and comes back as NaN.  The features do not depend on the head:
 * to train one from zero, or one with rows that are zero, take them under a
 * head without such rows.  RENO_E_STATE before predict_probs. */
reno_status reno_features(reno_ctx* ctx, int scale, float* features);

#ifdef __cplusplus
}
#endif
#endif /* RENO_HEAD_H */
