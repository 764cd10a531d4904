/*
 * flowpool_train.h -- C ABI of libflowpool's training operators: what a
 * training program does with a packed microbatch at the far end of its
 * backbone, on one MI355X (gfx950).
 *
 *   norm_forward, norm_backward              layer norm of the rows
 *   vocab_loss_forward, vocab_loss_backward  softmax cross entropy of the
 *                                            labelled rows over a vocabulary
 *   adamw_step, adamw_table_*, adamw_state_values
 *                                            one AdamW step over many tensors
 *
 * They are the library's own, not steps of the paper's method. They need no
 * pool, and keep the conventions of flowpool.h: fp_status and
 * fp_last_error(), host and device pointers, `stream` a hipStream_t cast to
 * void* (NULL = the null stream). Besides:
 *  - Every call checks its arguments on the host, then enqueues kernels on
 *    `stream` and returns without waiting. A refused call enqueues nothing.
 *  - Nothing is allocated. A call that needs scratch memory takes it from the
 *    caller: device memory, 256-byte aligned, of the bytes that the matching
 *    *_workspace function says. Its content need not be kept between calls,
 *    and calls that may run at once must not share it. So every call may be
 *    captured into a HIP graph; host arguments (sizes, rates, the step) are
 *    then those of the capture.
 *  - All run on the calling thread's current device. Device memory of the
 *    arguments must stay valid until the enqueued work has completed.
 *  - Results are deterministic: no sum depends on the order in which
 *    workgroups run.
 *  - Rows are addressed by a stride in elements, which may exceed the row.
 *    Offsets are 64-bit.
 *  - Sums, statistics and 32-bit states are f32; 16-bit results are rounded
 *    once, to nearest even.
 */
#ifndef FLOWPOOL_TRAIN_H
#define FLOWPOOL_TRAIN_H

#include "flowpool.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
enum { FP_F32 = 0, FP_BF16 = 1, FP_F16 = 2 };

/* ---------------------------------------------------------------- layer norm
 *
 * For each of `rows` rows of `hidden` elements:
 *   mean = sum(x) / hidden,  rstd = 1 / sqrt(sum((x - mean)^2) / hidden + eps),
 *   y = (x - mean) * rstd * weight + bias.
 *  x, y        device, `type` (FP_F32, FP_BF16, FP_F16), strides of at least
 *              `hidden`; y may be x itself with the same stride.
 *  weight      device, weight_type (FP_F32 or `type`) [hidden], NULL = ones.
 *  bias        the same, NULL = zeros.
 *  mean, rstd  device f32 [rows], written; both are needed by norm_backward.
 * hidden is 1 to 12288. Pointers are aligned to their elements; rows whose
 * addresses and size are multiples of 16 bytes (of all operands) are read and
 * written 16 bytes at a time, others element by element.
 * Errors: EINVAL (null x, y, mean or rstd with rows > 0, rows outside
 * [0, 2^31), hidden, stride, eps not above 0, types), EALIGN, EHIP. */
fp_status norm_forward(const void* x, int64_t x_stride, const void* weight, const void* bias, void* y, int64_t y_stride,
                       float* mean, float* rstd, int64_t rows, int32_t hidden, float eps, int32_t type,
                       int32_t weight_type, void* stream);

/* Bytes of workspace that norm_backward needs for these sizes; FP_EINVAL
 * (negative) for sizes it would refuse. */
int64_t norm_workspace(int64_t rows, int32_t hidden);

/* Gradients of norm_forward. With xhat = (x - mean) * rstd and a = dy * weight:
 *   dx = rstd * (a - sum(a) / hidden - xhat * sum(a * xhat) / hidden),
 *   dweight = sum over rows of dy * xhat,  dbias = sum over rows of dy.
 *  dy, x, dx       device, `type`; dx may be dy or x itself with its stride.
 *  dweight, dbias  device f32 [hidden], either may be NULL (not computed).
 *  accumulate      nonzero: the sums are added to what dweight and dbias
 *                  hold (zero rows leave them); else they replace it.
 * Errors: as norm_forward, and ECAPACITY (workspace too small). */
fp_status norm_backward(const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, const void* weight,
                        const float* mean, const float* rstd, void* dx, int64_t dx_stride, float* dweight, float* dbias,
                        int64_t rows, int32_t hidden, int32_t type, int32_t weight_type, int32_t accumulate,
                        void* workspace, int64_t workspace_bytes, void* stream);

/* ----------------------------------------------------------- vocabulary loss
 *
 * Softmax cross entropy of rows against a vocabulary of `vocab` classes, whose
 * logits are z[t][v] = x[t] . weight[v]. A row is labelled if its label lies
 * in [0, vocab); any other label means that the row has none. Rows without
 * one (image rows) take part in nothing: they are dropped before the products,
 * so they cost nothing there, and what they hold (NaN too) reaches no result.
 * With n labelled rows:
 *   lse[t] = log(sum over v of exp(z[t][v])), 0 for a row without a label,
 *   loss = (sum over labelled t of lse[t] - z[t][label[t]]) / n
 *          (FP_LOSS_MEAN; without the division FP_LOSS_SUM); 0 if n is 0.
 * The logits are formed in pieces, from f32 sums of the exact products of
 * 16-bit values, and are never kept.
 * The loss is computed as log(1 + the other classes' exp(z - z[label])), so it
 * keeps its relative accuracy where the label is nearly certain.
 *  x         device, `type` (FP_BF16 or FP_F16) [rows, hidden], row stride
 *            x_stride.
 *  weight    device, `type` [vocab, hidden], row stride weight_stride.
 *  labels    device int32 [rows].
 *  loss      device f32 [1].
 *  lse       device f32 [rows].
 *  n_labelled  device int32 [1], or NULL: n.
 * hidden is a multiple of 8 up to 12288, weight_stride at most 2^22; x, weight and the strides are
 * multiples of 16 bytes, as a pool's rows are. rows is at most 2^22, vocab at
 * most 2^22.
 * Errors: EINVAL, EALIGN, ECAPACITY (workspace too small), EHIP. */
enum { FP_LOSS_MEAN = 0, FP_LOSS_SUM = 1 };

/* Bytes of workspace of vocab_loss_forward (backward = 0) or of either call
 * (backward != 0); FP_EINVAL (negative) for sizes that they would refuse. */
int64_t vocab_loss_workspace(int64_t rows, int32_t hidden, int32_t vocab, int32_t backward);

fp_status vocab_loss_forward(const void* x, int64_t x_stride, const void* weight, int64_t weight_stride,
                             const int32_t* labels, int64_t rows, int32_t hidden, int32_t vocab, int32_t type,
                             int32_t reduction, float* loss, float* lse, int32_t* n_labelled, void* workspace,
                             int64_t workspace_bytes, void* stream);

/* Gradients of vocab_loss_forward. With
 *   g[t][v] = (exp(z[t][v] - lse[t]) - (v == label[t])) * dloss (/ n for
 *   FP_LOSS_MEAN) for labelled rows:
 *   dx = g weight (rows without a label: zero),  dweight = transposed g x.
 * The logits are formed again, piece by piece. exp(z - lse) of the classes
 * that are not the row's label is rounded to `type` for the two products, as x
 * and weight are; their sums are f32, and the factor dloss / n is applied to
 * them. g at the label is minus the f32 sum of the row's other exp(z - lse),
 * so that it keeps its relative accuracy where the label is nearly certain; its
 * parts of dx and dweight are added in f32.
 *  lse           what vocab_loss_forward wrote for the same x, weight, labels.
 *  dloss         device f32 [1], the gradient of the loss; NULL = 1. If it is
 *                not finite it reaches the labelled rows' results alone.
 *  dx            device, `type` [rows, hidden], row stride dx_stride, or NULL.
 *  dweight       device, dweight_type (`type`, or FP_F32) [vocab, hidden], row
 *                stride dweight_stride, or NULL (a frozen weight).
 *  accumulate    nonzero (dweight_type FP_F32 alone): added to what dweight
 *                holds, for gradients summed over microbatches.
 * dx and dweight are 16-byte aligned, their row strides multiples of 16 bytes.
 * Errors: as vocab_loss_forward. */
fp_status vocab_loss_backward(const void* x, int64_t x_stride, const void* weight, int64_t weight_stride,
                              const int32_t* labels, const float* lse, const float* dloss, int64_t rows, int32_t hidden,
                              int32_t vocab, int32_t type, int32_t reduction, void* dx, int64_t dx_stride,
                              void* dweight, int64_t dweight_stride, int32_t dweight_type, int32_t accumulate,
                              void* workspace, int64_t workspace_bytes, void* stream);

/* --------------------------------------------------------------------- AdamW
 *
 * One step over n_tensors tensors. For each element, with g = grad (times
 * *grad_scale), bc1 = 1 - beta1^step, bc2 = 1 - beta2^step:
 *   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2,
 *   param = param (1 - lr weight_decay)
 *           - (lr / bc1) m / (sqrt(v) / sqrt(bc2) + eps).
 * State of 32 bits: m and v are f32 [n]. State of 8 bits: m and v are uint8
 * [n]; each run of FP_ADAMW_BLOCK elements of a tensor (its last one may be
 * shorter) has a scale for m, the largest |m| of the run, and one for v, the
 * largest v:
 *   m's byte: bit 7 the sign, low 7 bits c:  |m| = scale (c / 127)^2,
 *   v's byte c:                               v  = scale (c / 255)^4.
 * c is the level whose neighbouring thresholds, ((c -+ 1/2) / 127)^2 and
 * ((c -+ 1/2) / 255)^4, the value lies between; a v above 0 never has level 0,
 * so that an element that has seen a gradient keeps a step of bounded size.
 * Both laws spend their levels evenly over the square root of |m| and the
 * fourth root of v: the step is 1.6 % of a run's largest value and grows as
 * 1 / root towards 0, reaching down 16 and 32 powers of two. All zero bytes
 * and scales are the state before the first step. The step itself is computed
 * in f32 before the new state is rounded.
 * Gradients have to be finite: a NaN or infinity reaches its element's
 * parameter (as NaN) and state, and with 8 bits the run's scale, which is then
 * the NaN or infinity and makes all of the run's parameters NaN a step later. */
#define FP_ADAMW_BLOCK 256

typedef struct fp_adamw_tensor {
  void* param;         /* device, param_type [n] */
  const void* grad;    /* device, grad_type [n] */
  void* m;             /* device, f32 [n] or uint8 [n] */
  void* v;
  float* m_scale;      /* device f32 [ceil(n / FP_ADAMW_BLOCK)] (8 bits), else NULL */
  float* v_scale;
  void* copy;          /* device, copy_type [n]: the new param rounded; NULL without one */
  int64_t n;           /* elements, 0 allowed */
  float weight_decay;
  int32_t reserved;    /* 0 */
} fp_adamw_tensor;

typedef struct fp_adamw_config {
  double lr, beta1, beta2, eps;
  int64_t step;          /* 1 for the first */
  int32_t param_type;    /* FP_F32 or FP_BF16 */
  int32_t grad_type;     /* FP_F32, FP_BF16 or FP_F16 */
  int32_t state_bits;    /* 32 or 8 */
  int32_t copy_type;     /* FP_BF16 or FP_F16: every tensor has a copy (param_type
                            FP_F32 alone); -1: none has */
} fp_adamw_config;

/*  tensors     host, read before the call returns. No two may overlap.
 *  grad_scale  device f32 [1] or NULL (= 1), for clipping or unscaling. If it
 *              is not finite the step changes nothing.
 * Pointers are aligned to their elements; a tensor whose pointers are all
 * aligned to 4 elements moves as vectors.
 * Errors: EINVAL (n_tensors < 0, step < 1, lr or eps below 0 or not finite,
 * beta outside [0, 1), types, null pointers, n < 0, reserved), EALIGN, EHIP. */
fp_status adamw_step(const fp_adamw_tensor* tensors, int32_t n_tensors, const fp_adamw_config* config,
                     const float* grad_scale, void* stream);

/* The same step over tensors that stay where they are: they are listed once, in
 * a table in the caller's device memory, and a step is one launch however many
 * they are. adamw_table_write checks the tensors as adamw_step does (the config
 * gives the types; its rates are not used) and enqueues the table's content on
 * `stream`; adamw_table_step has to run behind it, with a config of the same
 * types (of others, or with other groups than that of the table, it changes
 * nothing). The table holds the tensors' addresses: it is written again when
 * one moves, and kept unchanged and allocated while steps run.
 *  table       device, 256-byte aligned, adamw_table_bytes(n_tensors) bytes
 *              (negative FP_EINVAL for n_tensors < 0).
 *  out_groups  host int64: what adamw_table_step takes as groups.
 * Errors: as adamw_step, and ECAPACITY (table too small). */
int64_t adamw_table_bytes(int32_t n_tensors);

fp_status adamw_table_write(const fp_adamw_tensor* tensors, int32_t n_tensors, const fp_adamw_config* config, void* table,
                            int64_t table_bytes, int64_t* out_groups, void* stream);

fp_status adamw_table_step(const void* table, int64_t groups, const fp_adamw_config* config, const float* grad_scale,
                           void* stream);

/* The values that 8-bit states stand for (to save or inspect them): out[i]
 * from codes[i] and scales[i / FP_ADAMW_BLOCK], n elements; moment 1 for m, 2
 * for v. codes, scales and out are device memory. Errors: EINVAL, EALIGN,
 * EHIP. */
fp_status adamw_state_values(const void* codes, const float* scales, float* out, int64_t n, int32_t moment, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* FLOWPOOL_TRAIN_H */
