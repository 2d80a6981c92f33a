/*
 * huge2_train.h -- C ABI of libhuge2, continued: the operators that stand
 * between a generator's convolutions and around them when it is trained.
 *
 *   group norm with an activation, and its gradients: what follows a
 *     convolution (huge2.h) in a generator or a decoder;
 *   embedding lookup with a scale, and the table's gradient: class labels of a
 *     conditional generator, maps of code indices, text tokens;
 *   an AdamW step over many tensors in one call, with the moments in 32 bits
 *     or in 8: what takes the weight gradients.
 *
 * The conventions of huge2.h hold: device pointers owned by the caller,
 * contiguous in the stated order and 16-byte aligned unless stated; every
 * argument is checked before any HIP call, on an error nothing is enqueued;
 * work is enqueued on hip_stream and the call returns; no C++ exception
 * crosses the ABI; sums are held in fp32 (products of bf16 and fp32 inputs are
 * formed in fp32), each result is rounded once to its type, to nearest even;
 * results are deterministic (a fixed order of summation, no floating-point
 * atomics).  A plan's workspace is shared by the calls on it: enqueue them on
 * one stream, or order them.  The calls that run a plan allocate nothing and
 * can be recorded into a HIP graph, whose replays repeat them as they were recorded:
 * on the same pointers, and an AdamW step with its step number, rates and decays.
 */
#ifndef HUGE2_TRAIN_H
#define HUGE2_TRAIN_H

#include <stdint.h>

#include "huge2.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- group norm with an activation --------------------------------------- */

/* The first three are huge2_activation's; SILU: z / (1 + exp(-z)). */
typedef enum {
  HUGE2_NORM_NONE = 0,
  HUGE2_NORM_RELU = 1,
  HUGE2_NORM_TANH = 2,
  HUGE2_NORM_SILU = 3
} huge2_norm_activation;

/* x is n images of h x w pixels and c channels, in groups of d = c / groups
 * neighbouring channels.  For image i and group k, over its m = d*h*w values,
 *   mean = sum x / m,  var = sum (x - mean)^2 / m,  rstd = 1 / sqrt(var + eps),
 *   xh = (x - mean) * rstd,  z = xh * gamma[channel] + beta[channel],
 *   y = activation(z). */
typedef struct {
  int32_t n, c, h, w; /* >= 1; c*h*w below 2^31 */
  int32_t groups;     /* >= 1, divides c */
  int32_t layout;     /* huge2_layout of x, y, dy, dx */
  int32_t dtype;      /* huge2_dtype of x, y, dy, dx; the rest is float */
  int32_t activation; /* huge2_norm_activation */
  float eps;          /* > 0 and finite */
} huge2_norm_desc;

typedef struct huge2_norm_plan huge2_norm_plan;

/* Chooses the kernels for desc and allocates their workspace: 8 bytes for each
 * group of each image, and for each channel (and group) of each run of pixels that
 * an image is cut into: one run where the slabs of an image fit the registers of
 * compute units, else runs of 4 pixels or more.  No work is enqueued.  Errors:
 * INVALID_ARG, UNSUPPORTED (c*h*w of 2^31 or more, 2^40 elements in all, or more
 * groups and images than the 2^32 threads of a launch can take), ALLOC. */
huge2_status huge2_norm_plan_create(huge2_norm_plan** out, const huge2_norm_desc* desc);

/* Enqueues y from x.  gamma and beta are [c] float; NULL gamma is all ones,
 * NULL beta all zeros.  stats is NULL or [n][groups][2] float and then receives
 * (mean, rstd), which huge2_norm_grad_execute reads.  y and stats must not overlap
 * each other or an input.  Errors: INVALID_ARG, HIP. */
huge2_status huge2_norm_execute(const huge2_norm_plan* plan, const void* x, const float* gamma,
                                const float* beta, void* y, float* stats, void* hip_stream);

/* Enqueues the gradients of a forward call for the output error dy, from the
 * same x, gamma and beta and the stats that the call wrote:
 *   dz = dy * activation'(z),  dbeta = sum over n, pixels of dz,
 *   dgamma = sum over n, pixels of dz * xh,  t = dz * gamma,
 *   dx = rstd * (t - mean over the group of t - xh * mean over the group of t*xh).
 * A ReLU's z is formed with the forward's own roundings, so that it masks the same
 * values both ways (its slope at 0 is 0).  dgamma and dbeta are [c] float and
 * may be NULL.  dx, dgamma and dbeta must not overlap each other or an input.
 * Errors: INVALID_ARG, HIP. */
huge2_status huge2_norm_grad_execute(const huge2_norm_plan* plan, const void* x, const void* dy,
                                     const float* stats, const float* gamma, const float* beta,
                                     void* dx, float* dgamma, float* dbeta, void* hip_stream);

/* Names of the kernels that the plan launches: grad 0 for the forward, 1 for
 * the gradients.  Storage of the plan's; "" for a NULL plan. */
const char* huge2_norm_plan_kernel(const huge2_norm_plan* plan, int32_t grad);

/* Waits for the device and releases the plan.  NULL is accepted.  Errors: HIP. */
huge2_status huge2_norm_plan_destroy(huge2_norm_plan* plan);

/* ---- embedding lookup ----------------------------------------------------- */

/* y[t][:] = scale * table[id[t]][:].  An id outside [0, rows), such as -1 for
 * padding, reads as a row of zeros and adds to no row of the gradient. */
typedef struct {
  int32_t rows, dim; /* of the table, >= 1 */
  int32_t dtype;     /* huge2_dtype of table, y, dy, dtable */
  int32_t id_bits;   /* 32 or 64: ids are int32_t or int64_t (aligned to that) */
  float scale;
} huge2_embedding_desc;

/* Enqueues y for `tokens` ids (>= 0; none: nothing is done and the pointers may
 * be NULL).  y [tokens][dim] must not alias table [rows][dim].  Errors:
 * INVALID_ARG, UNSUPPORTED (2^31 tokens or more, or rows of 2^31 bytes), HIP. */
huge2_status huge2_embedding(const huge2_embedding_desc* desc, const void* ids, int64_t tokens,
                             const void* table, void* y, void* hip_stream);

typedef struct huge2_embedding_grad_plan huge2_embedding_grad_plan;

/* A plan for the gradients of up to max_tokens (>= 0) tokens.  Allocates the
 * buffers of the tokens' order and of partial sums: 16 bytes a token, 16 KB for each
 * 512 tokens up to 131072, and an 8th of dy's values (a 32nd above 131072 tokens) in
 * fp32.  No work is enqueued.  Errors: INVALID_ARG,
 * UNSUPPORTED (2^30 tokens or more, rows of 2^31 bytes, or more rows or tokens than
 * the 2^32 threads of a launch can take: 2^28 rows always fit), ALLOC. */
huge2_status huge2_embedding_grad_plan_create(huge2_embedding_grad_plan** out,
                                              const huge2_embedding_desc* desc,
                                              int64_t max_tokens);

/* Enqueues dtable[v][:] = scale * sum over t with id[t] = v of dy[t][:], every
 * row of it (zeros where no token has it), summed in fp32 in an order that
 * depends on the ids alone.  tokens <= max_tokens.  Errors: INVALID_ARG, HIP. */
huge2_status huge2_embedding_grad_execute(const huge2_embedding_grad_plan* plan, const void* ids,
                                          int64_t tokens, const void* dy, void* dtable,
                                          void* hip_stream);

/* Name of the kernel that adds up so many tokens' gradients.  Storage of the plan's;
 * "" for a NULL plan. */
const char* huge2_embedding_grad_plan_kernel(const huge2_embedding_grad_plan* plan,
                                             int64_t tokens);

/* Waits for the device and releases the plan.  NULL is accepted.  Errors: HIP. */
huge2_status huge2_embedding_grad_plan_destroy(huge2_embedding_grad_plan* plan);

/* ---- AdamW ----------------------------------------------------------------- */

/* A parameter tensor and its state, `count` elements each, all updated in place.
 * The moments m and v are float with 32 state bits.  With 8, m and u = sqrt(v)
 * are numbers of the OCP e4m3 format (one byte; the largest is 448), each block
 * of 256 elements (the last may be shorter) with a scale of its own in m_scale
 * and v_scale ([ceil(count / 256)] float, 4-byte aligned): value = number * scale.
 * The scale is the block's largest magnitude over 448; numbers are rounded to
 * nearest even, and a u that is not zero never to zero (a parameter whose
 * gradient stops must not be left with a moment over nothing).  A block with
 * nothing over 2^-100 has scale 0 and zeros.  States start as zeros.  A
 * gradient that is not finite makes its element's state (with 8 bits, its
 * block's) and its parameter NaN or infinite, as the formulas do. */
typedef struct {
  void* param;
  void* m;
  void* v;
  float* m_scale; /* 8 state bits only, else NULL */
  float* v_scale;
  void* copy; /* NULL, or bfloat16 [count]: receives the updated parameter rounded
                 (the working weights of a float parameter) */
  int64_t count;      /* >= 0 */
  int32_t dtype;      /* huge2_dtype of param */
  int32_t grad_dtype; /* huge2_dtype of its gradient */
  float weight_decay; /* >= 0 and finite */
} huge2_adamw_tensor;

typedef struct huge2_adamw_plan huge2_adamw_plan;

/* A plan for `count` tensors (>= 0), which must outlive it.  No two of their arrays
 * may overlap: a parameter that two layers share is listed once.  Allocates their
 * table and the list of work, copies both on hip_stream and waits for it.
 * Errors: INVALID_ARG, UNSUPPORTED (2^40 elements in all, or more), ALLOC, HIP. */
huge2_status huge2_adamw_plan_create(huge2_adamw_plan** out, const huge2_adamw_tensor* tensors,
                                     int32_t count, int32_t state_bits, void* hip_stream);

typedef struct {
  double lr, beta1, beta2, eps; /* lr >= 0, 0 <= beta < 1, eps >= 2^-126, all finite */
  int64_t step;                 /* of this call, from 1 */
} huge2_adamw_options;

/* Enqueues one step: with g = grad (* *grad_scale, a device float such as a
 * clipping factor, where that is not NULL),
 *   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,
 *   param = param (1 - lr weight_decay) - lr / (1 - beta1^step)
 *           * m / (sqrt(v) / sqrt(1 - beta2^step) + eps),
 * in fp32, from the new m and v before they are rounded to 8 bits.  grads is a
 * host array of `count` device pointers in the plan's order, none into an array that the
 * step writes; a tensor whose gradient is NULL is left as it is.  The options are taken on
 * the host: a recorded step keeps the bias corrections of its `step` and its lr in every
 * replay, so a training loop that replays a graph enqueues its step outside of it.
 * Errors: INVALID_ARG, HIP. */
huge2_status huge2_adamw_step(const huge2_adamw_plan* plan, const void* const* grads,
                              const huge2_adamw_options* options, const float* grad_scale,
                              void* hip_stream);

/* Waits for the device and releases the plan (not the tensors).  NULL is
 * accepted.  Errors: HIP. */
huge2_status huge2_adamw_plan_destroy(huge2_adamw_plan* plan);

#ifdef __cplusplus
}
#endif
#endif /* HUGE2_TRAIN_H */
