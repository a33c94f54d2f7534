/*
 * liec_train.h -- operators around the backward pass whose gradients a compressed step (liec.h) takes, for N simulated
 * workers at once: layer normalisation with weights of each worker's own and the gradients of those weights, the
 * global norm of a worker's gradient tensors, and clipping by it, in place or on the way into the fp32 rows of
 * liec_step.
 *
 * Tensors are DEVICE pointers of one of the types of liec_dtype, at any multiple of the element's size.  The entry
 * points need no context and allocate nothing: they enqueue kernels on `hip_stream` (a hipStream_t passed as void*,
 * NULL = null stream) of the current device and return.  Where scratch is needed the caller passes it (`workspace`,
 * 16-byte aligned DEVICE memory of at least the bytes that the matching ..._workspace call names; its contents need no
 * preparation, it shares no memory with the call's other arguments, and calls that may overlap need one each).  They may
 * be captured into a HIP graph.  Argument arrays are HOST memory, read before the call returns.  No entry point throws;
 * every failure is a status code of liec.h (LIEC_EINVAL: nothing was enqueued).
 *
 * Arithmetic: inputs are widened to fp32 exactly, results are rounded once to the output's type, to nearest; sums of
 * squares of gradients are carried in fp64, the sums of layer normalisation in fp32 over at most 256 rows or one row's
 * columns and in fp64 beyond.  The order of every sum is fixed by the sizes, so equal calls give equal bits.
 */
#ifndef LIEC_TRAIN_H
#define LIEC_TRAIN_H

#include <stdint.h>

#include "liec.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    LIEC_F32 = 0,
    LIEC_BF16 = 1,
    LIEC_F16 = 2
} liec_dtype;

/* The gradients of one parameter tensor: for worker i, `count` consecutive values from data + i * stride (in values).
 * count = 0 is allowed (data may then be NULL). */
typedef struct {
    void *data;
    int64_t count, stride;
    int32_t dtype; /* liec_dtype */
    int32_t reserved; /* 0 */
} liec_grad_tensor;

#define LIEC_GRAD_MAX_TENSORS 65536

/* Bytes of scratch that the calls below need for T tensors of N workers; -1 for bad arguments.  Host only. */
int64_t liec_grads_workspace(int32_t N, int32_t T);

/*
 * liec_grad_norm: norms[i] = sqrt(sum over the T tensors of the squares of worker i's values), i < N (DEVICE, fp32,
 * N values).  Infinities and NaN show in the norm of their worker, and only there.  T = 0 or no values: zero.
 *   1 <= N <= 65535, 0 <= T <= LIEC_GRAD_MAX_TENSORS, at most 2^35 values per worker.  stride may be anything, 0
 *   included (workers that share a tensor).  Two kernels; one more for every 184 further tensors (128 where a tensor's
 *   stride is not its count).
 */
liec_status liec_grad_norm(const liec_grad_tensor *tensors, int32_t T, int32_t N, float *norms, void *workspace,
                           int64_t workspace_bytes, void *hip_stream);

/*
 * liec_clip_grads: every value of worker i times c_i, in place, with c_i = 1 where norm_i <= max_norm and
 * max_norm / norm_i elsewhere (the quotient in fp64 from the fp64 norm, rounded to fp32; the product in fp32).
 * A worker whose norm is NaN gets NaN everywhere, one whose norm is infinite gets zeros and NaN; max_norm = +Inf
 * clips nothing.
 *   max_norm  >= 0, not NaN
 *   norms     NULL, or N fp32 values (DEVICE) outside the tensors: the norms before clipping
 * No two tensors, nor two workers' values of one, may share memory (LIEC_EINVAL, for instance for a tied tensor that
 * is listed twice).  They may lie between one another where their strides are equal or opposite in bytes, such as
 * columns of a matrix; tensors that do so at strides that differ count as sharing.
 */
liec_status liec_clip_grads(const liec_grad_tensor *tensors, int32_t T, int32_t N, float max_norm, float *norms,
                            void *workspace, int64_t workspace_bytes, void *hip_stream);

/*
 * liec_gather_grads: the tensors, clipped as by liec_clip_grads, one after the other into the fp32 rows that
 * liec_step reads: worker i's values of tensor t go to rows + i * row_stride + (counts of the tensors before t).
 * The tensors are read only (any stride); a tensor that shares memory with the rows or the norms is LIEC_EINVAL, and
 * so are norms in the rows.  At strides that
 * differ from the rows', more than 2^22 workers' values that lie between the rows count as sharing.
 *   row_stride  >= the sum of the counts
 *   max_norm = +Inf with norms = NULL only gathers: one kernel for up to 184 tensors (128 where a tensor's stride is not
 *   its count), each value read once.
 */
liec_status liec_gather_grads(const liec_grad_tensor *tensors, int32_t T, int32_t N, float *rows, int64_t row_stride,
                              float max_norm, float *norms, void *workspace, int64_t workspace_bytes, void *hip_stream);

/* Activations [N, R, C]: value (i, r, c) at data + i * worker_stride + r * row_stride + c. */
typedef struct {
    void *data;
    int64_t worker_stride, row_stride;
} liec_rows;

/* A weight or a bias, or its gradient: value c of worker i at data + i * stride + c.  stride = 0: one vector for all
 * workers.  data = NULL: none (weight 1, bias 0, gradient not asked for). */
typedef struct {
    void *data;
    int64_t stride;
} liec_param;

/*
 * liec_layer_norm: for every row, mu = mean(x), rstd = 1 / sqrt(mean((x - mu)^2) + eps) and
 * y = (x - mu) * rstd * weight + bias.
 *   mean, rstd   DEVICE fp32 [N, R] contiguous, for the backward pass; either may be NULL; memory of their own
 *   dtype        type of x and y;  param_dtype  type of weight and bias
 *   1 <= N <= 65535, 0 <= R < 2^31 (no rows: nothing to do), 1 <= C <= 2^28, at most 2^40 values, eps >= 0 and
 *                finite; no value lies further than 2^40 values from the first
 * y may be x itself (same pointer and strides); otherwise they must not overlap, and neither may y's rows one
 * another (LIEC_EINVAL; at strides that differ, more than 2^22 rows of both that lie between one another count as
 * overlapping).  y may not share memory with weight or bias.  Rows of 8 to 16384 columns are read once.
 */
liec_status liec_layer_norm(const liec_rows *x, const liec_param *weight, const liec_param *bias, const liec_rows *y,
                            float *mean, float *rstd, int32_t N, int64_t R, int64_t C, float eps, liec_dtype dtype,
                            liec_dtype param_dtype, void *hip_stream);

/* Bytes of scratch that liec_layer_norm_backward needs when weight or bias gradients are asked for; -1 for bad
 * arguments.  Host only. */
int64_t liec_layer_norm_workspace(int32_t N, int64_t R, int64_t C);

/*
 * liec_layer_norm_backward: with h = (x - mean) * rstd and a = dy * weight,
 *   dx = rstd * (a - mean(a) - h * mean(a h)),  dweight_i = sum over worker i's rows of dy * h,  dbias_i of dy.
 * dweight and dbias with stride 0 take the sum over all workers' rows.  They are written, not added to, also where
 * there are no rows (zeros).  They share no memory with each other or with other operands; either may take the place
 * of weight itself (same pointer and stride).
 *   dx           NULL, or data = NULL, where it is not asked for; dx may be dy or x itself (same pointer and strides),
 *                as for liec_layer_norm; its rows must not overlap, nor share memory with mean, rstd or weight
 *   mean, rstd   as liec_layer_norm left them
 *   param_dtype  type of weight, dweight and dbias
 */
liec_status liec_layer_norm_backward(const liec_rows *dy, const liec_rows *x, const float *mean, const float *rstd,
                                     const liec_param *weight, const liec_rows *dx, const liec_param *dweight,
                                     const liec_param *dbias, int32_t N, int64_t R, int64_t C, liec_dtype dtype,
                                     liec_dtype param_dtype, void *workspace, int64_t workspace_bytes,
                                     void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* LIEC_TRAIN_H */
