/*
 * liec_activations.h -- operators on the activations of N simulated workers at once, next to those of liec_train.h: activation
 * checkpoints in 8 bits, group normalisation with an activation function, channels last, with weights of each worker's own
 * and its gradients, and the gradient of a linear layer's weight from a checkpoint of the layer's input.
 *
 * The manner is that of liec_train.h: DEVICE pointers at any multiple of the element's size, no context, no allocation, kernels
 * enqueued on `hip_stream` of the current device, scratch from the caller (16-byte aligned, of at least the bytes that the
 * matching ..._workspace call names, not prepared, shared with nothing), status codes of liec.h (LIEC_EINVAL: nothing was
 * enqueued), no exceptions, capture into HIP graphs allowed.
 *
 * Arithmetic: inputs are widened to fp32 exactly, results are rounded once to the output's type, to nearest; sums are fp32 over at
 * most 256 rows of a thread and what its block adds to them, and fp64 beyond; products of matrices are exact and added up in
 * fp32 over at most 8192 rows, and in fp64 beyond.  The order of every sum is fixed by the sizes, so equal calls give equal bits.
 *
 * Operands that lie between one another are told apart exactly; at strides that differ, more than 2^22 runs of both that do so count as
 * sharing memory.
 */
#ifndef LIEC_ACTIVATIONS_H
#define LIEC_ACTIVATIONS_H

#include <stdint.h>

#include "liec_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * A checkpoint of activations [N, R, C] in 8 bits.  Every 32 consecutive columns of a row (fewer at its end) share an exponent
 * byte s: column c stands for values[c] * 2^(s - 127), for 0 where s = 0.  Both arrays are contiguous, in any memory of their
 * own: values [N, R, C], exponents [N, R, ceil(C / 32)].  s is the smallest from 1 on with which no value exceeds 127, and each
 * value is rounded to nearest, ties to even: it is off by at most 2^(s - 128), 1/127 of the largest of its 32.  s ends at 248, and what
 * exceeds 127 there (numbers next to the largest of fp32 and bf16) counts as 127.  s = 255 stands for NaN throughout: columns
 * that held an infinity or a NaN.  What a checkpoint stands for is exact in fp32 and in bf16.
 */
#define LIEC_CHECKPOINT_COLUMNS 32

typedef struct {
    int8_t *values;
    uint8_t *exponents;
} liec_checkpoint;

/*
 * liec_checkpoint_save: the checkpoint of x.
 *   1 <= N <= 65535, 0 <= R < 2^31 (no rows: nothing to do), 1 <= C <= 2^28, at most 2^40 values; x as in
 *   liec_layer_norm.  x, the values and the exponents share no memory.
 */
liec_status liec_checkpoint_save(const liec_rows *x, const liec_checkpoint *saved, int32_t N, int64_t R, int64_t C, liec_dtype dtype,
                                 void *hip_stream);

/* liec_checkpoint_load: what a checkpoint stands for, rounded to y's type (fp16: beyond its range an infinity).  y's rows do not
 * overlap, nor share memory with the checkpoint. */
liec_status liec_checkpoint_load(const liec_checkpoint *saved, const liec_rows *y, int32_t N, int64_t R, int64_t C, liec_dtype dtype,
                                 void *hip_stream);

typedef enum {
    LIEC_ACT_NONE = 0,
    LIEC_ACT_RELU = 1, /* max(z, 0); derivative 0 at 0 */
    LIEC_ACT_SILU = 2  /* z / (1 + exp(-z)) */
} liec_activation;

/* Images [N, B, S, C], channels last: value (i, b, s, c) at data + i * worker_stride + b * image_stride + s * row_stride + c. */
typedef struct {
    void *data;
    int64_t worker_stride, image_stride, row_stride;
} liec_images;

/* Bytes of scratch that liec_group_norm and liec_group_norm_backward need, 16 per channel and at most 256 MB more (or what one image's
 * sums take, if that is more: many images go in parts); -1 for bad arguments.  Host only. */
int64_t liec_group_norm_workspace(int32_t N, int64_t B, int64_t S, int64_t C, int64_t G);

/*
 * liec_group_norm: the C channels of an image fall into G groups of C / G neighbours; for every image and group, over its S positions
 * and its channels, mu = mean(x), rstd = 1 / sqrt(mean((x - mu)^2) + eps), and y = act((x - mu) * rstd * weight + bias).
 *   weight, bias [N, C] as in liec_layer_norm (stride 0: one vector for all workers; none: 1 and 0)
 *   mean, rstd   DEVICE fp32 [N, B, G] contiguous, for the backward pass; memory of their own; left as they are where S = 0
 *   saved        NULL, or a checkpoint of x as rows [N, B * S, C], written in the same pass; memory of its own
 *   1 <= N <= 65535, 0 <= B < 2^31, 0 <= S < 2^31 (nothing in an image: nothing to do), 1 <= C <= 2^20, G a divisor of C, at most
 *   2^40 values, eps >= 0 and finite; no value lies further than 2^40 values from the first
 * y may be x itself (same pointer and strides); otherwise they share no memory, and neither do y's rows with one another, or with
 * weight or bias.  A group that holds an infinity or a NaN gets NaN, and so may one whose values add up beyond the largest fp32 number;
 * where only the squares of their distances from the mean do (distances of 1e19, say), rstd is 0 and y = act(bias).
 */
liec_status liec_group_norm(const liec_images *x, const liec_param *weight, const liec_param *bias, const liec_images *y, float *mean, float *rstd,
                            const liec_checkpoint *saved, int32_t N, int64_t B, int64_t S, int64_t C, int64_t G, float eps,
                            liec_activation activation, liec_dtype dtype, liec_dtype param_dtype, void *workspace,
                            int64_t workspace_bytes, void *hip_stream);

/*
 * liec_group_norm_backward: with h = (x - mean) * rstd, z = h * weight + bias, dz = dy * act'(z) and a = dz * weight,
 *   dx = rstd * (a - mean(a) - h * mean(a h)),  dweight_i = sum over worker i's images and positions of dz * h,  dbias_i of dz.
 *   x, saved     one of the two: the forward pass's input, or a checkpoint of it (the other NULL, or its data / values NULL)
 *   dx           NULL, or data = NULL, where it is not asked for; it may be dy or x itself (same pointer and strides); otherwise it
 *                shares no memory with other operands, nor its rows with one another
 *   bias         is needed where the activation is (its derivative depends on z)
 *   dweight, dbias  as in liec_layer_norm_backward: written, zeros where there is nothing to add up; stride 0 takes the sum over all
 *                workers; memory of their own, that of weight and bias not among it
 *   mean, rstd   as liec_group_norm left them
 * Where z is so near to zero that fp32 does not tell its sign, ReLU's derivative is decided in fp64.  SiLU's z and slope are 0 where
 * exp(-z) is beyond fp32; results under 2^-119 may come as 0 before that.
 */
liec_status liec_group_norm_backward(const liec_images *dy, const liec_images *x, const liec_checkpoint *saved, const float *mean,
                                     const float *rstd, const liec_param *weight, const liec_param *bias, const liec_images *dx,
                                     const liec_param *dweight, const liec_param *dbias, int32_t N, int64_t B, int64_t S, int64_t C,
                                     int64_t G, liec_activation activation, liec_dtype dtype, liec_dtype param_dtype,
                                     void *workspace, int64_t workspace_bytes, void *hip_stream);

/* A matrix for each worker: value (o, c) of worker i at data + i * worker_stride + o * row_stride + c. */
typedef struct {
    void *data;
    int64_t worker_stride, row_stride;
} liec_matrices;

/* Bytes of scratch that liec_weight_grad needs; -1 for bad arguments.  Host only.  None where the rows are not split; otherwise the fp32 sums
 * of each split, 4 N O (C + 1) bytes: of up to 8192 rows, or of fewer where there are few weights, then for at most 512 blocks in all. */
int64_t liec_weight_grad_workspace(int32_t N, int64_t R, int64_t O, int64_t C);

/*
 * liec_weight_grad: gradients of the weight and the bias of y = x weight^T + bias for R rows of x of each worker, x given by its
 * checkpoint:  dweight_i[o, c] = sum over rows r of dy_i[r, o] * x_i[r, c],  dbias_i[o] = sum over rows of dy_i[r, o].
 *   dy           [N, R, O] of dtype, rows as in liec_layer_norm
 *   saved        checkpoint of x [N, R, C]
 *   dweight      [N, O, C] of param_dtype (columns of the rows of a step, say); its values share no memory
 *   dbias        [N, O] of param_dtype, or NULL, or data = NULL; for N > 1 its stride is at least O in size
 *   1 <= N <= 65535, 0 <= R < 2^31, 1 <= O, C <= 2^24, N O C, N R O and N R C at most 2^40; no rows: zeros
 * dweight and dbias are written, not added to, and share no memory with other operands.  Products are exact: what the
 * checkpoint stands for is a bf16 number, dy one (bf16), two (fp16) or three (fp32) of them; bits of an fp32 dy under 2^-133, which values
 * under 2^-110 can have, are left out.
 */
liec_status liec_weight_grad(const liec_rows *dy, const liec_checkpoint *saved, const liec_matrices *dweight, const liec_param *dbias, int32_t N,
                             int64_t R, int64_t O, int64_t C, liec_dtype dtype, liec_dtype param_dtype, void *workspace,
                             int64_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* LIEC_ACTIVATIONS_H */
