/*
 * ogq_layers.h -- C ABI of libogq_layers: what a training or serving program computes before, between and behind the operators of
 * ogq_groups.h, on one MI355X (gfx950): rows of a table by tokens, layer norm, a linear layer's product with its bias, activation and residual,
 * and the divergence from a teacher's distribution, each with its gradients.
 *
 * A linear layer's weight gradient is ogq_weight_gradient of ogq_groups.h; gradients of other parameters are made here, in fp32 as there, so that all of
 * them can lie in the flat gradient that ogq_quantize sends.
 *
 * Conventions for every entry point
 *   - Those of ogq.h: device pointers d_*, work enqueued on `hip_stream`, no synchronising, nothing allocated, no state kept
 *     but the code read by ogq_layers_last_hip_error(), a negative status on an error and nothing enqueued then.
 *   - A tensor of values is in one of the types of ogq_dtype_t, aligned to it, with consecutive values in a row and `stride` values from one row to the next: at
 *     least the columns for outputs, any for inputs (0: the same row again and again).  Weights and biases that are vectors are consecutive fp32.
 *   - Integers (tokens, places) are of one of the types of ogq_integer_t, aligned to it.
 *   - Rows and columns are below 2^31, rows * (columns + 127) of every tensor below 2^40, and where a text below says so less.  Else OGQ_ERR_SIZE.
 *   - Outputs overlap neither inputs nor each other, but where a text below allows it.
 *   - Outputs without values are a successful no-op; sums over nothing are 0.
 *   - d_workspace: as many bytes as the size helper beside the entry point says, 16-byte aligned, may be NULL where that is 0.  Its contents before the call do not matter.  Calls that may
 *     run at the same time, replays of captured graphs among them, need workspaces of their own.
 *   - A call may be several launches; where the runtime refuses one, those before it are enqueued all the same.
 *   - Sums are held in fp32 (or more) in an order that the sizes alone decide (and the tokens, where a text below says so): results are the same from call to call.  Values are rounded once, to the type of the output; outputs in fp32 are as
 *     exact for inputs in 16 bits as for those in fp32.
 */
#ifndef OGQ_LAYERS_H
#define OGQ_LAYERS_H

#include "ogq_groups.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Status codes besides those of ogq.h and ogq_groups.h. */
enum {
    OGQ_ERR_INTEGER = -30, /* unknown type of integers */
    OGQ_ERR_NUMBER = -31   /* eps is negative or not finite, a scale not finite, a temperature not a positive number with an inverse */
};

typedef enum { OGQ_INT32 = 0, OGQ_INT64 = 1 } ogq_integer_t;

/* No activation, besides those of ogq_activation_t. */
enum { OGQ_IDENTITY = 4 };

/* Layer norm of every row:
 *   y = (x - mean) * rstd * weight + bias,  rstd = 1 / sqrt(mean of (x - mean)^2 + eps).
 * d_weight, d_bias: [cols], or NULL for 1 and 0.  d_mean, d_rstd: [rows], for the backward pass, both given or both NULL (without columns neither is written).  The variance is that of the differences from the mean, not
 * one of squares; where it is beyond fp32 (differences of about 2^63 and more), rstd is 0 and y the bias. */
int ogq_layer_norm_forward(const void* d_x, size_t x_stride, size_t rows, size_t cols, uint32_t dtype, const float* d_weight, const float* d_bias, float eps, void* d_y,
                           size_t y_stride, float* d_mean, float* d_rstd, void* hip_stream);

/* Its backward pass.  With u = (x - mean) * rstd and g = dy * weight:
 *   dx = rstd * (g - mean of g - u * mean of (g * u)),   dweight = sum over the rows of dy * u,   dbias = sum over the rows of dy,
 * the last two in fp32 [cols], or added to what they hold (accumulate != 0).  In rows that lie more than 16 deviations from zero what the mean's rounding to fp32 leaves in u, whose mean over
 * a row is 0, is taken off it again, so that an offset costs no more than in the forward pass.  Rows whose rstd is 0 have dx 0 and no part in dweight.  d_dweight and d_dbias are both given or both NULL, and without them there is no workspace.  d_dx may be
 * d_dy with the same stride. */
size_t ogq_layer_norm_backward_workspace(size_t rows, size_t cols, uint32_t dtype);
int ogq_layer_norm_backward(const void* d_dy, size_t dy_stride, const void* d_x, size_t x_stride, size_t rows, size_t cols, uint32_t dtype, const float* d_weight,
                            const float* d_mean, const float* d_rstd, void* d_dx, size_t dx_stride, float* d_dweight, float* d_dbias, int accumulate, void* d_workspace,
                            size_t workspace_bytes, void* hip_stream);

/* A linear layer: z = x W^T + bias, y = act(z) + residual, x [tokens, cols], W [outs, cols], y [tokens, outs]; all of one type but the bias.
 * transposed != 0: W is [cols, outs], z = x W + bias: with a layer's own weights and the gradient of its outputs for x, the gradient of its inputs.
 * d_bias, d_residual: NULL for none.  d_before: z as well, for the backward pass, NULL for no need of it.
 * activation: one of ogq_activation_t or OGQ_IDENTITY.  Products of 16-bit types are exact; those of fp32 are made of pieces of bf16, less than 2^-21 of a product's size nearer
 * to zero, and what a value has below 2^-133 may be lost in them.  d_y may be d_residual with the same stride.  tokens * outs below 2^38 in whole tiles of 128 x 128. */
size_t ogq_linear_workspace(size_t tokens, size_t outs, size_t cols, uint32_t dtype, int transposed);
int ogq_linear(const void* d_x, size_t x_stride, const void* d_weight, size_t weight_stride, int transposed, size_t tokens, size_t outs, size_t cols, uint32_t dtype,
               const float* d_bias, uint32_t activation, const void* d_residual, size_t residual_stride, void* d_y, size_t y_stride, void* d_before, size_t before_stride,
               void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* What the backward pass of such a layer begins with: dz = dy * act'(z), z from d_before, and the bias' gradient, the sum of dz over the tokens (as it is before dz is rounded), in fp32
 * [outs], or added to what d_dbias holds.  The gradient of the residual is dy, that of x ogq_linear's with dz and the weights, that of the weights ogq_weight_gradient's.
 * Where z was beyond fp16, and is infinite in d_before, act' is
 * what it is far out: 0 or 1.  OGQ_IDENTITY: dz is dy, d_before and d_dz are NULL.  d_dbias may be NULL otherwise.  d_dz may be d_dy or d_before with the same stride. */
size_t ogq_linear_backward_workspace(size_t tokens, size_t outs, uint32_t dtype);
int ogq_linear_backward(const void* d_dy, size_t dy_stride, size_t tokens, size_t outs, uint32_t dtype, uint32_t activation, const void* d_before, size_t before_stride, void* d_dz,
                        size_t dz_stride, float* d_dbias, int accumulate, void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* Rows of a table [vocab, cols] by tokens, y[t] = scale * table[token[t]].  A token outside of 0 .. vocab - 1 stands for none: its row of y is 0. */
int ogq_embedding_forward(const void* d_tokens, uint32_t integer, size_t tokens, const void* d_table, size_t table_stride, size_t vocab, size_t cols, uint32_t dtype, float scale,
                          void* d_y, size_t y_stride, void* hip_stream);

/* The table's gradient [vocab, cols] in fp32, dtable[v] = scale * sum of dy[t] over the t with token[t] = v (0 where there is none), or that added to what dtable holds.  Tokens outside
 * of the table have no part in it.  The rows of a token are added in their order, in groups that all of the tokens
 * decide.  tokens below 2^30. */
size_t ogq_embedding_gradient_workspace(size_t tokens, size_t vocab, size_t cols);
int ogq_embedding_gradient(const void* d_tokens, uint32_t integer, size_t tokens, const void* d_dy, size_t dy_stride, size_t vocab, size_t cols, uint32_t dtype, float scale,
                           int accumulate, float* d_dtable, size_t dtable_stride, void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* Distillation from a teacher's largest logits: `top` places of a row of `cols` logits and the teacher's logits there.  With temperature T,
 *   p = softmax of values / T over the row's places,  q = softmax of logits / T over its columns,
 *   loss = row_weight * T^2 * sum over the places of p * (log p - log q[place]),   the gradient of the logits dlogits = row_weight * T * (q - p at its places).
 * d_places: [rows, top] consecutive, d_values: fp32 [rows, top] consecutive; a place outside of 0 .. cols - 1 stands for none, of places that are the same each counts.  One place with
 * any value is the cross entropy of a label.  Rows without a place, or whose values are all -infinity, have loss 0 and gradient 0; so have rows of row_weight 0, and what they hold is
 * not looked at.  d_row_weight: [rows], NULL for 1 everywhere.  A logit of -infinity has q = 0, and the loss is infinite where p is not 0 there.  A row in which a logit or a value is NaN or +infinity
 * has NaN for both.  d_loss: fp32 [rows]; for the gradient it may be NULL.  top is at most 1024.  d_dlogits may be d_logits with the same stride. */
size_t ogq_distill_workspace(size_t rows, size_t cols, uint32_t dtype, size_t top);
int ogq_distill_loss(const void* d_logits, size_t stride, size_t rows, size_t cols, uint32_t dtype, const void* d_places, uint32_t integer, const float* d_values, size_t top,
                     float temperature, const float* d_row_weight, float* d_loss, void* d_workspace, size_t workspace_bytes, void* hip_stream);
int ogq_distill_gradient(const void* d_logits, size_t stride, size_t rows, size_t cols, uint32_t dtype, const void* d_places, uint32_t integer, const float* d_values, size_t top,
                         float temperature, const float* d_row_weight, float* d_loss, void* d_dlogits, size_t dlogits_stride, void* d_workspace, size_t workspace_bytes,
                         void* hip_stream);

/* Text for a status code, those of ogq.h and ogq_groups.h included (static storage, never NULL). */
const char* ogq_layers_strerror(int status);

/* The hipError_t value of the last failed launch of this library on this thread (0 if none). */
int ogq_layers_last_hip_error(void);

#ifdef __cplusplus
}
#endif
#endif /* OGQ_LAYERS_H */
