/*
 * ogq_groups.h -- C ABI of libogq_groups: tensors held in groups of 8 or 4 bits, and the operators of a training or
 * serving program that read them, on one MI355X (gfx950).
 *
 * The gradient that ogq_quantize sends is made from activations that wait for the backward pass, and what it trains is
 * served afterwards.  Activations are held in 8 bits (a checkpoint) until the backward pass reads them, weights in 4 bits.
 *
 * The format.  A tensor [rows, cols] is cut into groups of `group_size` consecutive values of a row; the last group of a
 * row may be short.  A group has one exponent e and every value one code q, and stands for q * 2^e:
 *   8 bits   q = -127 .. 127
 *   4 bits   q = 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign
 * e is the smallest integer with |x| <= Q * 2^e for all values of the group (Q = 127 or 6), limited so that every q * 2^e is a
 * value of the tensor's type: -126 .. 121 (8 bits) and -125 .. 125 (4 bits) for fp32 and bf16, -24 .. 9 and -23 .. 13 for fp16.
 * q is x * 2^-e rounded to the nearest code, ties to the even one, and at most Q (which is less only at the upper limit of e).
 * A shared power of two makes q * 2^e exact in bf16 (and in fp16 where the tensor was fp16): what is read back needs no
 * rounding, and the products of the matrix cores below are exact.
 * A group that holds an infinity or a NaN stands for NaN in all of its values.
 *
 * In memory:
 *   exponents  uint8 [rows][groups], groups = ceil(cols / group_size): e + 127; 255 in a group of NaN, whose codes are 0
 *   codes      [rows][groups * group_size] values; 8 bits: one byte each, two's complement; 4 bits: two in a byte, the first in
 *              the low four bits, bit 3 the sign and bits 0..2 the index in the list above.  What lies behind a row's last value is 0.
 *
 * Conventions for every entry point
 *   - Those of ogq.h: device pointers d_*, work enqueued on `hip_stream`, no synchronising, nothing allocated, no state kept
 *     but the code read by ogq_groups_last_hip_error(), a negative status on an error and nothing enqueued then.
 *   - d_codes must be 16-byte aligned; values (d_x, d_y and so on) need the alignment of their type.
 *   - A tensor of values has consecutive values in a row and `stride` values from one row to the next: at least cols for
 *     outputs, any for inputs (0: the same row again and again).
 *   - Rows and columns are below 2^31, rows * (columns + 127) of every tensor below 2^40; of sums, outs * cols and (for more than one token) tokens * outs below 2^38 and 2^37 in whole
 *     tiles of 128 x 128 and 64 x 128.  Else OGQ_ERR_SIZE.
 *   - Outputs overlap neither inputs nor each other.
 *   - A tensor without values (0 rows or 0 columns) is a successful no-op, apart from sums over nothing, which are 0.
 *   - A call with a workspace may be two launches; where the runtime refuses the second, the first is enqueued all the same.
 */
#ifndef OGQ_GROUPS_H
#define OGQ_GROUPS_H

#include "ogq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Status codes besides those of ogq.h. */
enum {
    OGQ_ERR_GROUP_SIZE = -20, /* group_size is not 32, 64 or 128 */
    OGQ_ERR_GROUP_BITS = -21, /* bits is not 8 or 4, or not what the operator reads */
    OGQ_ERR_DTYPE = -22,      /* unknown type of values */
    OGQ_ERR_ACTIVATION = -23, /* unknown activation */
    OGQ_ERR_STRIDE = -24,     /* the stride of an output is less than its columns */
    OGQ_ERR_WORKSPACE = -25,  /* the workspace is smaller than the size helper says */
    OGQ_ERR_PAIR = -26        /* of the second factor's pointers only some are given */
};

typedef enum { OGQ_FP32 = 0, OGQ_BF16 = 1, OGQ_FP16 = 2 } ogq_dtype_t;

typedef enum {
    OGQ_RELU = 0,      /* max(x, 0) */
    OGQ_GELU = 1,      /* x * (1 + erf(x / sqrt(2))) / 2 */
    OGQ_GELU_TANH = 2, /* x * (1 + tanh(sqrt(2 / pi) * (x + 0.044715 x^3))) / 2 */
    OGQ_SILU = 3       /* x / (1 + exp(-x)) */
} ogq_activation_t;

typedef struct {
    uint32_t group_size; /* 32, 64 or 128 */
    uint32_t bits;       /* 8 or 4 */
} ogq_group_params_t;

/* Bytes of the codes and number of exponents of a tensor; 0 for parameters that do not exist. */
size_t ogq_group_codes_bytes(size_t rows, size_t cols, const ogq_group_params_t* params);
size_t ogq_group_exponents_count(size_t rows, size_t cols, const ogq_group_params_t* params);

/* A tensor into groups, 8 or 4 bits. */
int ogq_group_quantize(const void* d_x, size_t stride, size_t rows, size_t cols, uint32_t dtype,
                       const ogq_group_params_t* params, void* d_codes, uint8_t* d_exponents, void* hip_stream);

/* The values that codes and exponents stand for, 8 or 4 bits.  Exact where `dtype` is the type that was quantized (and in
 * fp32); values beyond the largest fp16 come out as infinities there. */
int ogq_group_dequantize(const void* d_codes, const uint8_t* d_exponents, size_t rows, size_t cols,
                         const ogq_group_params_t* params, void* d_out, size_t stride, uint32_t dtype, void* hip_stream);

/* The forward pass of an activation, which leaves what the backward pass needs in 8 bits:
 *   y = act(x), or y = act(x) * up where d_up is given,
 * from the values as they are, and x (and up) in groups.  Computed in fp32 and rounded once: fp32 results are off by 12 to 16 roundings
 * (gelu_tanh: and 13 |x + 0.045 x^3| more), for 16 bits the value that is rounded is off by 2^-15 of itself and may be 0 below 2^-119.  d_up, d_up_codes and
 * d_up_exponents are all given or all NULL. */
int ogq_activation_forward(const void* d_x, size_t x_stride, const void* d_up, size_t up_stride, size_t rows, size_t cols,
                           uint32_t dtype, uint32_t activation, const ogq_group_params_t* params, void* d_y, size_t y_stride,
                           void* d_codes, uint8_t* d_exponents, void* d_up_codes, uint8_t* d_up_exponents, void* hip_stream);

/* Its backward pass, from the values x^ and up^ that the groups stand for:
 *   dx = dy * act'(x^), or dx = dy * up^ * act'(x^) and dup = dy * act(x^),
 * computed in fp32, rounded once.  relu'(0) = 0.  d_up_codes, d_up_exponents and d_dup are all given or all NULL. */
int ogq_activation_backward(const void* d_dy, size_t dy_stride, const void* d_codes, const uint8_t* d_exponents,
                            const void* d_up_codes, const uint8_t* d_up_exponents, size_t rows, size_t cols, uint32_t dtype,
                            uint32_t activation, const ogq_group_params_t* params, void* d_dx, size_t dx_stride, void* d_dup,
                            size_t dup_stride, void* hip_stream);

/* The gradient of a linear layer's weights from the gradient of its outputs and its checkpointed inputs (8 bits):
 *   dw[o][i] = sum over the rows t of dy[t][o] * x^[t][i],  0 <= o < outs, 0 <= i < cols,
 * or that added to what dw holds (accumulate != 0).  Products are exact (fp32 gradients are cut into three pieces of bf16, in which
 * what a value has below 2^-133 is lost), sums are held in fp32 in an order that the sizes alone decide.  The checkpoint may be one of any type; fp16 gradients are multiplied
 * fastest where its exponents are an fp16 tensor's (-24 .. 9): tiles of sums that meet others are made again, as products of bf16 in an order of their own.
 * d_workspace: ogq_weight_gradient_workspace bytes, 16-byte aligned, may be NULL where that is 0. */
size_t ogq_weight_gradient_workspace(size_t rows, size_t outs, size_t cols, uint32_t dtype, const ogq_group_params_t* params);
int ogq_weight_gradient(const void* d_dy, size_t dy_stride, uint32_t dtype, const void* d_codes, const uint8_t* d_exponents,
                        size_t rows, size_t outs, size_t cols, const ogq_group_params_t* params, int accumulate, float* d_dw,
                        size_t dw_stride, void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* Tokens times the transpose of weights held in 4 bits (codes and exponents of a tensor [outs, cols]):
 *   y[t][o] = sum over i of x[t][i] * w^[o][i],  0 <= t < tokens, 0 <= o < outs.
 * Products are exact (for the matrix cores x is cut into pieces of bf16: one for bf16, two for fp16, three for fp32; on the vector unit, which
 * takes up to four tokens, they are those of a dot product or a fused multiply-add; what an fp32 value has below 2^-133 may be lost in
 * the pieces), sums are held in fp32 in an order that the sizes alone decide and rounded once.  Workspace as above. */
size_t ogq_group_matvec_workspace(size_t tokens, size_t outs, size_t cols, uint32_t dtype, const ogq_group_params_t* params);
int ogq_group_matvec(const void* d_codes, const uint8_t* d_exponents, size_t outs, size_t cols, const ogq_group_params_t* params,
                     const void* d_x, size_t x_stride, size_t tokens, uint32_t dtype, void* d_y, size_t y_stride,
                     void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* Text for a status code, those of ogq.h included (static storage, never NULL). */
const char* ogq_groups_strerror(int status);

/* The hipError_t value of the last failed launch of this library on this thread (0 if none). */
int ogq_groups_last_hip_error(void);

#ifdef __cplusplus
}
#endif
#endif /* OGQ_GROUPS_H */
