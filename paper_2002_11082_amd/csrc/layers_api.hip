// libogq_layers: the C ABI declared in ogq_layers.h.  This file checks the arguments and calls the launchers (layers_launch.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>
#include <initializer_list>

#include "layers_launch.h"
#include "ogq_layers.h"

namespace ogq {

hipError_t& launch_status()
{
    static thread_local hipError_t status = hipSuccess;
    return status;
}

}  // namespace ogq

namespace {

thread_local int g_last_hip_error = 0;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

size_t size_of(uint32_t dtype) { return dtype == OGQ_FP32 ? 4 : 2; }

// The first of several checks that fails.
int first_of(std::initializer_list<int> checks)
{
    for (const int rc : checks)
        if (rc != OGQ_OK) return rc;
    return OGQ_OK;
}

// Sizes for which every offset fits 64 bits and the pieces of a tensor 31 bits of workgroups.
int check_size(size_t rows, size_t cols)
{
    constexpr size_t kMost = (size_t)1 << 31;
    if (rows >= kMost || cols >= kMost) return OGQ_ERR_SIZE;
    return rows * (cols + 127) < ((size_t)1 << 40) ? OGQ_OK : OGQ_ERR_SIZE;
}

int check_dtype(uint32_t dtype) { return dtype <= OGQ_FP16 ? OGQ_OK : OGQ_ERR_DTYPE; }

// A tensor of values: given, of a type's alignment, its offsets within 2^60.
int check_values(const void* data, size_t stride, size_t rows, uint32_t dtype)
{
    if (!data) return OGQ_ERR_NULL_POINTER;
    if (!aligned(data, size_of(dtype))) return OGQ_ERR_ALIGNMENT;
    size_t span;
    if (__builtin_mul_overflow(stride, rows, &span) || span >= ((size_t)1 << 60)) return OGQ_ERR_SIZE;
    return OGQ_OK;
}

int check_result(const void* data, size_t stride, size_t rows, size_t cols, uint32_t dtype)
{
    if (stride < cols) return OGQ_ERR_STRIDE;
    return check_values(data, stride, rows, dtype);
}

// An fp32 vector that has to be given, or one that may be left out.
int check_vector(const float* data) { return !data ? OGQ_ERR_NULL_POINTER : aligned(data, 4) ? OGQ_OK : OGQ_ERR_ALIGNMENT; }
int check_optional(const float* data) { return aligned(data, 4) ? OGQ_OK : OGQ_ERR_ALIGNMENT; }

int check_integers(const void* data, uint32_t integer)
{
    if (!data) return OGQ_ERR_NULL_POINTER;
    return aligned(data, integer == OGQ_INT32 ? 4 : 8) ? OGQ_OK : OGQ_ERR_ALIGNMENT;
}

int check_integer(uint32_t integer) { return integer <= OGQ_INT64 ? OGQ_OK : OGQ_ERR_INTEGER; }

int check_workspace(const void* data, size_t bytes, size_t need)
{
    if (need == 0) return OGQ_OK;
    if (!data) return OGQ_ERR_NULL_POINTER;
    if (bytes < need) return OGQ_ERR_WORKSPACE;
    return aligned(data, 16) ? OGQ_OK : OGQ_ERR_ALIGNMENT;
}

int check_linear(size_t tokens, size_t outs, size_t cols, uint32_t dtype)
{
    const int rc = first_of({check_dtype(dtype), check_size(tokens, cols), check_size(tokens, outs), check_size(outs, cols), check_size(cols, outs)});
    if (rc != OGQ_OK) return rc;
    // tiles, and parts of their sums, are counted in 32 bits
    return (tokens + 127) / 128 * ((outs + 127) / 128) < ((size_t)1 << 24) ? OGQ_OK : OGQ_ERR_SIZE;
}

int check_distill(size_t rows, size_t cols, uint32_t dtype, uint32_t integer, size_t top, float temperature)
{
    const int rc = first_of({check_dtype(dtype), check_integer(integer), check_size(rows, cols)});
    if (rc != OGQ_OK) return rc;
    if (top > 1024) return OGQ_ERR_SIZE;
    return temperature > 0.0f && std::isfinite(1.0f / temperature) && std::isfinite(temperature * temperature) ? OGQ_OK : OGQ_ERR_NUMBER;
}

// As in ogq.h: the status is the one the runtime returned for this call's launches.
void begin_launches() { ogq::launch_status() = hipSuccess; }

int finish_launches()
{
    const hipError_t e = ogq::launch_status();
    if (e != hipSuccess) {
        g_last_hip_error = (int)e;
        return OGQ_ERR_LAUNCH;
    }
    return OGQ_OK;
}

hipStream_t stream(void* s) { return static_cast<hipStream_t>(s); }

}  // namespace

extern "C" {

int ogq_layer_norm_forward(const void* d_x, size_t x_stride, size_t rows, size_t cols, uint32_t dtype, const float* d_weight, const float* d_bias, float eps, void* d_y,
                           size_t y_stride, float* d_mean, float* d_rstd, void* hip_stream)
{
    int rc = first_of({check_dtype(dtype), check_size(rows, cols), eps >= 0.0f && std::isfinite(eps) ? OGQ_OK : OGQ_ERR_NUMBER});
    if (rc != OGQ_OK) return rc;
    if (rows == 0 || cols == 0) return OGQ_OK;
    if (!d_mean != !d_rstd) return OGQ_ERR_PAIR;
    rc = first_of({check_values(d_x, x_stride, rows, dtype), check_result(d_y, y_stride, rows, cols, dtype), check_optional(d_weight), check_optional(d_bias),
                   check_optional(d_mean), check_optional(d_rstd)});
    if (rc != OGQ_OK) return rc;
    begin_launches();
    ogq::launch_layer_norm_forward({d_x, x_stride}, rows, cols, dtype, d_weight, d_bias, eps, {d_y, y_stride}, d_mean, d_rstd, stream(hip_stream));
    return finish_launches();
}

size_t ogq_layer_norm_backward_workspace(size_t rows, size_t cols, uint32_t dtype)
{
    if (first_of({check_dtype(dtype), check_size(rows, cols)}) != OGQ_OK || rows == 0 || cols == 0) return 0;
    return ogq::layer_norm_backward_workspace(rows, cols, dtype);
}

int ogq_layer_norm_backward(const void* d_dy, size_t dy_stride, const void* d_x, size_t x_stride, size_t rows, size_t cols, uint32_t dtype, const float* d_weight,
                            const float* d_mean, const float* d_rstd, void* d_dx, size_t dx_stride, float* d_dweight, float* d_dbias, int accumulate, void* d_workspace,
                            size_t workspace_bytes, void* hip_stream)
{
    int rc = first_of({check_dtype(dtype), check_size(rows, cols)});
    if (rc != OGQ_OK) return rc;
    if (cols == 0) return OGQ_OK;
    if (!d_dweight != !d_dbias) return OGQ_ERR_PAIR;
    if (rows == 0 && (!d_dweight || accumulate)) return OGQ_OK;
    if (d_dweight) rc = first_of({check_vector(d_dweight), check_vector(d_dbias)});
    if (rc == OGQ_OK && rows != 0) {
        rc = first_of({check_values(d_dy, dy_stride, rows, dtype), check_values(d_x, x_stride, rows, dtype), check_result(d_dx, dx_stride, rows, cols, dtype),
                       check_optional(d_weight), check_vector(d_mean), check_vector(d_rstd),
                       check_workspace(d_workspace, workspace_bytes, d_dweight ? ogq::layer_norm_backward_workspace(rows, cols, dtype) : 0)});
    }
    if (rc != OGQ_OK) return rc;
    begin_launches();
    ogq::launch_layer_norm_backward({d_dy, dy_stride}, {d_x, x_stride}, rows, cols, dtype, d_weight, d_mean, d_rstd, {d_dx, dx_stride}, d_dweight, d_dbias, accumulate != 0,
                                    d_workspace, stream(hip_stream));
    return finish_launches();
}

size_t ogq_linear_workspace(size_t tokens, size_t outs, size_t cols, uint32_t dtype, int transposed)
{
    if (check_linear(tokens, outs, cols, dtype) != OGQ_OK || tokens == 0 || outs == 0) return 0;
    return ogq::linear_workspace(tokens, outs, cols, dtype, transposed != 0);
}

int ogq_linear(const void* d_x, size_t x_stride, const void* d_weight, size_t weight_stride, int transposed, size_t tokens, size_t outs, size_t cols, uint32_t dtype,
               const float* d_bias, uint32_t activation, const void* d_residual, size_t residual_stride, void* d_y, size_t y_stride, void* d_before, size_t before_stride,
               void* d_workspace, size_t workspace_bytes, void* hip_stream)
{
    int rc = first_of({check_linear(tokens, outs, cols, dtype), activation <= OGQ_IDENTITY ? OGQ_OK : OGQ_ERR_ACTIVATION});
    if (rc != OGQ_OK) return rc;
    if (tokens == 0 || outs == 0) return OGQ_OK;
    rc = first_of({check_result(d_y, y_stride, tokens, outs, dtype), check_optional(d_bias)});
    if (rc == OGQ_OK && cols != 0) rc = first_of({check_values(d_x, x_stride, tokens, dtype), check_values(d_weight, weight_stride, transposed ? cols : outs, dtype)});
    if (rc == OGQ_OK && d_residual) rc = check_values(d_residual, residual_stride, tokens, dtype);
    if (rc == OGQ_OK && d_before) rc = check_result(d_before, before_stride, tokens, outs, dtype);
    if (rc == OGQ_OK) rc = check_workspace(d_workspace, workspace_bytes, ogq::linear_workspace(tokens, outs, cols, dtype, transposed != 0));
    if (rc != OGQ_OK) return rc;
    begin_launches();
    ogq::launch_linear({d_x, x_stride}, {d_weight, weight_stride}, transposed != 0, tokens, outs, cols, dtype, d_bias, activation, {d_residual, residual_stride},
                       {d_y, y_stride}, {d_before, before_stride}, d_workspace, stream(hip_stream));
    return finish_launches();
}

size_t ogq_linear_backward_workspace(size_t tokens, size_t outs, uint32_t dtype)
{
    if (first_of({check_dtype(dtype), check_size(tokens, outs)}) != OGQ_OK || tokens == 0 || outs == 0) return 0;
    return ogq::linear_backward_workspace(tokens, outs, dtype);
}

int ogq_linear_backward(const void* d_dy, size_t dy_stride, size_t tokens, size_t outs, uint32_t dtype, uint32_t activation, const void* d_before, size_t before_stride, void* d_dz,
                        size_t dz_stride, float* d_dbias, int accumulate, void* d_workspace, size_t workspace_bytes, void* hip_stream)
{
    int rc = first_of({check_dtype(dtype), activation <= OGQ_IDENTITY ? OGQ_OK : OGQ_ERR_ACTIVATION, check_size(tokens, outs)});
    if (rc != OGQ_OK) return rc;
    const bool identity = activation == OGQ_IDENTITY;
    if (outs == 0 || (tokens == 0 && (!d_dbias || accumulate))) return OGQ_OK;
    if (identity && (d_before || d_dz)) return OGQ_ERR_PAIR;
    rc = identity ? check_vector(d_dbias) : check_optional(d_dbias);
    if (rc == OGQ_OK && tokens != 0) {
        rc = check_values(d_dy, dy_stride, tokens, dtype);
        if (rc == OGQ_OK && !identity) rc = first_of({check_values(d_before, before_stride, tokens, dtype), check_result(d_dz, dz_stride, tokens, outs, dtype)});
        if (rc == OGQ_OK) rc = check_workspace(d_workspace, workspace_bytes, d_dbias ? ogq::linear_backward_workspace(tokens, outs, dtype) : 0);
    }
    if (rc != OGQ_OK) return rc;
    begin_launches();
    ogq::launch_linear_backward({d_dy, dy_stride}, tokens, outs, dtype, activation, {d_before, before_stride}, {d_dz, dz_stride}, d_dbias, accumulate != 0, d_workspace,
                                stream(hip_stream));
    return finish_launches();
}

int ogq_embedding_forward(const void* d_tokens, uint32_t integer, size_t tokens, const void* d_table, size_t table_stride, size_t vocab, size_t cols, uint32_t dtype, float scale,
                          void* d_y, size_t y_stride, void* hip_stream)
{
    int rc = first_of({check_integer(integer), check_dtype(dtype), check_size(tokens, cols), check_size(vocab, cols), std::isfinite(scale) ? OGQ_OK : OGQ_ERR_NUMBER});
    if (rc != OGQ_OK) return rc;
    if (tokens == 0 || cols == 0) return OGQ_OK;
    rc = first_of({check_integers(d_tokens, integer), check_result(d_y, y_stride, tokens, cols, dtype), vocab != 0 ? check_values(d_table, table_stride, vocab, dtype) : OGQ_OK});
    if (rc != OGQ_OK) return rc;
    begin_launches();
    ogq::launch_embedding_forward({d_tokens, integer}, tokens, {d_table, table_stride}, vocab, cols, dtype, scale, {d_y, y_stride}, stream(hip_stream));
    return finish_launches();
}

size_t ogq_embedding_gradient_workspace(size_t tokens, size_t vocab, size_t cols)
{
    if (first_of({check_size(tokens, cols), check_size(vocab, cols)}) != OGQ_OK || tokens >= ((size_t)1 << 30) || tokens == 0 || vocab == 0 || cols == 0) return 0;
    return ogq::embedding_gradient_workspace(tokens, vocab, cols);
}

int ogq_embedding_gradient(const void* d_tokens, uint32_t integer, size_t tokens, const void* d_dy, size_t dy_stride, size_t vocab, size_t cols, uint32_t dtype, float scale,
                           int accumulate, float* d_dtable, size_t dtable_stride, void* d_workspace, size_t workspace_bytes, void* hip_stream)
{
    int rc = first_of({check_integer(integer), check_dtype(dtype), check_size(tokens, cols), check_size(vocab, cols), std::isfinite(scale) ? OGQ_OK : OGQ_ERR_NUMBER});
    if (rc != OGQ_OK) return rc;
    if (tokens >= ((size_t)1 << 30)) return OGQ_ERR_SIZE;
    if (vocab == 0 || cols == 0 || (tokens == 0 && accumulate)) return OGQ_OK;
    rc = check_result(d_dtable, dtable_stride, vocab, cols, OGQ_FP32);
    if (rc == OGQ_OK && tokens != 0)
        rc = first_of({check_integers(d_tokens, integer), check_values(d_dy, dy_stride, tokens, dtype),
                       check_workspace(d_workspace, workspace_bytes, ogq::embedding_gradient_workspace(tokens, vocab, cols))});
    if (rc != OGQ_OK) return rc;
    begin_launches();
    ogq::launch_embedding_gradient({d_tokens, integer}, tokens, {d_dy, dy_stride}, vocab, cols, dtype, scale, accumulate != 0, {d_dtable, dtable_stride}, d_workspace,
                                   stream(hip_stream));
    return finish_launches();
}

size_t ogq_distill_workspace(size_t rows, size_t cols, uint32_t dtype, size_t top)
{
    if (check_distill(rows, cols, dtype, OGQ_INT32, top, 1.0f) != OGQ_OK || rows == 0 || cols == 0) return 0;
    return ogq::distill_workspace(rows, cols, dtype, top);
}

int ogq_distill_loss(const void* d_logits, size_t stride, size_t rows, size_t cols, uint32_t dtype, const void* d_places, uint32_t integer, const float* d_values, size_t top,
                     float temperature, const float* d_row_weight, float* d_loss, void* d_workspace, size_t workspace_bytes, void* hip_stream)
{
    int rc = check_distill(rows, cols, dtype, integer, top, temperature);
    if (rc != OGQ_OK) return rc;
    if (rows == 0) return OGQ_OK;
    rc = first_of({check_vector(d_loss), check_optional(d_row_weight), cols != 0 ? check_values(d_logits, stride, rows, dtype) : OGQ_OK,
                   top != 0 ? first_of({check_integers(d_places, integer), check_vector(d_values)}) : OGQ_OK,
                   check_workspace(d_workspace, workspace_bytes, cols != 0 ? ogq::distill_workspace(rows, cols, dtype, top) : 0)});
    if (rc != OGQ_OK) return rc;
    begin_launches();
    ogq::launch_distill({d_logits, stride}, rows, cols, dtype, {d_places, integer}, d_values, top, temperature, d_row_weight, d_loss, {nullptr, 0}, d_workspace,
                        stream(hip_stream));
    return finish_launches();
}

int ogq_distill_gradient(const void* d_logits, size_t stride, size_t rows, size_t cols, uint32_t dtype, const void* d_places, uint32_t integer, const float* d_values, size_t top,
                         float temperature, const float* d_row_weight, float* d_loss, void* d_dlogits, size_t dlogits_stride, void* d_workspace, size_t workspace_bytes,
                         void* hip_stream)
{
    int rc = check_distill(rows, cols, dtype, integer, top, temperature);
    if (rc != OGQ_OK) return rc;
    if (rows == 0 || (cols == 0 && !d_loss)) return OGQ_OK;
    rc = first_of({check_optional(d_loss), check_optional(d_row_weight), cols != 0 ? check_values(d_logits, stride, rows, dtype) : OGQ_OK,
                   cols != 0 ? check_result(d_dlogits, dlogits_stride, rows, cols, dtype) : OGQ_OK,
                   top != 0 ? first_of({check_integers(d_places, integer), check_vector(d_values)}) : OGQ_OK,
                   check_workspace(d_workspace, workspace_bytes, cols != 0 ? ogq::distill_workspace(rows, cols, dtype, top) : 0)});
    if (rc != OGQ_OK) return rc;
    begin_launches();
    ogq::launch_distill({d_logits, stride}, rows, cols, dtype, {d_places, integer}, d_values, top, temperature, d_row_weight, d_loss, {d_dlogits, dlogits_stride},
                        d_workspace, stream(hip_stream));
    return finish_launches();
}

const char* ogq_layers_strerror(int status)
{
    switch (status) {
        case OGQ_OK: return "ok";
        case OGQ_ERR_NULL_POINTER: return "a required pointer is NULL";
        case OGQ_ERR_ALIGNMENT: return "workspaces must be 16-byte aligned, values and integers aligned to their type";
        case OGQ_ERR_LAUNCH: return "HIP kernel launch failed";
        case OGQ_ERR_SIZE: return "a tensor, its stride or the number of places is too large for one call";
        case OGQ_ERR_GROUP_SIZE: return "group_size must be 32, 64 or 128";
        case OGQ_ERR_GROUP_BITS: return "bits must be 8 or 4: 8 for activations and weight gradients, 4 for products with weights";
        case OGQ_ERR_DTYPE: return "unknown type of values";
        case OGQ_ERR_ACTIVATION: return "unknown activation";
        case OGQ_ERR_STRIDE: return "the stride of an output is less than its columns";
        case OGQ_ERR_WORKSPACE: return "the workspace is too small";
        case OGQ_ERR_PAIR: return "of pointers that belong together only some are given, or one is given that the call does not have";
        case OGQ_ERR_INTEGER: return "unknown type of integers";
        case OGQ_ERR_NUMBER: return "eps must be finite and not negative, a scale finite, a temperature positive with an inverse and a square";
        default: return "unknown status";
    }
}

int ogq_layers_last_hip_error(void) { return g_last_hip_error; }

}  // extern "C"
