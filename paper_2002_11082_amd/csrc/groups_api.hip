// libogq_groups: the C ABI declared in ogq_groups.h.  This file checks the arguments and calls the launchers (groups_launch.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <initializer_list>

#include "groups_launch.h"
#include "ogq_groups.h"

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

size_t padded(size_t cols, const ogq_group_params_t* p) { return (cols + p->group_size - 1) / p->group_size * p->group_size; }

bool exist(const ogq_group_params_t* p)
{
    return p && (p->group_size == 32 || p->group_size == 64 || p->group_size == 128) && (p->bits == 8 || p->bits == 4);
}

int check_params(const ogq_group_params_t* p, uint32_t bits)
{
    if (!p) return OGQ_ERR_NULL_POINTER;
    if (p->group_size != 32 && p->group_size != 64 && p->group_size != 128) return OGQ_ERR_GROUP_SIZE;
    if (bits ? p->bits != bits : p->bits != 8 && p->bits != 4) return OGQ_ERR_GROUP_BITS;
    return OGQ_OK;
}

// Sizes for which every offset fits 64 bits and the pieces of a tensor 31 bits of workgroups.
int check_size(size_t rows, size_t cols)
{
    constexpr size_t kMost = (size_t)1 << 31;
    if (rows >= kMost || cols >= kMost) return OGQ_ERR_SIZE;
    return rows * (cols + 127) < ((size_t)1 << 40) ? OGQ_OK : OGQ_ERR_SIZE;
}

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

int check_groups(const void* codes, const uint8_t* exponents)
{
    if (!codes || !exponents) return OGQ_ERR_NULL_POINTER;
    return aligned(codes, 16) ? OGQ_OK : OGQ_ERR_ALIGNMENT;
}

// The first of several checks that fails.
int first_of(std::initializer_list<int> checks)
{
    for (const int rc : checks)
        if (rc != OGQ_OK) return rc;
    return OGQ_OK;
}

int check_dtype(uint32_t dtype) { return dtype <= OGQ_FP16 ? OGQ_OK : OGQ_ERR_DTYPE; }

// The least tiles that the kernels for sums cut `a` by `b` of them into, `wide` of b to one, to workgroups of 256 threads in one dimension: 2^32 threads are too many for a launch.
int check_tiles(size_t a, size_t b, size_t wide)
{
    return (a + 127) / 128 * ((b + wide - 1) / wide) < ((size_t)1 << 24) ? OGQ_OK : OGQ_ERR_SIZE;
}

int check_gradient(size_t rows, size_t outs, size_t cols, uint32_t dtype, const ogq_group_params_t* params)
{
    return first_of({check_params(params, 8), check_dtype(dtype), check_size(rows, cols), check_size(rows, outs), check_size(outs, cols), check_tiles(outs, cols, 128)});
}

int check_product(size_t tokens, size_t outs, size_t cols, uint32_t dtype, const ogq_group_params_t* params)
{
    return first_of({check_params(params, 4), check_dtype(dtype), check_size(outs, cols), check_size(tokens, cols), check_size(tokens, outs),
                     tokens > 1 ? check_tiles(outs, tokens, 64) : OGQ_OK});
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

ogq::Groups groups(const void* codes, const uint8_t* exponents)
{
    return {const_cast<void*>(codes), const_cast<uint8_t*>(exponents)};
}

}  // namespace

extern "C" {

size_t ogq_group_codes_bytes(size_t rows, size_t cols, const ogq_group_params_t* p)
{
    return exist(p) ? rows * (padded(cols, p) * p->bits / 8) : 0;
}

size_t ogq_group_exponents_count(size_t rows, size_t cols, const ogq_group_params_t* p)
{
    return exist(p) ? rows * (padded(cols, p) / p->group_size) : 0;
}

int ogq_group_quantize(const void* d_x, size_t stride, size_t rows, size_t cols, uint32_t dtype, const ogq_group_params_t* params,
                       void* d_codes, uint8_t* d_exponents, void* hip_stream)
{
    int rc = first_of({check_params(params, 0), check_dtype(dtype), check_size(rows, cols)});
    if (rc != OGQ_OK) return rc;
    if (rows == 0 || cols == 0) return OGQ_OK;
    rc = first_of({check_values(d_x, stride, rows, dtype), check_groups(d_codes, d_exponents)});
    if (rc != OGQ_OK) return rc;
    begin_launches();
    ogq::launch_group_quantize({d_x, stride}, rows, cols, dtype, params, groups(d_codes, d_exponents), static_cast<hipStream_t>(hip_stream));
    return finish_launches();
}

int ogq_group_dequantize(const void* d_codes, const uint8_t* d_exponents, size_t rows, size_t cols, const ogq_group_params_t* params,
                         void* d_out, size_t stride, uint32_t dtype, void* hip_stream)
{
    int rc = first_of({check_params(params, 0), check_dtype(dtype), check_size(rows, cols)});
    if (rc != OGQ_OK) return rc;
    if (rows == 0 || cols == 0) return OGQ_OK;
    rc = first_of({check_groups(d_codes, d_exponents), check_result(d_out, stride, rows, cols, dtype)});
    if (rc != OGQ_OK) return rc;
    begin_launches();
    ogq::launch_group_dequantize(groups(d_codes, d_exponents), rows, cols, params, {d_out, stride}, dtype, static_cast<hipStream_t>(hip_stream));
    return finish_launches();
}

int ogq_activation_forward(const void* d_x, size_t x_stride, const void* d_up, size_t up_stride, size_t rows, size_t cols, uint32_t dtype,
                           uint32_t activation, const ogq_group_params_t* params, void* d_y, size_t y_stride, void* d_codes,
                           uint8_t* d_exponents, void* d_up_codes, uint8_t* d_up_exponents, void* hip_stream)
{
    const bool gated = d_up || d_up_codes || d_up_exponents;
    int rc = first_of({check_params(params, 8), check_dtype(dtype), activation <= OGQ_SILU ? OGQ_OK : OGQ_ERR_ACTIVATION, check_size(rows, cols)});
    if (rc != OGQ_OK) return rc;
    if (rows == 0 || cols == 0) return OGQ_OK;
    if (gated && !(d_up && d_up_codes && d_up_exponents)) return OGQ_ERR_PAIR;
    rc = first_of({check_values(d_x, x_stride, rows, dtype), check_result(d_y, y_stride, rows, cols, dtype), check_groups(d_codes, d_exponents),
                   gated ? check_values(d_up, up_stride, rows, dtype) : OGQ_OK, gated ? check_groups(d_up_codes, d_up_exponents) : OGQ_OK});
    if (rc != OGQ_OK) return rc;
    begin_launches();
    ogq::launch_activation_forward({d_x, x_stride}, {d_up, up_stride}, rows, cols, dtype, activation, params, {d_y, y_stride},
                                   groups(d_codes, d_exponents), groups(d_up_codes, d_up_exponents), static_cast<hipStream_t>(hip_stream));
    return finish_launches();
}

int ogq_activation_backward(const void* d_dy, size_t dy_stride, const void* d_codes, const uint8_t* d_exponents, const void* d_up_codes,
                            const uint8_t* d_up_exponents, size_t rows, size_t cols, uint32_t dtype, uint32_t activation,
                            const ogq_group_params_t* params, void* d_dx, size_t dx_stride, void* d_dup, size_t dup_stride, void* hip_stream)
{
    const bool gated = d_up_codes || d_up_exponents || d_dup;
    int rc = first_of({check_params(params, 8), check_dtype(dtype), activation <= OGQ_SILU ? OGQ_OK : OGQ_ERR_ACTIVATION, check_size(rows, cols)});
    if (rc != OGQ_OK) return rc;
    if (rows == 0 || cols == 0) return OGQ_OK;
    if (gated && !(d_up_codes && d_up_exponents && d_dup)) return OGQ_ERR_PAIR;
    rc = first_of({check_values(d_dy, dy_stride, rows, dtype), check_groups(d_codes, d_exponents), check_result(d_dx, dx_stride, rows, cols, dtype),
                   gated ? check_groups(d_up_codes, d_up_exponents) : OGQ_OK, gated ? check_result(d_dup, dup_stride, rows, cols, dtype) : OGQ_OK});
    if (rc != OGQ_OK) return rc;
    begin_launches();
    ogq::launch_activation_backward({d_dy, dy_stride}, groups(d_codes, d_exponents), groups(d_up_codes, d_up_exponents), rows, cols, dtype, activation,
                                    params, {d_dx, dx_stride}, {d_dup, dup_stride}, static_cast<hipStream_t>(hip_stream));
    return finish_launches();
}

size_t ogq_weight_gradient_workspace(size_t rows, size_t outs, size_t cols, uint32_t dtype, const ogq_group_params_t* params)
{
    if (check_gradient(rows, outs, cols, dtype, params) != OGQ_OK) return 0;
    if (outs == 0 || cols == 0) return 0;
    return ogq::weight_gradient_workspace(rows, outs, cols, dtype);
}

int ogq_weight_gradient(const void* d_dy, size_t dy_stride, uint32_t dtype, const void* d_codes, const uint8_t* d_exponents, size_t rows,
                        size_t outs, size_t cols, const ogq_group_params_t* params, int accumulate, float* d_dw, size_t dw_stride,
                        void* d_workspace, size_t workspace_bytes, void* hip_stream)
{
    int rc = check_gradient(rows, outs, cols, dtype, params);
    if (rc != OGQ_OK) return rc;
    if (outs == 0 || cols == 0 || (rows == 0 && accumulate)) return OGQ_OK;
    rc = check_result(d_dw, dw_stride, outs, cols, OGQ_FP32);
    if (rc == OGQ_OK && rows != 0) {
        rc = first_of({check_values(d_dy, dy_stride, rows, dtype), check_groups(d_codes, d_exponents)});
    }
    if (rc != OGQ_OK) return rc;
    const size_t need = ogq::weight_gradient_workspace(rows, outs, cols, dtype);
    if (need != 0) {
        if (!d_workspace) return OGQ_ERR_NULL_POINTER;
        if (workspace_bytes < need) return OGQ_ERR_WORKSPACE;
        if (!aligned(d_workspace, 16)) return OGQ_ERR_ALIGNMENT;
    }
    begin_launches();
    ogq::launch_weight_gradient({d_dy, dy_stride}, dtype, groups(d_codes, d_exponents), rows, outs, cols, params, accumulate != 0, d_dw, dw_stride,
                                d_workspace, static_cast<hipStream_t>(hip_stream));
    return finish_launches();
}

size_t ogq_group_matvec_workspace(size_t tokens, size_t outs, size_t cols, uint32_t dtype, const ogq_group_params_t* params)
{
    if (check_product(tokens, outs, cols, dtype, params) != OGQ_OK) return 0;
    if (tokens == 0 || outs == 0) return 0;
    return ogq::group_matvec_workspace(tokens, outs, cols, dtype);
}

int ogq_group_matvec(const void* d_codes, const uint8_t* d_exponents, size_t outs, size_t cols, const ogq_group_params_t* params, const void* d_x,
                     size_t x_stride, size_t tokens, uint32_t dtype, void* d_y, size_t y_stride, void* d_workspace, size_t workspace_bytes,
                     void* hip_stream)
{
    int rc = check_product(tokens, outs, cols, dtype, params);
    if (rc != OGQ_OK) return rc;
    if (tokens == 0 || outs == 0) return OGQ_OK;
    rc = check_result(d_y, y_stride, tokens, outs, dtype);
    if (rc == OGQ_OK && cols != 0) rc = first_of({check_values(d_x, x_stride, tokens, dtype), check_groups(d_codes, d_exponents)});
    if (rc != OGQ_OK) return rc;
    const size_t need = ogq::group_matvec_workspace(tokens, outs, cols, dtype);
    if (need != 0) {
        if (!d_workspace) return OGQ_ERR_NULL_POINTER;
        if (workspace_bytes < need) return OGQ_ERR_WORKSPACE;
        if (!aligned(d_workspace, 16)) return OGQ_ERR_ALIGNMENT;
    }
    begin_launches();
    ogq::launch_group_matvec(groups(d_codes, d_exponents), outs, cols, params, {d_x, x_stride}, tokens, dtype, {d_y, y_stride}, d_workspace,
                             static_cast<hipStream_t>(hip_stream));
    return finish_launches();
}

const char* ogq_groups_strerror(int status)
{
    switch (status) {
        case OGQ_OK: return "ok";
        case OGQ_ERR_NULL_POINTER: return "a required pointer is NULL";
        case OGQ_ERR_ALIGNMENT: return "codes and workspaces must be 16-byte aligned, values aligned to their type";
        case OGQ_ERR_LAUNCH: return "HIP kernel launch failed";
        case OGQ_ERR_SIZE: return "the tensor or its stride is too large for one call";
        case OGQ_ERR_GROUP_SIZE: return "group_size must be 32, 64 or 128";
        case OGQ_ERR_GROUP_BITS: return "bits must be 8 or 4: 8 for activations and weight gradients, 4 for products with weights";
        case OGQ_ERR_DTYPE: return "unknown type of values";
        case OGQ_ERR_ACTIVATION: return "unknown activation";
        case OGQ_ERR_STRIDE: return "the stride of an output is less than its columns";
        case OGQ_ERR_WORKSPACE: return "the workspace is too small";
        case OGQ_ERR_PAIR: return "of the second factor's pointers only some are given";
        default: return "unknown status";
    }
}

int ogq_groups_last_hip_error(void) { return g_last_hip_error; }

}  // extern "C"
