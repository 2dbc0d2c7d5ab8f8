// Internal header of libogq_groups: the host-side launchers that groups_api.hip calls.
#ifndef OGQ_GROUPS_LAUNCH_H
#define OGQ_GROUPS_LAUNCH_H

#include "launch.h"
#include "ogq_groups.h"

namespace ogq {

// groups_elementwise.hip, groups_gradient.hip, groups_matvec.hip.  Arguments already checked, no tensor without values (but for sums over nothing).
struct Values {
    const void* data;
    size_t stride;
};
struct Result {
    void* data;
    size_t stride;
};
struct Groups {
    void* codes;
    uint8_t* exponents;
};
void launch_group_quantize(const Values& x, size_t rows, size_t cols, uint32_t dtype, const ogq_group_params_t* p,
                           const Groups& to, hipStream_t st);
void launch_group_dequantize(const Groups& from, size_t rows, size_t cols, const ogq_group_params_t* p, const Result& out,
                             uint32_t dtype, hipStream_t st);
void launch_activation_forward(const Values& x, const Values& up, size_t rows, size_t cols, uint32_t dtype, uint32_t act,
                               const ogq_group_params_t* p, const Result& y, const Groups& x_to, const Groups& up_to, hipStream_t st);
void launch_activation_backward(const Values& dy, const Groups& x, const Groups& up, size_t rows, size_t cols, uint32_t dtype,
                                uint32_t act, const ogq_group_params_t* p, const Result& dx, const Result& dup, hipStream_t st);
size_t weight_gradient_workspace(size_t rows, size_t outs, size_t cols, uint32_t dtype);
void launch_weight_gradient(const Values& dy, uint32_t dtype, const Groups& x, size_t rows, size_t outs, size_t cols,
                            const ogq_group_params_t* p, bool accumulate, float* dw, size_t dw_stride, void* workspace, hipStream_t st);
size_t group_matvec_workspace(size_t tokens, size_t outs, size_t cols, uint32_t dtype);
void launch_group_matvec(const Groups& w, size_t outs, size_t cols, const ogq_group_params_t* p, const Values& x, size_t tokens,
                         uint32_t dtype, const Result& y, void* workspace, hipStream_t st);

}  // namespace ogq
#endif  // OGQ_GROUPS_LAUNCH_H
