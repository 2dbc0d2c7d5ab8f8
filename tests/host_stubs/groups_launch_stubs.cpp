// Test infrastructure: stand-ins for the kernel launchers of libogq_groups, so that the argument checks of groups_api.hip can be built for the
// host alone (g++, AddressSanitizer + UndefinedBehaviorSanitizer).  Every launcher records a refused launch instead of touching a device.
#include "groups_launch.h"

namespace ogq {

static void refuse() { launch_status() = hipErrorInvalidDevice; }

void launch_group_quantize(const Values&, size_t, size_t, uint32_t, const ogq_group_params_t*, const Groups&, hipStream_t) { refuse(); }
void launch_group_dequantize(const Groups&, size_t, size_t, const ogq_group_params_t*, const Result&, uint32_t, hipStream_t) { refuse(); }
void launch_activation_forward(const Values&, const Values&, size_t, size_t, uint32_t, uint32_t, const ogq_group_params_t*, const Result&, const Groups&,
                               const Groups&, hipStream_t)
{
    refuse();
}
void launch_activation_backward(const Values&, const Groups&, const Groups&, size_t, size_t, uint32_t, uint32_t, const ogq_group_params_t*, const Result&,
                                const Result&, hipStream_t)
{
    refuse();
}
size_t weight_gradient_workspace(size_t rows, size_t, size_t, uint32_t) { return rows > 1000 ? 4096 : 0; }
void launch_weight_gradient(const Values&, uint32_t, const Groups&, size_t, size_t, size_t, const ogq_group_params_t*, bool, float*, size_t, void*, hipStream_t)
{
    refuse();
}
size_t group_matvec_workspace(size_t, size_t, size_t, uint32_t) { return 0; }
void launch_group_matvec(const Groups&, size_t, size_t, const ogq_group_params_t*, const Values&, size_t, uint32_t, const Result&, void*, hipStream_t)
{
    refuse();
}

}  // namespace ogq
