// Test infrastructure: stand-ins for the kernel launchers of libogq_layers, so that the argument checks of layers_api.hip can be built for the
// host alone (g++, AddressSanitizer + UndefinedBehaviorSanitizer).  Every launcher records a refused launch instead of touching a device.
#include "layers_launch.h"

namespace ogq {

static void refuse() { launch_status() = hipErrorInvalidDevice; }

void launch_layer_norm_forward(const Values&, size_t, size_t, uint32_t, const float*, const float*, float, const Result&, float*, float*, hipStream_t) { refuse(); }
size_t layer_norm_backward_workspace(size_t rows, size_t, uint32_t) { return rows > 1000 ? 4096 : 0; }
void launch_layer_norm_backward(const Values&, const Values&, size_t, size_t, uint32_t, const float*, const float*, const float*, const Result&, float*, float*, bool, void*,
                                hipStream_t)
{
    refuse();
}
size_t linear_backward_workspace(size_t tokens, size_t, uint32_t) { return tokens > 100 ? 4096 : 0; }
void launch_linear_backward(const Values&, size_t, size_t, uint32_t, uint32_t, const Values&, const Result&, float*, bool, void*, hipStream_t) { refuse(); }
size_t linear_workspace(size_t, size_t, size_t cols, uint32_t, bool) { return cols > 1000 ? 4096 : 0; }
void launch_linear(const Values&, const Values&, bool, size_t, size_t, size_t, uint32_t, const float*, uint32_t, const Values&, const Result&, const Result&, void*, hipStream_t)
{
    refuse();
}
void launch_embedding_forward(const Integers&, size_t, const Values&, size_t, size_t, uint32_t, float, const Result&, hipStream_t) { refuse(); }
size_t embedding_gradient_workspace(size_t number, size_t, size_t) { return number * 16; }
void launch_embedding_gradient(const Integers&, size_t, const Values&, size_t, size_t, uint32_t, float, bool, const Result&, void*, hipStream_t) { refuse(); }
size_t distill_workspace(size_t, size_t cols, uint32_t, size_t) { return cols > 10000 ? 4096 : 0; }
void launch_distill(const Values&, size_t, size_t, uint32_t, const Integers&, const float*, size_t, float, const float*, float*, const Result&, void*, hipStream_t) { refuse(); }

}  // namespace ogq
