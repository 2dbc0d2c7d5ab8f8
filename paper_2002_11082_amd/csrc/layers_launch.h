// Internal header of libogq_layers: the host-side launchers that layers_api.hip calls.
#ifndef OGQ_LAYERS_LAUNCH_H
#define OGQ_LAYERS_LAUNCH_H

#include "groups_launch.h"
#include "ogq_layers.h"

namespace ogq {

// Arguments already checked, no output without values (but for sums over nothing).

// Integers of one of two types.
struct Integers {
    const void* data;
    uint32_t type;
};

// layers_norm.hip
void launch_layer_norm_forward(const Values& x, size_t rows, size_t cols, uint32_t dtype, const float* weight, const float* bias, float eps, const Result& y, float* mean,
                               float* rstd, hipStream_t st);
size_t layer_norm_backward_workspace(size_t rows, size_t cols, uint32_t dtype);
void launch_layer_norm_backward(const Values& dy, const Values& x, size_t rows, size_t cols, uint32_t dtype, const float* weight, const float* mean, const float* rstd,
                                const Result& dx, float* dweight, float* dbias, bool accumulate, void* workspace, hipStream_t st);
size_t linear_backward_workspace(size_t tokens, size_t outs, uint32_t dtype);
void launch_linear_backward(const Values& dy, size_t tokens, size_t outs, uint32_t dtype, uint32_t act, const Values& before, const Result& dz, float* dbias, bool accumulate,
                            void* workspace, hipStream_t st);

// layers_linear.hip
size_t linear_workspace(size_t tokens, size_t outs, size_t cols, uint32_t dtype, bool transposed);
void launch_linear(const Values& x, const Values& weight, bool transposed, size_t tokens, size_t outs, size_t cols, uint32_t dtype, const float* bias, uint32_t act,
                   const Values& residual, const Result& y, const Result& before, void* workspace, hipStream_t st);

// layers_embedding.hip
void launch_embedding_forward(const Integers& tokens, size_t number, const Values& table, size_t vocab, size_t cols, uint32_t dtype, float scale, const Result& y,
                              hipStream_t st);
size_t embedding_gradient_workspace(size_t number, size_t vocab, size_t cols);
void launch_embedding_gradient(const Integers& tokens, size_t number, const Values& dy, size_t vocab, size_t cols, uint32_t dtype, float scale, bool accumulate,
                               const Result& dtable, void* workspace, hipStream_t st);

// layers_distill.hip; without a gradient dlogits.data is null
size_t distill_workspace(size_t rows, size_t cols, uint32_t dtype, size_t top);
void launch_distill(const Values& logits, size_t rows, size_t cols, uint32_t dtype, const Integers& places, const float* values, size_t top, float temperature,
                    const float* row_weight, float* loss, const Result& dlogits, void* workspace, hipStream_t st);

}  // namespace ogq
#endif  // OGQ_LAYERS_LAUNCH_H
