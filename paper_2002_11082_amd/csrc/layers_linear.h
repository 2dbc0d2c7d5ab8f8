// Internal header of libogq_layers: what the kernels for linear layers share -- the epilogue, and how a product is cut.
#ifndef OGQ_LAYERS_LINEAR_H
#define OGQ_LAYERS_LINEAR_H

#include "layers_common.h"

namespace ogq {

// What happens to a sum on its way out.
template <class T>
struct Epilogue {
    const float* bias;
    const T* residual;
    T *y, *before;
    uint64_t residual_stride, y_stride, before_stride;
    uint32_t outs, act;

    // Sums of a token for the outputs at `out` ..., of which `valid` are there.
    __device__ __forceinline__ void operator()(uint64_t token, uint32_t out, int valid, float (&v)[kPiece<T>]) const
    {
        constexpr int N = kPiece<T>;
        if (bias != nullptr) {
            float b[N];
            load_vector<T>(bias + out, valid, 0.0f, b);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += b[i];
        }
        if (before != nullptr) store_piece<false>(before + token * before_stride + out, valid, v);
        if (act != OGQ_IDENTITY) {
            float x[N];
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = v[i];
            each_of(act, x, [&](int i, float value, float) { v[i] = value; });
        }
        if (residual != nullptr) {
            float r[N];
            load_piece<false>(residual + token * residual_stride + out, valid, r);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += r[i];
        }
        store_piece<false>(y + token * y_stride + out, valid, v);
    }
};

struct LinearShape {
    uint32_t tokens, outs, cols;
    uint64_t x_stride, weight_stride;
    uint32_t tiles_out, tiles_token;
    uint32_t part, parts;   // columns of a part of the sum, and how many there are
    uint32_t pitch;         // of the parts' sums, [parts][tokens][pitch]
    float* sums;            // null where the sum is whole
};

// layers_few.hip: products of up to kFewTokens tokens, on the vector unit.
constexpr uint32_t kFewTokens = 8;
struct FewPlan {
    uint32_t rows, split;   // weights' rows of a wavefront and wavefronts to a row; or
    uint32_t part, parts;   // transposed: rows of a part of the sum, and how many
};
FewPlan few_plan(size_t tokens, size_t outs, size_t cols, uint32_t dtype, bool transposed);
template <class T>
void launch_few(const FewPlan& plan, const T* x, const T* weight, bool transposed, const LinearShape& s, const Epilogue<T>& e, hipStream_t st);

// layers_linear.hip: the parts' sums, added in their order, through the epilogue.
template <class T>
void launch_join_parts(const LinearShape& s, const Epilogue<T>& e, hipStream_t st);

}  // namespace ogq
#endif  // OGQ_LAYERS_LINEAR_H
