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

    // The same for ROWS tokens, `apart` from one to the next, below `tokens`, of 16-bit types: what is loaded is under way together.  The bias comes from the caller.
    template <int ROWS>
    __device__ __forceinline__ void rows(uint32_t first, uint32_t apart, uint32_t tokens, uint32_t out, int valid, const float (&b)[8], float (&v)[ROWS][8]) const
    {
        static_assert(kPiece<T> == 8);
        uint4 r[ROWS];
        if (residual != nullptr) {
#pragma unroll
            for (int n = 0; n < ROWS; ++n) r[n] = load_raw(residual + min(first + n * apart, tokens - 1) * residual_stride + out, valid);
        }
#pragma unroll
        for (int n = 0; n < ROWS; ++n)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[n][i] += b[i];
        if (before != nullptr) {
#pragma unroll
            for (int n = 0; n < ROWS; ++n)
                if (first + n * apart < tokens) store_piece<false>(before + (first + n * apart) * before_stride + out, valid, v[n]);
        }
        if (act != OGQ_IDENTITY) {
            float a[ROWS * 8];
#pragma unroll
            for (int i = 0; i < ROWS * 8; ++i) a[i] = v[i / 8][i % 8];
            each_of(act, a, [&](int i, float value, float) { v[i / 8][i % 8] = value; });
        }
        if (residual != nullptr) {
#pragma unroll
            for (int n = 0; n < ROWS; ++n) {
                float add[8];
                values_of<T>(r[n], add);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[n][i] += add[i];
            }
        }
#pragma unroll
        for (int n = 0; n < ROWS; ++n)
            if (first + n * apart < tokens) store_piece<false>(y + (first + n * apart) * y_stride + out, valid, v[n]);
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

// layers_few.hip: products of few tokens on the vector unit, which reads the weights at memory's rate and loses to the matrix cores with every token that it multiplies them with.
// On the vector unit and in tiles, bf16: 16384 x 4096 2 tokens 19.9 us and 23.8, 4 22.0 and 23.9, 6 26.2 and 24.0; 4096 x 4096 2 4.6 and 10.5, 8 11.0 and 11.1; 50000 x 1024 1 15.5 and 18.9, 2 21.6 and
// 18.8; transposed (16384 x 4096) 1 34.0 and 24.3, 8 40.5 and 24.9.  fp32: 16384 x 4096 1 38.6 and 57.9, 8 49.7 and 59.6; 4096 x 4096 8 15.5 and 22.0; transposed 16384 x 4096 1 41.3 and
// 61.6, 8 50.6 and 63.1.
// Transposed in fp32 alone.
inline bool few_tokens(size_t tokens, size_t outs, size_t cols, uint32_t dtype, bool transposed)
{
    if (tokens > 8 || dtype == OGQ_FP32) return tokens <= 8;
    if (transposed) return false;
    return tokens == 1 || outs * cols <= (size_t)1 << 24 || (tokens <= 4 && cols >= 2048);
}
template <class T>
void launch_few(const T* x, const T* weight, const LinearShape& s, const Epilogue<T>& e, hipStream_t st);
// Transposed: rows of weights in a part of the sum, and how many parts.
struct FewParts {
    uint32_t part, parts;
};
FewParts few_parts(size_t outs, size_t cols);
void launch_few_across(const float* x, const float* weight, LinearShape s, const Epilogue<float>& e, float* workspace, hipStream_t st);

// layers_linear.hip: the parts' sums, added in their order, through the epilogue.
template <class T>
void launch_join_parts(const LinearShape& s, const Epilogue<T>& e, hipStream_t st);

}  // namespace ogq
#endif  // OGQ_LAYERS_LINEAR_H
