// Internal header of libogq_layers: what its kernel sources share.
#ifndef OGQ_LAYERS_COMMON_H
#define OGQ_LAYERS_COMMON_H

#include <type_traits>

#include "activations.h"
#include "layers_launch.h"

namespace ogq {

// HIP takes less than 2^32 threads along a dimension of a grid: more than 2^20 workgroups, of up to 1024 threads, go to rows of 2^20.  The last row is as long as the others: its workgroups
// behind the last one have nothing to do.
constexpr uint32_t kRowOfBlocksLog2 = 20;

inline dim3 grid_of(uint64_t blocks)
{
    constexpr uint64_t kRow = (uint64_t)1 << kRowOfBlocksLog2;
    return blocks <= kRow ? dim3((uint32_t)blocks) : dim3((uint32_t)kRow, (uint32_t)((blocks + kRow - 1) >> kRowOfBlocksLog2));
}

__device__ __forceinline__ uint32_t this_block() { return blockIdx.y << kRowOfBlocksLog2 | blockIdx.x; }

inline uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

// Two sums over a workgroup of WAVES wavefronts, in all of its threads: across lanes, then the wavefronts' in their order.  `space` is used by the next call but one.
template <int WAVES>
struct BlockSums {
    float2 (*space)[WAVES];
    uint32_t turn = 0;
    __device__ __forceinline__ float2 operator()(float a, float b)
    {
        a = wave_sum_f32(a), b = wave_sum_f32(b);
        if constexpr (WAVES == 1) return make_float2(a, b);
        float2* const s = space[turn];
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = make_float2(a, b);
        __syncthreads();
        float2 t = s[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) t.x += s[w].x, t.y += s[w].y;
        return t;
    }
    // The larger of each instead of the sum; a NaN does not count.
    __device__ __forceinline__ float2 largest(float a, float b)
    {
        a = wave_max(a), b = wave_max(b);
        if constexpr (WAVES == 1) return make_float2(a, b);
        float2* const s = space[turn];
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = make_float2(a, b);
        __syncthreads();
        float2 t = s[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) t.x = fmaxf(t.x, s[w].x), t.y = fmaxf(t.y, s[w].y);
        return t;
    }
};

// A piece as it is in memory (what a row does not have as 0), and its values.
template <class T>
__device__ __forceinline__ uint4 load_raw(const T* from, int valid)
{
    uint32_t w[4];
    if (valid >= kPiece<T>) return __builtin_bit_cast(uint4, *reinterpret_cast<const Words*>(from));
    load_some<T, kPiece<T>>(from, valid, w);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Where a piece of a row of at least kPiece values lies: the last piece ends with the row, and what it has of the piece before it (`again` values) is computed twice and stored twice, the
// same both times, but counts once in a sum.  So every piece is one load and one store.  A piece behind the row is its last one, of which nothing counts.
template <class T>
struct PieceAt {
    uint32_t col;
    int again;
    bool there;
    __device__ __forceinline__ PieceAt(uint32_t wanted, uint32_t cols)
    {
        there = wanted < cols;
        col = min(wanted, cols - kPiece<T>);
        again = (int)(wanted - col);
    }
    __device__ __forceinline__ explicit PieceAt(uint32_t whole) : col(whole), again(0), there(true) {}
    __device__ __forceinline__ bool counts(int i) const { return i >= again; }
};

// Piece p of P of a thread, of a row that THREADS threads hold and for which half as many pieces would not do: the first half of them is whole.
template <class T, int THREADS, int P>
__device__ __forceinline__ PieceAt<T> piece_at(int p, uint32_t thread, uint32_t cols)
{
    const uint32_t col = (p * THREADS + thread) * kPiece<T>;
    return p < P / 2 ? PieceAt<T>(col) : PieceAt<T>(col, cols);
}

template <class T>
__device__ __forceinline__ uint4 load_whole(const T* from)
{
    return __builtin_bit_cast(uint4, *reinterpret_cast<const Words*>(from));
}

template <class T>
__device__ __forceinline__ void values_of(const uint4& w, float (&v)[kPiece<T>])
{
    T raw[kPiece<T>];
    memcpy(raw, &w, 16);
#pragma unroll
    for (int i = 0; i < kPiece<T>; ++i) v[i] = (float)raw[i];
}

// How many values of a piece at `col` a row of `cols` has: none to all.
template <class T>
__device__ __forceinline__ int valid_of(uint32_t col, uint32_t cols)
{
    return col >= cols ? 0 : (int)min((uint32_t)kPiece<T>, cols - col);
}

// A piece of an fp32 vector that has as many values as a piece of T: bias, weight.  `other` where it is not there.
template <class T>
__device__ __forceinline__ void load_vector(const float* from, int valid, float other, float (&v)[kPiece<T>])
{
    if (from != nullptr && valid >= kPiece<T>) {
        memcpy(v, from, sizeof v);
        return;
    }
#pragma unroll
    for (int i = 0; i < kPiece<T>; ++i) v[i] = from != nullptr && i < valid ? from[i] : other;
}

template <class T>
__device__ __forceinline__ void load_vector(const float* from, uint32_t col, float other, float (&v)[kPiece<T>])
{
    if (from != nullptr) {
        memcpy(v, from + col, sizeof v);
        return;
    }
#pragma unroll
    for (int i = 0; i < kPiece<T>; ++i) v[i] = other;
}

// f(a null pointer of the values' type).
template <class F>
inline void with_type(uint32_t dtype, F f)
{
    if (dtype == OGQ_FP32) f((float*)nullptr);
    else if (dtype == OGQ_BF16) f((__bf16*)nullptr);
    else f((_Float16*)nullptr);
}

// layers_norm.hip: the rows of `parts` vectors [2][pitch] each, added column by column in an order that their number alone decides, to one or two vectors of `cols` values.
void launch_add_vectors(const float* parts, uint32_t number, size_t cols, size_t pitch, float* first, float* second, bool accumulate, hipStream_t st);

}  // namespace ogq
#endif  // OGQ_LAYERS_COMMON_H
