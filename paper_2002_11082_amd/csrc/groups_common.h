// Internal header of libogq_groups: the format of ogq_groups.h in device code.
#ifndef OGQ_GROUPS_COMMON_H
#define OGQ_GROUPS_COMMON_H

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>
#include <string.h>

#include "device_common.h"
#include "groups_launch.h"

namespace ogq {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// HIP takes less than 2^32 threads along a dimension of a grid: more than 2^22 workgroups go to rows of 2^22.  The last row is as long as the others: its workgroups behind the last
// one have nothing to do.
constexpr uint32_t kGridRowLog2 = 22;

inline dim3 grid_of_blocks(uint64_t blocks)
{
    constexpr uint64_t kRow = (uint64_t)1 << kGridRowLog2;
    return blocks <= kRow ? dim3((uint32_t)blocks) : dim3((uint32_t)kRow, (uint32_t)((blocks + kRow - 1) >> kGridRowLog2));
}

__device__ __forceinline__ uint32_t block_number() { return blockIdx.y << kGridRowLog2 | blockIdx.x; }

// The limits of a group's exponent: every q * 2^e is a value of T.
template <class T, int BITS>
struct ExponentLimits {
    static constexpr bool kHalf = sizeof(T) == 2 && !__is_same(T, __bf16);
    static constexpr int kLow = BITS == 8 ? (kHalf ? -24 : -126) : (kHalf ? -23 : -125);
    static constexpr int kHigh = BITS == 8 ? (kHalf ? 9 : 121) : (kHalf ? 13 : 125);
};

// N consecutive values as they are in memory, N * sizeof(T) / 4 words, of which only the first `valid` are there: the others are 0.  Every load is one of a value that
// is there, so that none waits for another's turn.
template <class T, int N>
__device__ __forceinline__ void load_some(const T* from, int valid, uint32_t (&to)[N * sizeof(T) / 4])
{
#pragma unroll
    for (int i = 0; i < (int)(N * sizeof(T) / 4); ++i) to[i] = 0;
    if (valid <= 0) return;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) memcpy(&to[i], from + min(i, valid - 1), 4);
#pragma unroll
        for (int i = 0; i < N; ++i) to[i] = i < valid ? to[i] : 0u;
    } else {
        uint16_t v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) memcpy(&v[i], from + min(i, valid - 1), 2);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) to[i] = (2 * i < valid ? v[2 * i] : 0u) | (2 * i + 1 < valid ? (uint32_t)v[2 * i + 1] << 16 : 0u);
    }
}

// A lane's piece of a row: 16 bytes of values, so that a wavefront reads and writes 1 KB without a gap.
template <class T>
constexpr int kPiece = 16 / sizeof(T);

typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(2)));

// The values of a piece in 32 bits; only the first `valid` are read, the others are 0.  No alignment but the type's: the hardware takes wide loads
// from any address.  STREAM: the cache need not keep them.
template <bool STREAM, class T>
__device__ __forceinline__ void load_piece(const T* from, int valid, float (&v)[kPiece<T>])
{
    T raw[kPiece<T>];
    if (valid >= kPiece<T>) {
        const Words* words = reinterpret_cast<const Words*>(from);
        const uint4 w = __builtin_bit_cast(uint4, STREAM ? __builtin_nontemporal_load(words) : *words);
        memcpy(raw, &w, 16);
    } else {
        uint32_t words[4];
        load_some<T, kPiece<T>>(from, valid, words);
        memcpy(raw, words, 16);
    }
#pragma unroll
    for (int i = 0; i < kPiece<T>; ++i) v[i] = (float)raw[i];
}

template <bool STREAM, class T>
__device__ __forceinline__ void store_piece(T* to, int valid, const float (&v)[kPiece<T>])
{
    T raw[kPiece<T>];
#pragma unroll
    for (int i = 0; i < kPiece<T>; ++i) raw[i] = (T)v[i];
    if (valid >= kPiece<T>) {
        Words w;
        memcpy(&w, raw, 16);
        if (STREAM) __builtin_nontemporal_store(w, reinterpret_cast<Words*>(to));
        else *reinterpret_cast<Words*>(to) = w;
    } else {
#pragma unroll
        for (int i = 0; i < kPiece<T>; ++i)
            if (i < valid) to[i] = raw[i];
    }
}

// The exponent byte of the group whose values are held by 1 << lanes_log2 (2 to 5) neighbouring lanes, N to each; all lanes of the wavefront are active.
// The largest magnitude as an integer: infinities and NaN are the largest of all.
template <class T, int BITS, int N>
__device__ __forceinline__ uint32_t exponent_byte(const float (&v)[N], uint32_t lanes_log2)
{
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) most = max(most, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    most = max(most, dpp_u32<kDppXor1>(most));
    most = max(most, dpp_u32<kDppXor2>(most));
    if (lanes_log2 > 2) most = max(most, dpp_u32<kDppHalfMirror>(most));
    if (lanes_log2 > 3) most = max(most, dpp_u32<kDppMirror>(most));
    if (lanes_log2 > 4) {
        const auto r = __builtin_amdgcn_permlane16_swap(most, most, false, false);
        most = max((uint32_t)r[0], (uint32_t)r[1]);
    }
    // 127 = 1.984375 * 2^6, 6 = 1.5 * 2^2
    int byte = (int)(most >> 23) - (BITS == 8 ? 6 : 2) + ((most & 0x7FFFFFu) > (BITS == 8 ? 0x7E0000u : 0x400000u) ? 1 : 0);
    byte = min(max(byte, ExponentLimits<T, BITS>::kLow + 127), ExponentLimits<T, BITS>::kHigh + 127);
    return most >= 0x7F800000u ? 255u : (uint32_t)byte;
}

// 2^-e for an exponent byte (1 <= byte <= 252).
__device__ __forceinline__ float inverse_power(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// 2^e for an exponent byte; infinite for 255, and a code of 0 times that is NaN.
__device__ __forceinline__ float power(uint32_t byte) { return __uint_as_float(byte << 23); }

// Four values as 8-bit codes.  x * 2^-e + 1.5 * 2^23 has the rounded number in its low bits, ties to even.
__device__ __forceinline__ uint32_t encode8(const float* v, uint32_t byte)
{
    constexpr float kShift = 12582912.0f;
    const float inverse = inverse_power(byte);
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        r[i] = __float_as_uint(__builtin_amdgcn_fmed3f(__builtin_fmaf(v[i], inverse, kShift), kShift - 127.0f, kShift + 127.0f));
    const uint32_t w = __builtin_amdgcn_perm(__builtin_amdgcn_perm(r[3], r[2], 0x0C0C0400u), __builtin_amdgcn_perm(r[1], r[0], 0x0C0C0400u), 0x05040100u);
    return byte != 255u ? w : 0u;
}

// Four or eight values as 4-bit codes: the conversion of the hardware rounds to the nearest of the eight numbers, ties to even, and takes
// larger ones to 6.
template <int N>
__device__ __forceinline__ uint32_t encode4(const float (&v)[N], uint32_t byte)
{
    const float unit = power(byte);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], unit, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], unit, 1);
    if constexpr (N == 8) {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], unit, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], unit, 3);
    }
    return byte != 255u ? w : 0u;
}

// What four 8-bit codes stand for.
__device__ __forceinline__ void decode8(uint32_t w, uint32_t byte, float* v)
{
    const float unit = power(byte);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)(int8_t)(w >> (8 * i)) * unit;  // (a signed byte becomes a float in one instruction)
}

__device__ __forceinline__ float2 decode4_pair(bf16x2 p)
{
    uint32_t u;
    memcpy(&u, &p, 4);
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
}

// What four or eight 4-bit codes stand for.
template <int N>
__device__ __forceinline__ void decode4(uint32_t w, uint32_t byte, float (&v)[N])
{
    const float unit = power(byte);
    const float2 a = decode4_pair(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 0)), b = decode4_pair(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 1));
    v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
    if constexpr (N == 8) {
        const float2 c = decode4_pair(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 2)), d = decode4_pair(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 3));
        v[4] = c.x, v[5] = c.y, v[6] = d.x, v[7] = d.y;
    }
}

// The three pieces of a value in bf16, 8 bits of its fraction each; their sum is the value.  An infinity is its first piece alone.
__device__ __forceinline__ void split3(float x, uint32_t& high, uint32_t& middle, uint32_t& low)
{
    const uint32_t u = __float_as_uint(x);
    high = u & 0xFFFF0000u;
    float rest = x - __uint_as_float(high);
    rest = (u & 0x7FFFFFFFu) == 0x7F800000u ? 0.0f : rest;
    middle = __float_as_uint(rest) & 0xFFFF0000u;
    low = __float_as_uint(rest - __uint_as_float(middle));
}

}  // namespace ogq
#endif  // OGQ_GROUPS_COMMON_H
