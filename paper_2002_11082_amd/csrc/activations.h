// Internal header: the activations of ogq_groups.h and their derivatives in device code.
#ifndef OGQ_ACTIVATIONS_H
#define OGQ_ACTIVATIONS_H

#include "groups_common.h"

namespace ogq {

constexpr float kLog2e = 1.44269504088896f, kLog2eRest = 1.92596299112662e-8f;  // log2(e) in two pieces

// exp(a + b), |b| far below |a|, to 3 * 2^-24: a whole power of two, and the instruction's power of a fraction of at most a half, whose rounding is 2^-25 of the result.
__device__ __forceinline__ float exp_of(float a, float b)
{
    const float n = rintf(a * kLog2e);
    const float f = __builtin_fmaf(b, kLog2e, __builtin_fmaf(a, kLog2eRest, __builtin_fmaf(a, kLog2e, -n)));
    return ldexpf(__builtin_amdgcn_exp2f(f), (int)n);
}

// 1 / d for 1 <= d < 2^64, to 2^-24.
__device__ __forceinline__ float reciprocal(float d)
{
    const float r = __builtin_amdgcn_rcpf(d);
    return __builtin_fmaf(__builtin_fmaf(-d, r, 1.0f), r, r);
}

// s = 1 / (1 + exp(-x)) and 1 - s.  EXACT: to a few roundings of 32 bits, both of them, whatever x; otherwise to 2^-17 where exp(-x) is below 2^126, which is for 16-bit results.
template <bool EXACT>
__device__ __forceinline__ void sigmoid(float x, float& s, float& rest)
{
    if constexpr (EXACT) {
        const float e = exp_of(-fminf(fabsf(x), 200.0f), 0.0f), r = reciprocal(1.0f + e);
        s = x < 0.0f ? e * r : r;
        rest = x < 0.0f ? r : e * r;
    } else {
        s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -kLog2e));
        rest = 1.0f - s;
    }
}

// p = (1 + erf(x / sqrt(2))) / 2 without the difference that cancels for negative x, and g = exp(-x^2 / 2), which the slope has too.  With z = |x|, the smaller one of p and 1 - p is
// R(z) * g, where R(z) = exp(z^2 / 2) * erfc(z / sqrt(2)) / 2 falls slowly from 1/2 like 1 / z: t times a polynomial of t = 1 / (1 + c z), whose coefficients are least squares of the
// relative error up to z = 16, weighted until it was even.  16 bits: seven steps, off by 2^-22.  EXACT: six for z >= 1, off by 2^-23.3, and the exponential of x^2 with what its rounding
// leaves; for z < 1, where p and 1 - p are alike, 1/2 + x times a polynomial of x^2, found in the same way, off by 2^-31, which has fewer roundings.
template <bool EXACT>
__device__ __forceinline__ void normal_distribution(float x, float& p, float& g)
{
    if constexpr (EXACT) {
        const float z = fminf(fabsf(x), 16.0f), square = z * z;  // (exp(-128) is below the least number)
        g = exp_of(-0.5f * square, -0.5f * __builtin_fmaf(z, z, -square));
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(z, 0.4f, 1.0f));
        float r = __builtin_fmaf(0.06771772354841232f, t, -0.18541577458381653f);
        r = __builtin_fmaf(r, t, 0.10434761643409729f);
        r = __builtin_fmaf(r, t, 0.05605988949537277f);
        r = __builtin_fmaf(r, t, 0.13886022567749023f);
        r = __builtin_fmaf(r, t, 0.1591196209192276f);
        r = __builtin_fmaf(r, t, 0.15959471464157104f);
        const float smaller = r * t * g;
        float c = __builtin_fmaf(-7.66467837820528e-06f, square, 0.00011351265129633248f);
        c = __builtin_fmaf(c, square, -0.0011863530380651355f);
        c = __builtin_fmaf(c, square, 0.009973331354558468f);
        c = __builtin_fmaf(c, square, -0.06649035960435867f);
        c = __builtin_fmaf(c, square, 0.3989422917366028f);
        p = z < 1.0f ? __builtin_fmaf(x, c, 0.5f) : x < 0.0f ? smaller : 1.0f - smaller;
    } else {
        g = __builtin_amdgcn_exp2f(x * x * (-0.5f * kLog2e));
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(fabsf(x), 0.3f, 1.0f));
        float r = __builtin_fmaf(0.034704964607954025f, t, -0.15318746864795685f);
        r = __builtin_fmaf(r, t, 0.19948841631412506f);
        r = __builtin_fmaf(r, t, -0.04742685705423355f);
        r = __builtin_fmaf(r, t, 0.12529200315475464f);
        r = __builtin_fmaf(r, t, 0.10088922083377838f);
        r = __builtin_fmaf(r, t, 0.12060054391622543f);
        r = __builtin_fmaf(r, t, 0.1196390762925148f);
        const float smaller = r * t * g;
        p = x < 0.0f ? smaller : 1.0f - smaller;
    }
}

constexpr float kTanhScale = 0.797884560802865f, kCubic = 0.044715f;  // sqrt(2 / pi)

// act(x) and act'(x).
template <uint32_t ACT, bool EXACT>
__device__ __forceinline__ void activation(float x, float& value, float& slope)
{
    if constexpr (ACT == OGQ_RELU) {
        value = x < 0.0f ? 0.0f : x;  // (NaN stays)
        slope = x > 0.0f ? 1.0f : x == x ? 0.0f : x;
    } else if constexpr (ACT == OGQ_SILU) {
        float s, rest;
        sigmoid<EXACT>(x, s, rest);
        value = x * s;
        slope = s * __builtin_fmaf(x, rest, 1.0f);
    } else if constexpr (ACT == OGQ_GELU) {
        float p, g;
        normal_distribution<EXACT>(x, p, g);
        value = x * p;
        slope = __builtin_fmaf(x, 0.398942280401433f * g, p);
    } else {
        // (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u)).  The square is limited: behind 100 the slope's second term is 0, where an infinite square
        // would make it NaN.
        const float square = fminf(x * x, 10000.0f);
        float s, rest;
        sigmoid<EXACT>(2.0f * kTanhScale * x * __builtin_fmaf(kCubic, square, 1.0f), s, rest);
        value = x * s;
        slope = __builtin_fmaf(x * s * rest, 2.0f * kTanhScale * __builtin_fmaf(3.0f * kCubic, square, 1.0f), s);
    }
}

template <uint32_t ACT, bool EXACT, int N, class F>
__device__ __forceinline__ void each(const float (&x)[N], F f)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float value, slope;
        activation<ACT, EXACT>(x[i], value, slope);
        f(i, value, slope);
    }
}

// f(i, act(x[i]), act'(x[i])): the activation is the same in all lanes, a branch of the scalar unit.
template <bool EXACT, int N, class F>
__device__ __forceinline__ void each_as(uint32_t act, const float (&x)[N], F f)
{
    if (act == OGQ_RELU) each<OGQ_RELU, EXACT>(x, f);
    else if (act == OGQ_GELU) each<OGQ_GELU, EXACT>(x, f);
    else if (act == OGQ_GELU_TANH) each<OGQ_GELU_TANH, EXACT>(x, f);
    else each<OGQ_SILU, EXACT>(x, f);
}

// As exact as the results need it: a piece of four values is one of 32 bits.
template <int N, class F>
__device__ __forceinline__ void each_of(uint32_t act, const float (&x)[N], F f)
{
    each_as<N == kPiece<float>>(act, x, f);
}

}  // namespace ogq
#endif  // OGQ_ACTIVATIONS_H
