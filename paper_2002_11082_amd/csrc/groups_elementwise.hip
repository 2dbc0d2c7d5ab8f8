// libogq_groups: tensors into groups and back, and activations that leave their inputs in groups.
//
// Every lane holds eight consecutive values of a row (an octet), 4, 8 or 16 neighbouring lanes a group, whose largest magnitude goes round
// in two to four DPP moves: one pass over the data, no LDS.  All four operators are bound by HBM.
#include "groups_common.h"

namespace ogq {

namespace {

// How a launch cuts a tensor into octets.  Codes lie at octet * 8 (* 4) and exponents at octet / (group_size / 8) whatever the
// row; only the values' own rows take the octet apart.
struct Octets {
    uint64_t total;        // rows * per_row
    uint64_t per_row;      // groups of a row, whole
    uint64_t magic;        // floor(2^64 / per_row) + 1
    uint64_t cols;
    uint32_t lanes_log2;   // log2(group_size / 8)
};

struct Place {
    uint64_t row;
    uint64_t col;
    int valid;  // values of the octet that the row has
};

// octet / per_row as the high half of a product; the quotient is at most one too large.
__device__ __forceinline__ Place place_of(uint64_t octet, const Octets& s)
{
    Place p;
    p.row = __umul64hi(octet, s.magic);
    uint64_t rest = octet - p.row * s.per_row;
    if ((int64_t)rest < 0) {
        --p.row;
        rest += s.per_row;
    }
    p.col = rest * 8;
    const int64_t left = (int64_t)(s.cols - p.col);
    p.valid = octet >= s.total || left <= 0 ? 0 : left >= 8 ? 8 : (int)left;
    return p;
}

template <class T, int BITS>
__device__ __forceinline__ void hold(const float (&v)[8], uint64_t octet, const Octets& s, void* codes, uint8_t* exponents)
{
    const uint32_t byte = exponent_byte<T, BITS>(v, s.lanes_log2);
    if (octet >= s.total) return;
    if constexpr (BITS == 8) reinterpret_cast<uint2*>(codes)[octet] = encode8(v, byte);
    else reinterpret_cast<uint32_t*>(codes)[octet] = encode4(v, byte);
    if ((octet & ((1u << s.lanes_log2) - 1u)) == 0u) exponents[octet >> s.lanes_log2] = (uint8_t)byte;
}

template <int BITS>
__device__ __forceinline__ void held(uint64_t octet, const Octets& s, const void* codes, const uint8_t* exponents, float (&v)[8])
{
    const uint32_t byte = exponents[octet >> s.lanes_log2];
    if constexpr (BITS == 8) decode8(reinterpret_cast<const uint2*>(codes)[octet], byte, v);
    else decode4(reinterpret_cast<const uint32_t*>(codes)[octet], byte, v);
}

template <class T, int BITS>
__global__ __launch_bounds__(kBlock) void group_quantize_kernel(const T* x, uint64_t stride, Octets s, void* codes, uint8_t* exponents)
{
    const uint64_t octet = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
    const Place at = place_of(octet, s);
    float v[8];
    load8(x + at.row * stride + at.col, at.valid, v);
    hold<T, BITS>(v, octet, s, codes, exponents);
}

template <class T, int BITS>
__global__ __launch_bounds__(kBlock) void group_dequantize_kernel(const void* codes, const uint8_t* exponents, Octets s, T* out, uint64_t stride)
{
    const uint64_t octet = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
    const Place at = place_of(octet, s);
    if (at.valid == 0) return;
    float v[8];
    held<BITS>(octet, s, codes, exponents, v);
    store8(out + at.row * stride + at.col, at.valid, v);
}

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896f); }
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + exp_of(-x)); }

constexpr float kTanhScale = 0.797884560802865f, kCubic = 0.044715f;  // sqrt(2 / pi)

// act(x) and act'(x).
template <uint32_t ACT>
__device__ __forceinline__ void activation(float x, float& value, float& slope)
{
    if constexpr (ACT == OGQ_RELU) {
        value = x < 0.0f ? 0.0f : x;  // (NaN stays)
        slope = x > 0.0f ? 1.0f : x == x ? 0.0f : x;
    } else if constexpr (ACT == OGQ_SILU) {
        const float s = sigmoid(x);
        value = x * s;
        slope = s * (1.0f + x * (1.0f - s));
    } else if constexpr (ACT == OGQ_GELU) {
        const float p = 0.5f * (1.0f + erff(x * 0.707106781186548f));
        value = x * p;
        slope = p + x * (0.398942280401433f * exp_of(-0.5f * x * x));
    } else {
        // (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u)).  The square is limited: behind 10 the slope's second term is 0, where an infinite square
        // would make it NaN.
        const float square = fminf(x * x, 100.0f);
        const float s = sigmoid(2.0f * kTanhScale * x * (1.0f + kCubic * square));
        value = x * s;
        slope = s + x * s * (1.0f - s) * 2.0f * kTanhScale * (1.0f + 3.0f * kCubic * square);
    }
}

template <uint32_t ACT, class F>
__device__ __forceinline__ void each(const float (&x)[8], F f)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float value, slope;
        activation<ACT>(x[i], value, slope);
        f(i, value, slope);
    }
}

// f(i, act(x[i]), act'(x[i])): the activation is the same in all lanes, a branch of the scalar unit.
template <class F>
__device__ __forceinline__ void each_of(uint32_t act, const float (&x)[8], F f)
{
    if (act == OGQ_RELU) each<OGQ_RELU>(x, f);
    else if (act == OGQ_GELU) each<OGQ_GELU>(x, f);
    else if (act == OGQ_GELU_TANH) each<OGQ_GELU_TANH>(x, f);
    else each<OGQ_SILU>(x, f);
}

template <class T, bool GATED>
__global__ __launch_bounds__(kBlock) void activation_forward_kernel(const T* x, uint64_t x_stride, const T* up, uint64_t up_stride, Octets s,
                                                                    uint32_t act, T* y, uint64_t y_stride, void* codes, uint8_t* exponents,
                                                                    void* up_codes, uint8_t* up_exponents)
{
    const uint64_t octet = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
    const Place at = place_of(octet, s);
    float v[8], u[8], r[8];
    load8(x + at.row * x_stride + at.col, at.valid, v);
    if constexpr (GATED) load8(up + at.row * up_stride + at.col, at.valid, u);
    each_of(act, v, [&](int i, float value, float) { r[i] = GATED ? value * u[i] : value; });
    store8(y + at.row * y_stride + at.col, at.valid, r);
    hold<T, 8>(v, octet, s, codes, exponents);
    if constexpr (GATED) hold<T, 8>(u, octet, s, up_codes, up_exponents);
}

template <class T, bool GATED>
__global__ __launch_bounds__(kBlock) void activation_backward_kernel(const T* dy, uint64_t dy_stride, const void* codes, const uint8_t* exponents,
                                                                     const void* up_codes, const uint8_t* up_exponents, Octets s, uint32_t act,
                                                                     T* dx, uint64_t dx_stride, T* dup, uint64_t dup_stride)
{
    const uint64_t octet = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
    const Place at = place_of(octet, s);
    if (at.valid == 0) return;
    float v[8], u[8], d[8], r[8], t[8];
    load8(dy + at.row * dy_stride + at.col, at.valid, d);
    held<8>(octet, s, codes, exponents, v);
    if constexpr (GATED) held<8>(octet, s, up_codes, up_exponents, u);
    each_of(act, v, [&](int i, float value, float slope) {
        r[i] = GATED ? d[i] * u[i] * slope : d[i] * slope;
        t[i] = d[i] * value;
    });
    store8(dx + at.row * dx_stride + at.col, at.valid, r);
    if constexpr (GATED) store8(dup + at.row * dup_stride + at.col, at.valid, t);
}

// A tensor whose rows follow each other without a gap, in whole groups, is one long row.
Octets octets_of(size_t rows, size_t cols, uint32_t group_size, bool one_row)
{
    Octets s;
    if (one_row) {
        cols *= rows;
        rows = 1;
    }
    s.cols = cols;
    s.per_row = (cols + group_size - 1) / group_size * (group_size / 8);
    s.total = s.per_row * rows;
    s.magic = UINT64_MAX / s.per_row + 1;
    s.lanes_log2 = group_size == 32 ? 2u : group_size == 64 ? 3u : 4u;
    return s;
}

dim3 grid_of(const Octets& s) { return dim3((uint32_t)((s.total + kBlock - 1) / kBlock)); }

template <class F>
void by_type(uint32_t dtype, F f)
{
    if (dtype == OGQ_FP32) f((float*)nullptr);
    else if (dtype == OGQ_BF16) f((__bf16*)nullptr);
    else f((_Float16*)nullptr);
}

}  // namespace

void launch_group_quantize(const Values& x, size_t rows, size_t cols, uint32_t dtype, const ogq_group_params_t* p, const Groups& to, hipStream_t st)
{
    const Octets s = octets_of(rows, cols, p->group_size, x.stride == cols && cols % p->group_size == 0);
    by_type(dtype, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        launch_kernel(p->bits == 8 ? group_quantize_kernel<T, 8> : group_quantize_kernel<T, 4>, grid_of(s), dim3(kBlock), st,
                      static_cast<const T*>(x.data), x.stride, s, to.codes, to.exponents);
    });
}

void launch_group_dequantize(const Groups& from, size_t rows, size_t cols, const ogq_group_params_t* p, const Result& out, uint32_t dtype, hipStream_t st)
{
    const Octets s = octets_of(rows, cols, p->group_size, out.stride == cols && cols % p->group_size == 0);
    by_type(dtype, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        launch_kernel(p->bits == 8 ? group_dequantize_kernel<T, 8> : group_dequantize_kernel<T, 4>, grid_of(s), dim3(kBlock), st, from.codes,
                      from.exponents, s, static_cast<T*>(out.data), out.stride);
    });
}

void launch_activation_forward(const Values& x, const Values& up, size_t rows, size_t cols, uint32_t dtype, uint32_t act,
                               const ogq_group_params_t* p, const Result& y, const Groups& x_to, const Groups& up_to, hipStream_t st)
{
    const bool gated = up.data != nullptr;
    const Octets s = octets_of(rows, cols, p->group_size,
                               x.stride == cols && y.stride == cols && (!gated || up.stride == cols) && cols % p->group_size == 0);
    by_type(dtype, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        launch_kernel(gated ? activation_forward_kernel<T, true> : activation_forward_kernel<T, false>, grid_of(s), dim3(kBlock), st,
                      static_cast<const T*>(x.data), x.stride, static_cast<const T*>(up.data), up.stride, s, act, static_cast<T*>(y.data), y.stride,
                      x_to.codes, x_to.exponents, up_to.codes, up_to.exponents);
    });
}

void launch_activation_backward(const Values& dy, const Groups& x, const Groups& up, size_t rows, size_t cols, uint32_t dtype, uint32_t act,
                                const ogq_group_params_t* p, const Result& dx, const Result& dup, hipStream_t st)
{
    const bool gated = up.codes != nullptr;
    const Octets s = octets_of(rows, cols, p->group_size,
                               dy.stride == cols && dx.stride == cols && (!gated || dup.stride == cols) && cols % p->group_size == 0);
    by_type(dtype, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        launch_kernel(gated ? activation_backward_kernel<T, true> : activation_backward_kernel<T, false>, grid_of(s), dim3(kBlock), st,
                      static_cast<const T*>(dy.data), dy.stride, x.codes, x.exponents, up.codes, up.exponents, s, act, static_cast<T*>(dx.data),
                      dx.stride, static_cast<T*>(dup.data), dup.stride);
    });
}

}  // namespace ogq
