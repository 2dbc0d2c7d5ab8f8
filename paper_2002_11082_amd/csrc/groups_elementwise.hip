// libogq_groups: tensors into groups and back, and activations that leave their inputs in groups.
//
// A lane holds 16 bytes of a row's values (a piece), 4 to 32 neighbouring lanes a group, whose largest magnitude goes round in two to five moves across
// lanes: one pass over the data, no LDS.  All four operators are bound by HBM.
#include <type_traits>

#include "groups_common.h"

namespace ogq {

namespace {

// How a launch cuts a tensor into pieces.  Codes lie at the piece's number times its bytes and exponents at that number / (pieces of a group) whatever the row;
// only the values' own rows take it apart.
struct Pieces {
    uint64_t total;        // rows * per_row
    uint64_t per_row;      // groups of a row, whole
    uint64_t magic;        // floor(2^64 / per_row) + 1
    uint64_t cols;
    uint32_t lanes_log2;   // log2(pieces of a group)
};

struct Place {
    uint64_t row;
    uint64_t col;
    int valid;  // values of the piece that the row has
};

// piece / per_row as the high half of a product; the quotient is at most one too large.
template <class T>
__device__ __forceinline__ Place place_of(uint64_t piece, const Pieces& s)
{
    Place p;
    p.row = __umul64hi(piece, s.magic);
    uint64_t rest = piece - p.row * s.per_row;
    if ((int64_t)rest < 0) {
        --p.row;
        rest += s.per_row;
    }
    p.col = rest * kPiece<T>;
    const int64_t left = (int64_t)(s.cols - p.col);
    p.valid = piece >= s.total || left <= 0 ? 0 : left >= kPiece<T> ? kPiece<T> : (int)left;
    return p;
}

// The codes of a piece: 8 bits 8 bytes (4 in fp32), 4 bits 4 (2).
template <class T, int BITS>
__device__ __forceinline__ void hold(const float (&v)[kPiece<T>], uint64_t piece, const Pieces& s, void* codes, uint8_t* exponents)
{
    const uint32_t byte = exponent_byte<T, BITS>(v, s.lanes_log2);
    if (piece >= s.total) return;
    if constexpr (BITS == 8) {
        if constexpr (kPiece<T> == 8) reinterpret_cast<uint2*>(codes)[piece] = make_uint2(encode8(v, byte), encode8(v + 4, byte));
        else reinterpret_cast<uint32_t*>(codes)[piece] = encode8(v, byte);
    } else {
        if constexpr (kPiece<T> == 8) reinterpret_cast<uint32_t*>(codes)[piece] = encode4(v, byte);
        else reinterpret_cast<uint16_t*>(codes)[piece] = (uint16_t)encode4(v, byte);
    }
    if ((piece & ((1u << s.lanes_log2) - 1u)) == 0u) exponents[piece >> s.lanes_log2] = (uint8_t)byte;
}

template <class T, int BITS>
__device__ __forceinline__ void held(uint64_t piece, const Pieces& s, const void* codes, const uint8_t* exponents, float (&v)[kPiece<T>])
{
    const uint32_t byte = exponents[piece >> s.lanes_log2];
    if constexpr (BITS == 8) {
        if constexpr (kPiece<T> == 8) {
            const uint2 w = reinterpret_cast<const uint2*>(codes)[piece];
            decode8(w.x, byte, v);
            decode8(w.y, byte, v + 4);
        } else {
            decode8(reinterpret_cast<const uint32_t*>(codes)[piece], byte, v);
        }
    } else {
        if constexpr (kPiece<T> == 8) decode4(reinterpret_cast<const uint32_t*>(codes)[piece], byte, v);
        else decode4(reinterpret_cast<const uint16_t*>(codes)[piece], byte, v);
    }
}

// Pieces of a thread, whose loads are under way together.  4096 x 25088 values of fp32 into 4 bits: one 87.7 us, two 79.6, four 76.1, and back 63.4, 61.4, 64.8;
// 8192 x 4096 of bf16 into 8 bits: 19.7, 20.5, 21.6; a gated activation of 8192 x 16384 in bf16: 162, 160, 184, and its backward pass 167, 175, 227.
template <class T>
constexpr int kItems = sizeof(T) == 4 ? 2 : 1;

template <class T>
__device__ __forceinline__ uint64_t piece_of(int item)
{
    return ((uint64_t)block_number() * kItems<T> + item) * kBlock + threadIdx.x;
}

// Bound by memory: 8192 x 4096 of bf16 into 8 bits 20.0 us, 5.1 TB/s read and written (a copy reaches 4.85); 4096 x 25088 of fp32 into 4 bits 78 us, 6.0 TB/s; one row of 4096
// 2.0 us, a launch.
template <class T, int BITS, bool STREAM>
__global__ __launch_bounds__(kBlock) void group_quantize_kernel(const T* x, uint64_t stride, Pieces s, void* codes, uint8_t* exponents)
{
    float v[kItems<T>][kPiece<T>];
#pragma unroll
    for (int n = 0; n < kItems<T>; ++n) {
        const Place at = place_of<T>(piece_of<T>(n), s);
        load_piece<STREAM>(x + at.row * stride + at.col, at.valid, v[n]);
    }
#pragma unroll
    for (int n = 0; n < kItems<T>; ++n) hold<T, BITS>(v[n], piece_of<T>(n), s, codes, exponents);
}

// Bound by memory: 8192 x 4096 of bf16 from 8 bits 16.3 us, 6.2 TB/s; 4096 x 25088 of fp32 from 4 bits 61.5 us, 7.6 TB/s, nearly all of it written.
template <class T, int BITS, bool STREAM>
__global__ __launch_bounds__(kBlock) void group_dequantize_kernel(const void* codes, const uint8_t* exponents, Pieces s, T* out, uint64_t stride)
{
    float v[kItems<T>][kPiece<T>];
#pragma unroll
    for (int n = 0; n < kItems<T>; ++n)
        if (piece_of<T>(n) < s.total) held<T, BITS>(piece_of<T>(n), s, codes, exponents, v[n]);
#pragma unroll
    for (int n = 0; n < kItems<T>; ++n) {
        const Place at = place_of<T>(piece_of<T>(n), s);
        store_piece<STREAM>(out + at.row * stride + at.col, at.valid, v[n]);
    }
}

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

template <uint32_t ACT, int N, class F>
__device__ __forceinline__ void each(const float (&x)[N], F f)
{
    constexpr bool kExact = N == kPiece<float>;  // (a piece of 32-bit values)
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float value, slope;
        activation<ACT, kExact>(x[i], value, slope);
        f(i, value, slope);
    }
}

// f(i, act(x[i]), act'(x[i])): the activation is the same in all lanes, a branch of the scalar unit.
template <int N, class F>
__device__ __forceinline__ void each_of(uint32_t act, const float (&x)[N], F f)
{
    if (act == OGQ_RELU) each<OGQ_RELU>(x, f);
    else if (act == OGQ_GELU) each<OGQ_GELU>(x, f);
    else if (act == OGQ_GELU_TANH) each<OGQ_GELU_TANH>(x, f);
    else each<OGQ_SILU>(x, f);
}

// Bound by memory: 8192 x 16384 of bf16, gated, silu 165 us, 6.6 TB/s; gelu, with 1.4 times the vector instructions, 169; 8192 x 8192 of fp32, gelu, 139 us, 6.7 TB/s.
template <class T, bool GATED, bool STREAM>
__global__ __launch_bounds__(kBlock) void activation_forward_kernel(const T* x, uint64_t x_stride, const T* up, uint64_t up_stride, Pieces s,
                                                                    uint32_t act, T* y, uint64_t y_stride, void* codes, uint8_t* exponents,
                                                                    void* up_codes, uint8_t* up_exponents)
{
    float v[kItems<T>][kPiece<T>], u[kItems<T>][kPiece<T>];
#pragma unroll
    for (int n = 0; n < kItems<T>; ++n) {
        const Place at = place_of<T>(piece_of<T>(n), s);
        load_piece<STREAM>(x + at.row * x_stride + at.col, at.valid, v[n]);
        if constexpr (GATED) load_piece<STREAM>(up + at.row * up_stride + at.col, at.valid, u[n]);
    }
#pragma unroll
    for (int n = 0; n < kItems<T>; ++n) {
        const uint64_t piece = piece_of<T>(n);
        float r[kPiece<T>];
        each_of(act, v[n], [&](int i, float value, float) { r[i] = GATED ? value * u[n][i] : value; });
        const Place at = place_of<T>(piece, s);
        store_piece<STREAM>(y + at.row * y_stride + at.col, at.valid, r);
        hold<T, 8>(v[n], piece, s, codes, exponents);
        if constexpr (GATED) hold<T, 8>(u[n], piece, s, up_codes, up_exponents);
    }
}

// As the forward pass: 8192 x 16384 of bf16, gated, silu 160 us, 6.8 TB/s; gelu 171; 8192 x 8192 of fp32, gelu, 138 us.
template <class T, bool GATED, bool STREAM>
__global__ __launch_bounds__(kBlock) void activation_backward_kernel(const T* dy, uint64_t dy_stride, const void* codes, const uint8_t* exponents,
                                                                     const void* up_codes, const uint8_t* up_exponents, Pieces s, uint32_t act,
                                                                     T* dx, uint64_t dx_stride, T* dup, uint64_t dup_stride)
{
    float v[kItems<T>][kPiece<T>], u[kItems<T>][kPiece<T>], d[kItems<T>][kPiece<T>];
#pragma unroll
    for (int n = 0; n < kItems<T>; ++n) {
        const uint64_t piece = piece_of<T>(n);
        const Place at = place_of<T>(piece, s);
        load_piece<STREAM>(dy + at.row * dy_stride + at.col, at.valid, d[n]);
        if (piece >= s.total) continue;
        held<T, 8>(piece, s, codes, exponents, v[n]);
        if constexpr (GATED) held<T, 8>(piece, s, up_codes, up_exponents, u[n]);
    }
#pragma unroll
    for (int n = 0; n < kItems<T>; ++n) {
        const Place at = place_of<T>(piece_of<T>(n), s);
        float r[kPiece<T>], t[kPiece<T>];
        each_of(act, v[n], [&](int i, float value, float slope) {
            r[i] = GATED ? d[n][i] * u[n][i] * slope : d[n][i] * slope;
            t[i] = d[n][i] * value;
        });
        store_piece<STREAM>(dx + at.row * dx_stride + at.col, at.valid, r);
        if constexpr (GATED) store_piece<STREAM>(dup + at.row * dup_stride + at.col, at.valid, t);
    }
}

// A tensor whose rows follow each other without a gap, in whole groups, is one long row.
Pieces pieces_of(size_t rows, size_t cols, uint32_t group_size, uint32_t dtype, bool one_row)
{
    const uint32_t piece = dtype == OGQ_FP32 ? 4 : 8;
    Pieces s;
    if (one_row) {
        cols *= rows;
        rows = 1;
    }
    s.cols = cols;
    s.per_row = (cols + group_size - 1) / group_size * (group_size / piece);
    s.total = s.per_row * rows;
    s.magic = UINT64_MAX / s.per_row + 1;
    s.lanes_log2 = (group_size == 32 ? 5u : group_size == 64 ? 6u : 7u) - (piece == 4 ? 2u : 3u);
    return s;
}

template <class T>
dim3 grid_of(const Pieces& s)
{
    constexpr uint32_t kEach = kItems<T> * kBlock;
    return grid_of_blocks((s.total + kEach - 1) / kEach);
}

// f(a value's type, whether a tensor is larger than the eight 4 MB caches of the chip together): such a one is read and written past them (4096 x 25088 of fp32
// into 4 bits 105 -> 87 us, and back 94 -> 63; the activation of 8192 x 16384 in bf16 182 -> 161, its backward pass 180 -> 168; 8192 x 4096 of bf16 20.4 -> 19.6 and 17.2 ->
// 16.4).
template <class F>
void by_type(uint32_t dtype, const Pieces& s, F f)
{
    const auto of = [&](auto* type) {
        if (s.total * 16 >= ((uint64_t)32 << 20)) f(type, std::true_type());
        else f(type, std::false_type());
    };
    if (dtype == OGQ_FP32) of((float*)nullptr);
    else if (dtype == OGQ_BF16) of((__bf16*)nullptr);
    else of((_Float16*)nullptr);
}

}  // namespace

void launch_group_quantize(const Values& x, size_t rows, size_t cols, uint32_t dtype, const ogq_group_params_t* p, const Groups& to, hipStream_t st)
{
    const Pieces s = pieces_of(rows, cols, p->group_size, dtype, x.stride == cols && cols % p->group_size == 0);
    by_type(dtype, s, [&](auto* type, auto large) {
        using T = std::remove_pointer_t<decltype(type)>;
        constexpr bool kStream = decltype(large)::value;
        launch_kernel(p->bits == 8 ? group_quantize_kernel<T, 8, kStream> : group_quantize_kernel<T, 4, kStream>, grid_of<T>(s), dim3(kBlock), st,
                      static_cast<const T*>(x.data), x.stride, s, to.codes, to.exponents);
    });
}

void launch_group_dequantize(const Groups& from, size_t rows, size_t cols, const ogq_group_params_t* p, const Result& out, uint32_t dtype, hipStream_t st)
{
    const Pieces s = pieces_of(rows, cols, p->group_size, dtype, out.stride == cols && cols % p->group_size == 0);
    by_type(dtype, s, [&](auto* type, auto large) {
        using T = std::remove_pointer_t<decltype(type)>;
        constexpr bool kStream = decltype(large)::value;
        launch_kernel(p->bits == 8 ? group_dequantize_kernel<T, 8, kStream> : group_dequantize_kernel<T, 4, kStream>, grid_of<T>(s), dim3(kBlock), st, from.codes,
                      from.exponents, s, static_cast<T*>(out.data), out.stride);
    });
}

void launch_activation_forward(const Values& x, const Values& up, size_t rows, size_t cols, uint32_t dtype, uint32_t act,
                               const ogq_group_params_t* p, const Result& y, const Groups& x_to, const Groups& up_to, hipStream_t st)
{
    const bool gated = up.data != nullptr;
    const Pieces s = pieces_of(rows, cols, p->group_size, dtype,
                               x.stride == cols && y.stride == cols && (!gated || up.stride == cols) && cols % p->group_size == 0);
    by_type(dtype, s, [&](auto* type, auto large) {
        using T = std::remove_pointer_t<decltype(type)>;
        constexpr bool kStream = decltype(large)::value;
        launch_kernel(gated ? activation_forward_kernel<T, true, kStream> : activation_forward_kernel<T, false, kStream>, grid_of<T>(s), dim3(kBlock), st,
                      static_cast<const T*>(x.data), x.stride, static_cast<const T*>(up.data), up.stride, s, act, static_cast<T*>(y.data), y.stride,
                      x_to.codes, x_to.exponents, up_to.codes, up_to.exponents);
    });
}

void launch_activation_backward(const Values& dy, const Groups& x, const Groups& up, size_t rows, size_t cols, uint32_t dtype, uint32_t act,
                                const ogq_group_params_t* p, const Result& dx, const Result& dup, hipStream_t st)
{
    const bool gated = up.codes != nullptr;
    const Pieces s = pieces_of(rows, cols, p->group_size, dtype,
                               dy.stride == cols && dx.stride == cols && (!gated || dup.stride == cols) && cols % p->group_size == 0);
    by_type(dtype, s, [&](auto* type, auto large) {
        using T = std::remove_pointer_t<decltype(type)>;
        constexpr bool kStream = decltype(large)::value;
        launch_kernel(gated ? activation_backward_kernel<T, true, kStream> : activation_backward_kernel<T, false, kStream>, grid_of<T>(s), dim3(kBlock), st,
                      static_cast<const T*>(dy.data), dy.stride, x.codes, x.exponents, up.codes, up.exponents, s, act, static_cast<T*>(dx.data),
                      dx.stride, static_cast<T*>(dup.data), dup.stride);
    });
}

}  // namespace ogq
