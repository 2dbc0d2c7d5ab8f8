// libogq_groups: tensors into groups and back, and activations that leave their inputs in groups.
//
// A lane holds 16 bytes of a row's values (a piece), 4 to 32 neighbouring lanes a group, whose largest magnitude goes round in two to five moves across
// lanes: one pass over the data, no LDS.  All four operators are bound by HBM.
#include <type_traits>

#include "activations.h"

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
