// libogq_groups: the gradient of a linear layer's weights from the gradient of its outputs and its 8-bit inputs,
//   dw[o][i] = sum over t of dy[t][o] * x^[t][i].
//
// A workgroup holds a tile of 128 x 128 sums in registers and goes along t in steps of 32 rows.  In memory both factors have the summed index
// outside; the matrix instruction wants eight of it per lane.  The rows go to LDS as they are and come back transposed (ds_read_b64_tr_b16: 16
// lanes read four rows of 16 values and receive four values of one column each).  The codes become 16-bit values on the way to LDS, exactly.
#include "groups_common.h"

namespace ogq {

namespace {

constexpr int kTile = 128;   // inputs and outputs of a workgroup's sums
constexpr int kDepth = 32;   // rows of a step
constexpr int kRowBytes = kTile * 2;

typedef short s16x8 __attribute__((ext_vector_type(8)));

// A row of a tile in LDS is eight chunks of 32 bytes (16 values); chunk c of row k lies at c ^ twist(k): the eight rows that half a wavefront reads
// at once lie in different banks.
__device__ __forceinline__ uint32_t twist(uint32_t k) { return (k & 3u) | ((k >> 1) & 4u); }

// Sixteen values of a row of dy in the pieces that the matrix cores take: one for 16-bit types, three for fp32.
template <class T>
struct Rows16 {
    static constexpr int kPieces = 1;
    uint4 raw[2];
    __device__ __forceinline__ void load(const T* from, int valid)
    {
        if (valid >= 16) {
            memcpy(raw, from, 32);
        } else {
            uint16_t v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                v[i] = 0;
                if (i < valid) memcpy(&v[i], from + i, 2);
            }
            memcpy(raw, v, 32);
        }
    }
    __device__ __forceinline__ void store(char* to, int) const
    {
        reinterpret_cast<uint4*>(to)[0] = raw[0];
        reinterpret_cast<uint4*>(to)[1] = raw[1];
    }
};
template <>
struct Rows16<float> {
    static constexpr int kPieces = 3;
    float raw[16];
    __device__ __forceinline__ void load(const float* from, int valid)
    {
        if (valid >= 16) {
            memcpy(raw, from, 64);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) raw[i] = i < valid ? from[i] : 0.0f;
        }
    }
    __device__ __forceinline__ void store(char* to, int plane) const
    {
        uint32_t w[3][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t a[3], b[3];
            split3(raw[2 * i], a[0], a[1], a[2]);
            split3(raw[2 * i + 1], b[0], b[1], b[2]);
#pragma unroll
            for (int p = 0; p < 3; ++p) w[p][i] = __builtin_amdgcn_perm(b[p], a[p], 0x07060302u);
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) memcpy(to + p * plane, w[p], 32);
    }
};

// Sixteen codes as 16-bit values.
template <class T>
__device__ __forceinline__ void store_codes(const uint4& codes, uint32_t byte, char* to)
{
    float v[8];
    uint32_t w[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        decode8(h ? make_uint2(codes.z, codes.w) : make_uint2(codes.x, codes.y), byte, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (__is_same(T, _Float16)) {
                const _Float16 a[2] = {(_Float16)v[2 * i], (_Float16)v[2 * i + 1]};
                memcpy(&w[4 * h + i], a, 4);
            } else {  // the upper halves, exactly
                w[4 * h + i] = __builtin_amdgcn_perm(__float_as_uint(v[2 * i + 1]), __float_as_uint(v[2 * i]), 0x07060302u);
            }
        }
    }
    memcpy(to, w, 32);
}

__device__ __forceinline__ s16x8 read_transposed(const char* at)
{
    typedef __attribute__((address_space(3))) s16x4* Lds;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)at), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + 4 * kRowBytes));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

template <class T>
__device__ __forceinline__ f32x4 multiply_add(s16x8 a, s16x8 b, f32x4 c)
{
    if constexpr (__is_same(T, _Float16)) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

struct GradientShape {
    uint32_t rows, outs, cols, groups, group_log2;
    uint32_t tiles_in, tiles_out;  // tiles along the inputs and the outputs
    uint32_t part;                 // rows of a part of the sum, a multiple of kDepth
    uint64_t dy_stride, out_stride, out_part;
};

// `out` is dw, or the workspace where the sum is cut into parts (out_part values from one part to the next).
template <class T>
__global__ __launch_bounds__(256) void weight_gradient_kernel(const T* dy, const uint8_t* codes, const uint8_t* exponents, GradientShape s, bool accumulate,
                                                              float* out)
{
    constexpr int kPieces = Rows16<T>::kPieces, kPlane = kDepth * kRowBytes;
    __shared__ __align__(16) char lds[(1 + kPieces) * kPlane];
    const uint32_t tile = blockIdx.x % (s.tiles_in * s.tiles_out), part = blockIdx.x / (s.tiles_in * s.tiles_out);
    const uint32_t i0 = tile % s.tiles_in * kTile, o0 = tile / s.tiles_in * kTile;
    const uint32_t first = part * s.part, last = min(s.rows, first + s.part);
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // what this thread brings to LDS: sixteen values of one row of either factor
    const uint32_t row = threadIdx.x >> 3, chunk = threadIdx.x & 7;
    const uint32_t i_mine = i0 + chunk * 16, o_mine = o0 + chunk * 16;
    const uint64_t pitch = (uint64_t)s.groups << s.group_log2;
    const bool has_codes = i_mine < pitch;
    const int valid = o_mine >= s.outs ? 0 : (int)min(16u, s.outs - o_mine);
    char* to = lds + row * kRowBytes + ((chunk ^ twist(row)) * 32);
    Rows16<T> g;
    uint4 q;
    uint32_t byte;
    const auto fetch = [&](uint32_t t) {
        t += row;
        q = make_uint4(0, 0, 0, 0);
        byte = 127;
        if (t < last && has_codes) {
            q = *reinterpret_cast<const uint4*>(codes + t * pitch + i_mine);
            byte = exponents[(uint64_t)t * s.groups + (i_mine >> s.group_log2)];
        }
        g.load(dy + t * s.dy_stride + o_mine, t < last ? valid : 0);
    };
    f32x4 sum[4][4] = {};
    const uint32_t k = (lane >> 4) * 8 + ((lane >> 2) & 3), f = twist(k);
    const char* from = lds + k * kRowBytes + (lane & 3) * 8;
    const uint32_t ci = (wave & 1) * 4, co = (wave >> 1) * 4;  // first chunk of the wavefront's sums
    if (first < last) fetch(first);
    for (uint32_t t = first; t < last; t += kDepth) {
        __syncthreads();
        store_codes<T>(q, byte, to);
        g.store(to + kPlane, kPlane);
        __syncthreads();
        if (t + kDepth < last) fetch(t + kDepth);
        s16x8 a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = read_transposed(from + ((ci + i) ^ f) * 32);
#pragma unroll
        for (int p = kPieces - 1; p >= 0; --p)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const s16x8 b = read_transposed(from + (1 + p) * kPlane + ((co + j) ^ f) * 32);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i][j] = multiply_add<T>(a[i], b, sum[i][j]);
            }
    }
    out += part * s.out_part;
    const bool wide = ((reinterpret_cast<uintptr_t>(out) | s.out_stride * 4) & 15) == 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t o = o0 + (co + j) * 16 + (lane & 15);
        if (o >= s.outs) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t at = i0 + (ci + i) * 16 + (lane >> 4) * 4;
            if (at >= s.cols) continue;
            float* p = out + o * s.out_stride + at;
            f32x4 v = sum[i][j];
            if (wide && at + 4 <= s.cols) {
                if (accumulate) v += *reinterpret_cast<f32x4*>(p);
                *reinterpret_cast<f32x4*>(p) = v;
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (at + r < s.cols) p[r] = accumulate ? p[r] + v[r] : v[r];
            }
        }
    }
}

// The parts of the sum, added in their order.
__global__ __launch_bounds__(kBlock) void add_parts_kernel(const float* parts, uint32_t number, uint64_t part, uint64_t pitch, uint32_t cols, bool accumulate,
                                                           float* dw, uint64_t dw_stride)
{
    const uint32_t i = (blockIdx.x * kBlock + threadIdx.x) * 4;
    if (i >= cols) return;
    const float* from = parts + blockIdx.y * pitch + i;
    float* to = dw + blockIdx.y * dw_stride + i;
    const int valid = min(4u, cols - i);
    f32x4 v = *reinterpret_cast<const f32x4*>(from);
    for (uint32_t n = 1; n < number; ++n) v += *reinterpret_cast<const f32x4*>(from + n * part);
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (r < valid) to[r] = accumulate ? to[r] + v[r] : v[r];
}

uint32_t ceil_div(uint64_t a, uint64_t b) { return (uint32_t)((a + b - 1) / b); }

// Into how many parts a sum is cut: where the tiles alone do not fill the chip, as many as make 512 workgroups, of 256 rows at least.
uint32_t parts_of(size_t rows, size_t outs, size_t cols)
{
    const uint64_t tiles = (uint64_t)ceil_div(outs, kTile) * ceil_div(cols, kTile);
    const uint64_t wanted = tiles >= 256 ? 1 : (512 + tiles - 1) / tiles, most = (rows + 255) / 256;
    const uint64_t n = wanted < most ? wanted : most;
    return n < 1 ? 1 : (uint32_t)n;
}

uint64_t pitch_of(size_t cols) { return (cols + 3) / 4 * 4; }

}  // namespace

size_t weight_gradient_workspace(size_t rows, size_t outs, size_t cols, uint32_t)
{
    const uint32_t parts = parts_of(rows, outs, cols);
    return parts > 1 ? parts * outs * pitch_of(cols) * sizeof(float) : 0;
}

void launch_weight_gradient(const Values& dy, uint32_t dtype, const Groups& x, size_t rows, size_t outs, size_t cols, const ogq_group_params_t* p,
                            bool accumulate, float* dw, size_t dw_stride, void* workspace, hipStream_t st)
{
    GradientShape s;
    s.rows = (uint32_t)rows, s.outs = (uint32_t)outs, s.cols = (uint32_t)cols;
    s.groups = ceil_div(cols, p->group_size);
    s.group_log2 = p->group_size == 32 ? 5 : p->group_size == 64 ? 6 : 7;
    s.tiles_in = ceil_div(cols, kTile), s.tiles_out = ceil_div(outs, kTile);
    const uint32_t wanted = parts_of(rows, outs, cols);
    s.part = ceil_div(ceil_div(rows, wanted), kDepth) * kDepth;
    const uint32_t parts = wanted;  // (the last ones may be empty: their sums are 0)
    s.dy_stride = dy.stride;
    s.out_stride = parts > 1 ? pitch_of(cols) : dw_stride;
    s.out_part = parts > 1 ? outs * s.out_stride : 0;
    float* out = parts > 1 ? static_cast<float*>(workspace) : dw;
    const bool add = accumulate && parts == 1;
    const dim3 grid(s.tiles_in * s.tiles_out * parts), block(256);
    const auto codes = static_cast<const uint8_t*>(x.codes);
    if (dtype == OGQ_FP32) launch_kernel(weight_gradient_kernel<float>, grid, block, st, static_cast<const float*>(dy.data), codes, x.exponents, s, add, out);
    else if (dtype == OGQ_BF16) launch_kernel(weight_gradient_kernel<__bf16>, grid, block, st, static_cast<const __bf16*>(dy.data), codes, x.exponents, s, add, out);
    else launch_kernel(weight_gradient_kernel<_Float16>, grid, block, st, static_cast<const _Float16*>(dy.data), codes, x.exponents, s, add, out);
    if (parts > 1)
        launch_kernel(add_parts_kernel, dim3(ceil_div(cols, 4 * kBlock), (uint32_t)outs), dim3(kBlock), st, out, parts, s.out_part, s.out_stride, s.cols,
                      accumulate, dw, (uint64_t)dw_stride);
}

}  // namespace ogq
