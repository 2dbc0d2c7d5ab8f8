// libogq_groups: tokens times the transpose of weights held in 4 bits,
//   y[t][o] = sum over i of x[t][i] * w^[o][i].
//
// The weights are read once, 16 bytes per lane, and become 8 values of bf16 per dword in four conversions that take the group's power along;
// they are the left operand of a matrix instruction whose 16 columns are tokens.  The order of the summed index within an instruction does
// not matter as long as both operands have it: lane l holds 32 consecutive weights of row l % 16, and the tokens' values follow them.
#include "groups_common.h"

namespace ogq {

namespace {

constexpr int kRows = 16;     // rows of weights of a workgroup
constexpr int kStep = 128;    // columns of a wavefront's step: 32 weights in each of four lanes
constexpr int kSplit = 8;     // wavefronts of a workgroup, which share the columns

template <class T>
constexpr int kPiecesOf = __is_same(T, __bf16) ? 1 : __is_same(T, _Float16) ? 2 : 3;

// Eight values of a token in pieces of bf16 whose sum they are.
template <class T>
__device__ __forceinline__ void pieces_of(const T* x, int valid, bf16x8 (&out)[kPiecesOf<T>])
{
    if constexpr (__is_same(T, __bf16)) {
        uint16_t v[8];
        if (valid >= 8) {
            memcpy(v, x, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = 0;
                if (i < valid) memcpy(&v[i], x + i, 2);
            }
        }
        memcpy(&out[0], v, 16);
    } else {
        float v[8];
        load8(x, valid, v);
        uint32_t w[3][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t a[3], b[3];
            split3(v[2 * i], a[0], a[1], a[2]);
            split3(v[2 * i + 1], b[0], b[1], b[2]);
#pragma unroll
            for (int p = 0; p < 3; ++p) w[p][i] = __builtin_amdgcn_perm(b[p], a[p], 0x07060302u);
        }
#pragma unroll
        for (int p = 0; p < kPiecesOf<T>; ++p) memcpy(&out[p], w[p], 16);
    }
}

struct MatvecShape {
    uint32_t tokens, outs, cols, groups, group_log2, row_blocks;
    uint64_t x_stride, y_stride;
};

template <class T>
__global__ __launch_bounds__(64 * kSplit) void group_matvec_kernel(const uint8_t* codes, const uint8_t* exponents, const T* x, MatvecShape s, T* y)
{
    constexpr int kPieces = kPiecesOf<T>;
    __shared__ f32x4 parts[kSplit][64];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t o0 = blockIdx.x % s.row_blocks * kRows, t0 = blockIdx.x / s.row_blocks * 16;
    const uint32_t row = min(o0 + (lane & 15), s.outs - 1), token = min(t0 + (lane & 15), s.tokens - 1);  // (what is not there repeats the last)
    const uint64_t pitch = (uint64_t)s.groups << s.group_log2;
    const uint8_t* w_row = codes + row * (pitch / 2);
    const uint8_t* e_row = exponents + (uint64_t)row * s.groups;
    const T* x_row = x + token * s.x_stride;
    f32x4 sum = {};
    for (uint32_t i = wave * kStep + (lane >> 4) * 32; i - (lane >> 4) * 32 < pitch; i += kSplit * kStep) {
        uint4 w = make_uint4(0, 0, 0, 0);
        uint32_t byte = 127;
        if (i < pitch) {
            w = *reinterpret_cast<const uint4*>(w_row + i / 2);
            byte = e_row[i >> s.group_log2];
        }
        const float unit = power(byte);
        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            bf16x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word[j], unit, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word[j], unit, 1),
                           __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word[j], unit, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word[j], unit, 3)};
            bf16x8 a;
            memcpy(&a, p, 16);
            bf16x8 b[kPieces];
            const int left = (int)s.cols - (int)(i + 8 * j);
            pieces_of<T>(x_row + i + 8 * j, left, b);
#pragma unroll
            for (int q = kPieces - 1; q >= 0; --q) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b[q], sum, 0, 0, 0);
        }
    }
    parts[wave][lane] = sum;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int n = 1; n < kSplit; ++n) sum += parts[n][lane];
    const uint32_t t = t0 + (lane & 15), o = o0 + (lane >> 4) * 4;
    if (t >= s.tokens) return;
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (o + r < s.outs) y[t * s.y_stride + o + r] = (T)sum[r];
}

}  // namespace

size_t group_matvec_workspace(size_t, size_t, size_t, uint32_t) { return 0; }

void launch_group_matvec(const Groups& w, size_t outs, size_t cols, const ogq_group_params_t* p, const Values& x, size_t tokens, uint32_t dtype,
                         const Result& y, void*, hipStream_t st)
{
    MatvecShape s;
    s.tokens = (uint32_t)tokens, s.outs = (uint32_t)outs, s.cols = (uint32_t)cols;
    s.groups = (uint32_t)((cols + p->group_size - 1) / p->group_size);
    s.group_log2 = p->group_size == 32 ? 5 : p->group_size == 64 ? 6 : 7;
    s.x_stride = x.stride, s.y_stride = y.stride;
    s.row_blocks = (uint32_t)((outs + kRows - 1) / kRows);
    const dim3 grid(s.row_blocks * (uint32_t)((tokens + 15) / 16)), block(64 * kSplit);
    const auto codes = static_cast<const uint8_t*>(w.codes);
    if (dtype == OGQ_FP32) launch_kernel(group_matvec_kernel<float>, grid, block, st, codes, w.exponents, static_cast<const float*>(x.data), s, static_cast<float*>(y.data));
    else if (dtype == OGQ_BF16) launch_kernel(group_matvec_kernel<__bf16>, grid, block, st, codes, w.exponents, static_cast<const __bf16*>(x.data), s, static_cast<__bf16*>(y.data));
    else launch_kernel(group_matvec_kernel<_Float16>, grid, block, st, codes, w.exponents, static_cast<const _Float16*>(x.data), s, static_cast<_Float16*>(y.data));
}

}  // namespace ogq
