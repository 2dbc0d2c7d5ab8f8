// libogq_layers: products of a few tokens with a layer's weights, which are read once: bound by memory, on the vector unit.
#include "layers_linear.h"

namespace ogq {

namespace {

// y[t][o] = sum over i of x[t][i] * W[o][i]: ROWS rows of weights to a wavefront, or a share of their columns where SPLIT wavefronts of a workgroup have the same rows.  A lane
// takes every 64th piece of a row.  One token through 16384 x 4096 bf16: 20 to 23 us, 5.9 to 6.9 TB/s, the rate at which memory is read.
template <class T, int TOKENS, int ROWS, int SPLIT>
__global__ __launch_bounds__(kBlock) void few_tokens_kernel(const T* x, const T* weight, LinearShape s, Epilogue<T> e)
{
    constexpr int N = kPiece<T>;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), share = SPLIT == 1 ? 0 : wave;
    const uint32_t first = (this_block() * (4 / SPLIT) + (SPLIT == 1 ? wave : 0)) * ROWS;
    float sum[ROWS][TOKENS] = {};
    if (first < s.outs) {
        const T* rows[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) rows[r] = weight + (uint64_t)min(first + r, s.outs - 1) * s.weight_stride;
        const auto products = [&](const uint4 (&w)[ROWS], const uint4 (&v)[TOKENS]) __attribute__((always_inline)) {
            float a[ROWS][N];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) values_of<T>(w[r], a[r]);
#pragma unroll
            for (int t = 0; t < TOKENS; ++t) {
                float b[N];
                values_of<T>(v[t], b);
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
#pragma unroll
                    for (int i = 0; i < N; ++i) sum[r][t] = __builtin_fmaf(a[r][i], b[i], sum[r][t]);
            }
        };
        const uint32_t step = 64 * SPLIT * N;
        uint32_t at = (share * 64 + lane) * N;
        uint4 w[ROWS], v[TOKENS];
        // what a lane's last piece does not have is 0 in both
        const auto fetch = [&](uint32_t col) __attribute__((always_inline)) {
            const int valid = valid_of<T>(col, s.cols);
#pragma unroll
            for (int r = 0; r < ROWS; ++r) w[r] = load_raw(rows[r] + col, valid);
#pragma unroll
            for (int t = 0; t < TOKENS; ++t) v[t] = load_raw(x + t * s.x_stride + col, valid);
        };
        const uint32_t whole = s.cols / N * N;
        // two steps' loads under way together
        for (; at + step < whole; at += 2 * step) {
            uint4 w2[ROWS], v2[TOKENS];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) w[r] = load_whole(rows[r] + at), w2[r] = load_whole(rows[r] + at + step);
#pragma unroll
            for (int t = 0; t < TOKENS; ++t) v[t] = load_whole(x + t * s.x_stride + at), v2[t] = load_whole(x + t * s.x_stride + at + step);
            products(w, v);
            products(w2, v2);
        }
        for (; at < s.cols; at += step) {
            fetch(at);
            products(w, v);
        }
    }
    // all lanes' sums; lane r * TOKENS + t of the wavefront keeps the sum of row r and token t
    float mine = 0.0f;
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) {
            const float total = wave_sum_f32(sum[r][t]);
            if (lane == r * TOKENS + t) mine = total;
        }
    if constexpr (SPLIT != 1) {
        __shared__ float space[SPLIT][64];
        space[wave][lane] = mine;
        __syncthreads();
        if (wave != 0) return;
        mine = space[0][lane];
#pragma unroll
        for (int n = 1; n < SPLIT; ++n) mine += space[n][lane];
    }
    const uint32_t out = first + lane / TOKENS, token = lane % TOKENS;
    if (lane >= ROWS * TOKENS || out >= s.outs) return;
    float v[N] = {mine};
    e(token, out, 1, v);
}

// y[t][o] = sum over k of x[t][k] * W[k][o], in fp32: 64 pieces of a row of weights to a workgroup, and `part` rows, which its four wavefronts take in turn.  One token, 4096 x 16384: 41 us
// (6.5 TB/s).
template <int TOKENS>
__global__ __launch_bounds__(kBlock) void few_tokens_across_kernel(const float* x, const float* weight, LinearShape s, Epilogue<float> e)
{
    constexpr int N = kPiece<float>, kAhead = 8;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t block = this_block() % s.tiles_out, part = this_block() / s.tiles_out;
    if (part >= s.parts) return;
    const uint32_t out = (block * 64 + lane) * N;
    const int valid = valid_of<float>(out, s.outs);
    const uint32_t first = part * s.part, last = min(s.cols, first + s.part);
    float sum[TOKENS][N] = {};
    if (valid != 0) {
        for (uint32_t at = first + wave * kAhead; at < last; at += 4 * kAhead) {
            uint4 w[kAhead];
            float v[TOKENS][kAhead];
#pragma unroll
            for (int n = 0; n < kAhead; ++n) {
                const uint32_t row = min(at + n, last - 1);
                w[n] = load_raw(weight + (uint64_t)row * s.weight_stride + out, valid);
#pragma unroll
                for (int t = 0; t < TOKENS; ++t) v[t][n] = x[t * s.x_stride + row];
            }
#pragma unroll
            for (int n = 0; n < kAhead; ++n) {
                if (at + n >= last) break;
                float a[N];
                values_of<float>(w[n], a);
#pragma unroll
                for (int t = 0; t < TOKENS; ++t)
#pragma unroll
                    for (int i = 0; i < N; ++i) sum[t][i] = __builtin_fmaf(a[i], v[t][n], sum[t][i]);
            }
        }
    }
    __shared__ float space[3][N][64];
#pragma unroll 1
    for (int t = 0; t < TOKENS; ++t) {
        float mine[N];
#pragma unroll
        for (int k = 0; k < TOKENS; ++k)
            if (k == t) {
#pragma unroll
                for (int i = 0; i < N; ++i) mine[i] = sum[k][i];
            }
        if (wave != 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) space[wave - 1][i][lane] = mine[i];
        }
        __syncthreads();
        if (wave == 0 && valid != 0) {
#pragma unroll
            for (int n = 0; n < 3; ++n)
#pragma unroll
                for (int i = 0; i < N; ++i) mine[i] += space[n][i][lane];
            if (s.sums == nullptr) e(t, out, valid, mine);
            else memcpy(s.sums + ((uint64_t)part * TOKENS + t) * s.pitch + out, mine, sizeof mine);
        }
        __syncthreads();
    }
}

}  // namespace

// Rows of weights: four to a wavefront or, where all of a workgroup's wavefronts find a piece of a row, to a workgroup; one where there are few.  bf16, one token, by wavefront and by workgroup:
// 16384 x 4096 22.8 us and 19.5, 4096 x 16384 26.6 and 20.0, 50000 x 1024 15.7 and 15.5, 16384 x 1024 4.0 and 5.8, 16384 x 256 4.1 and 5.1; 4096 x 256 4.6 and 4.3.
template <class T>
void launch_few(const T* x, const T* weight, const LinearShape& s, const Epilogue<T>& e, hipStream_t st)
{
    const bool split = s.outs < 8192 || s.cols >= (sizeof(T) == 4 ? 1024u : 2048u);
    const auto go = [&](auto number) {
        constexpr int kTokens = decltype(number)::value;
        if (s.tokens != kTokens) return;
        if (s.outs < 2048) launch_kernel(few_tokens_kernel<T, kTokens, 1, 4>, grid_of(s.outs), dim3(kBlock), st, x, weight, s, e);
        else if (split) launch_kernel(few_tokens_kernel<T, kTokens, 4, 4>, grid_of(ceil_div(s.outs, 4)), dim3(kBlock), st, x, weight, s, e);
        else launch_kernel(few_tokens_kernel<T, kTokens, 4, 1>, grid_of(ceil_div(s.outs, 16)), dim3(kBlock), st, x, weight, s, e);
    };
    go(std::integral_constant<int, 1>{}), go(std::integral_constant<int, 2>{}), go(std::integral_constant<int, 3>{}), go(std::integral_constant<int, 4>{});
    go(std::integral_constant<int, 5>{}), go(std::integral_constant<int, 6>{}), go(std::integral_constant<int, 7>{}), go(std::integral_constant<int, 8>{});
}

// As many parts as give enough workgroups, of 32 rows at least, since the parts' sums are written and read again.
FewParts few_parts(size_t outs, size_t cols)
{
    if (cols == 0) return {32, 1};
    const uint64_t blocks = ceil_div(outs, 256), wanted = blocks < 512 ? 512 / blocks : 1, most = cols < 64 ? 1 : cols / 32, parts = wanted < most ? wanted : most;
    const uint32_t part = (uint32_t)(ceil_div(ceil_div(cols, parts), 32) * 32);
    return {part, (uint32_t)ceil_div(cols, part)};
}

void launch_few_across(const float* x, const float* weight, LinearShape s, const Epilogue<float>& e, float* workspace, hipStream_t st)
{
    const FewParts parts = few_parts(s.outs, s.cols);
    s.tiles_out = (uint32_t)ceil_div(s.outs, 256), s.part = parts.part, s.parts = parts.parts;
    s.sums = parts.parts > 1 ? workspace : nullptr;
    const auto go = [&](auto number) {
        constexpr int kTokens = decltype(number)::value;
        if (s.tokens == kTokens) launch_kernel(few_tokens_across_kernel<kTokens>, grid_of((uint64_t)s.tiles_out * s.parts), dim3(kBlock), st, x, weight, s, e);
    };
    go(std::integral_constant<int, 1>{}), go(std::integral_constant<int, 2>{}), go(std::integral_constant<int, 3>{}), go(std::integral_constant<int, 4>{});
    go(std::integral_constant<int, 5>{}), go(std::integral_constant<int, 6>{}), go(std::integral_constant<int, 7>{}), go(std::integral_constant<int, 8>{});
    if (s.sums != nullptr) launch_join_parts(s, e, st);
}

template void launch_few(const float*, const float*, const LinearShape&, const Epilogue<float>&, hipStream_t);
template void launch_few(const __bf16*, const __bf16*, const LinearShape&, const Epilogue<__bf16>&, hipStream_t);
template void launch_few(const _Float16*, const _Float16*, const LinearShape&, const Epilogue<_Float16>&, hipStream_t);

}  // namespace ogq
