// libogq_layers: layer norm and its backward pass, and what a linear layer's backward pass begins with; sums over the rows of all of them.
//
// A row stays in the registers of 64, 256 or 1024 threads from its only load on: its mean, the differences from it, their squares, the result.  Bound by memory.
#include "layers_common.h"

namespace ogq {

namespace {

// How rows are cut: a workgroup of 256 threads has four rows of 64 threads each, or one row; one of 1024 threads one row.
constexpr int block_of(int threads) { return threads == 64 ? kBlock : threads; }

template <int THREADS>
__device__ __forceinline__ uint64_t first_row()
{
    return THREADS == 64 ? (uint64_t)this_block() * 4 + (threadIdx.x >> 6) : this_block();
}

constexpr float kDown = 0x1p-32f, kUp = 0x1p32f, kLargest = 0x1.fffffep127f;

// A row's mean; sum_of(factor) is the sum of its values times a factor.  Where the sum is beyond fp32 though the values are not, it is taken of 2^-32 times the values.
template <class F>
__device__ __forceinline__ float mean_of(F sum_of, float per_col)
{
    const float m = sum_of(1.0f) * per_col;
    if (fabsf(m) < INFINITY) return m;  // (NaN where parts of the sum are infinite)
    const float sum = sum_of(kDown);
    // (the mean of the largest values may be rounded beyond them)
    return !(fabsf(sum) < INFINITY) ? sum : fminf(fmaxf(sum * per_col, -kLargest * kDown), kLargest * kDown) * kUp;
}

// What is left of the mean's rounding, and 1 / deviation, from the sums of the differences from the mean and of their squares; squares_of(factor) is the sum of squares of the differences times a factor, for
// sums that are beyond fp32 where the variance is not, and for squares that are too small for it.  rstd is 0 where the variance is beyond fp32, NaN where a value is NaN or infinite.
struct Spread {
    float rest, rstd;
};

template <class F>
__device__ __forceinline__ Spread spread_of(float2 sums, float per_col, float eps, F squares_of)
{
    const float rest = sums.x * per_col;
    float variance = sums.y * per_col;
    if (variance == INFINITY) variance = squares_of(kDown) * per_col * kUp * kUp;
    if (variance == INFINITY) return {fabsf(rest) < INFINITY ? rest : 0.0f, 0.0f};  // (of infinite differences: the sum may be NaN)
    variance = __builtin_fmaf(-rest, rest, variance);
    variance = variance < 0.0f ? 0.0f : variance;
    if (variance + eps < 0x1p-96f) {  // (squares are lost below the least number)
        constexpr float kFactor = 0x1p80f;
        const float scaled = __builtin_fmaf(-rest * kFactor, rest * kFactor, squares_of(kFactor) * per_col);
        return {rest, kFactor / sqrtf((scaled < 0.0f ? 0.0f : scaled) + eps * kFactor * kFactor)};
    }
    return {rest, 1.0f / sqrtf(variance + eps)};
}

// P pieces of a row to each of THREADS threads.  `off`, the differences from the mean as it came out of fp32 sums, are summed too: what is left of the mean's rounding is taken off
// again, so that an offset of the whole row costs nothing but the rounding of x.  Bound by memory: 8192 x 4096 bf16 24.7 us, 5.4 TB/s read and written; one row of 4096 2.9 us, latency.
template <class T, int THREADS, int P>
__global__ __launch_bounds__(block_of(THREADS)) void layer_norm_forward_kernel(const T* x, uint64_t x_stride, uint32_t rows, uint32_t cols, const float* weight, const float* bias,
                                                                             float eps, float per_col, T* y, uint64_t y_stride, float* mean, float* rstd)
{
    constexpr int kWaves = THREADS / 64;
    __shared__ float2 space[2][kWaves];
    BlockSums<kWaves> sums{space};
    const uint64_t row = first_row<THREADS>();
    if (row >= rows) return;
    const uint32_t thread = threadIdx.x & (THREADS - 1);
    const T* from = x + row * x_stride;
    const auto at = [&](int p) __attribute__((always_inline)) { return piece_at<T, THREADS, P>(p, thread, cols); };
    float v[P][kPiece<T>];
#pragma unroll
    for (int p = 0; p < P; ++p) values_of<T>(load_whole(from + at(p).col), v[p]);
    const float m = mean_of(
        [&](float factor) __attribute__((always_inline)) {
            float total = 0.0f;
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < kPiece<T>; ++i) total += at(p).counts(i) ? v[p][i] * factor : 0.0f;
            return sums(total, 0.0f).x;
        },
        per_col);
    float off = 0.0f, squares = 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < kPiece<T>; ++i) {
            v[p][i] -= m;
            const float d = at(p).counts(i) ? v[p][i] : 0.0f;
            off += d;
            squares = __builtin_fmaf(d, d, squares);
        }
    const Spread s = spread_of(sums(off, squares), per_col, eps, [&](float factor) __attribute__((always_inline)) {
        float squares = 0.0f;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < kPiece<T>; ++i) {
                const float d = at(p).counts(i) ? v[p][i] * factor : 0.0f;
                squares = __builtin_fmaf(d, d, squares);
            }
        return sums(squares, 0.0f).x;
    });
    const float rest = s.rest, r = s.rstd;
    if (thread == 0 && mean != nullptr) mean[row] = m + rest, rstd[row] = r;
    if (r == 0.0f) {  // (differences may be infinite)
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < kPiece<T>; ++i) v[p][i] = rest;
    }
    T* to = y + row * y_stride;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (!at(p).there) continue;
        float w[kPiece<T>], b[kPiece<T>];
        load_vector<T>(weight, at(p).col, 1.0f, w);
        load_vector<T>(bias, at(p).col, 0.0f, b);
#pragma unroll
        for (int i = 0; i < kPiece<T>; ++i) v[p][i] = __builtin_fmaf((v[p][i] - rest) * r, w[i], b[i]);
        store_piece<false>(to + at(p).col, kPiece<T>, v[p]);
    }
}

// Rows of any length, read three times (twice from the caches), by a workgroup each.
template <class T>
__global__ __launch_bounds__(1024) void layer_norm_forward_long_kernel(const T* x, uint64_t x_stride, uint32_t rows, uint32_t cols, const float* weight, const float* bias, float eps,
                                                                     float per_col, T* y, uint64_t y_stride, float* mean, float* rstd)
{
    __shared__ float2 space[2][16];
    BlockSums<16> sums{space};
    const uint64_t row = this_block();
    if (row >= rows) return;
    const T* from = x + row * x_stride;
    float v[kPiece<T>];
    const float m = mean_of(
        [&](float factor) __attribute__((always_inline)) {
            float total = 0.0f;
            for (uint32_t col = threadIdx.x * kPiece<T>; col < cols; col += 1024 * kPiece<T>) {
                load_piece<false>(from + col, valid_of<T>(col, cols), v);
                float t = 0.0f;
#pragma unroll
                for (int i = 0; i < kPiece<T>; ++i) t += v[i] * factor;
                total += t;
            }
            return sums(total, 0.0f).x;
        },
        per_col);
    // the sums of the differences and of their squares, these of `factor` times them
    const auto differences = [&](float factor) __attribute__((always_inline)) {
        float off = 0.0f, squares = 0.0f;
        for (uint32_t col = threadIdx.x * kPiece<T>; col < cols; col += 1024 * kPiece<T>) {
            const int valid = valid_of<T>(col, cols);
            load_piece<false>(from + col, valid, v);
            float o = 0.0f, q = 0.0f;
#pragma unroll
            for (int i = 0; i < kPiece<T>; ++i) {
                const float d = i < valid ? v[i] - m : 0.0f;
                o += d;
                q = __builtin_fmaf(d * factor, d * factor, q);
            }
            off += o, squares += q;
        }
        return sums(off, squares);
    };
    const Spread s = spread_of(differences(1.0f), per_col, eps, [&](float factor) { return differences(factor).y; });
    const float rest = s.rest, r = s.rstd;
    if (threadIdx.x == 0 && mean != nullptr) mean[row] = m + rest, rstd[row] = r;
    T* to = y + row * y_stride;
    for (uint32_t col = threadIdx.x * kPiece<T>; col < cols; col += 1024 * kPiece<T>) {
        const int valid = valid_of<T>(col, cols);
        load_piece<false>(from + col, valid, v);
        float w[kPiece<T>], b[kPiece<T>];
        load_vector<T>(weight == nullptr ? nullptr : weight + col, valid, 1.0f, w);
        load_vector<T>(bias == nullptr ? nullptr : bias + col, valid, 0.0f, b);
#pragma unroll
        for (int i = 0; i < kPiece<T>; ++i) v[i] = __builtin_fmaf((r == 0.0f ? 0.0f : v[i] - m - rest) * r, w[i], b[i]);  // (differences may be infinite)
        store_piece<false>(to + col, valid, v);
    }
}

// A row's mean for its backward pass: differences from it, which may be infinite where the variance is beyond fp32, count for nothing there.
__device__ __forceinline__ float mean_for(float mean, float rstd) { return rstd == 0.0f ? 0.0f : mean; }

// Rows that lie far from zero, measured by their deviation: what the rounding of their mean has left in u is taken off it again, the mean of u.  (Of other rows it is at most 2^-20.)
__device__ __forceinline__ bool is_far(float mean, float rstd) { return fabsf(mean * rstd) > 16.0f; }

// What a row's gradient takes from the whole row: the mean of u, where the row is far from zero, and with what is left of u the means of g and g * u.
struct RowMeans {
    float off, plain, along;
};

// What the kernels that add over the rows have in common: rows first ... last of workgroup n are n * part ..., its sums go to parts[n][2][pitch] (weight, then bias).
struct RowParts {
    uint32_t rows, cols, part, pitch;
    float per_col;
    float* parts;  // null: no sums, or those of the only part
    float *first, *second;  // where these go: weight and bias, or the one vector there is, in `first`
    bool accumulate;
};

// Sums of an only part: one or two vectors, of which a thread has these values.
template <int N, class F>
__device__ __forceinline__ void store_only(float* to, bool accumulate, const float (&v)[N], F counts)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (counts(i)) to[i] = accumulate ? to[i] + v[i] : v[i];
}

// The backward pass of rows that THREADS threads hold, P pieces each.  A row's values set off while the one before is worked on.  64 threads to a row: the four wavefronts of a workgroup
// take its rows in turn, and add their sums over the rows in LDS in the end.  Bound by memory: 8192 x 4096 bf16 45 us, 4.9 TB/s with the parts' sums (36 with what the caches hold); 1237 x 1001 fp32 5.8 us, latency.
template <class T, int THREADS, int P>
__global__ __launch_bounds__(block_of(THREADS)) void layer_norm_backward_kernel(const T* dy, uint64_t dy_stride, const T* x, uint64_t x_stride, RowParts s, const float* weight,
                                                                              const float* mean, const float* rstd, T* dx, uint64_t dx_stride)
{
    constexpr int kWaves = THREADS / 64, N = kPiece<T>, kTurn = THREADS == 64 ? 4 : 1;
    __shared__ float2 space[2][kWaves];
    BlockSums<kWaves> sums{space};
    const uint32_t thread = threadIdx.x & (THREADS - 1), mine = THREADS == 64 ? threadIdx.x >> 6 : 0;
    const uint32_t first = this_block() * s.part, last = min(s.rows, first + s.part);
    const auto at = [&](int p) __attribute__((always_inline)) { return piece_at<T, THREADS, P>(p, thread, s.cols); };
    float w[P][N], dw[P][N], db[P][N];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        load_vector<T>(weight, at(p).col, 1.0f, w[p]);
#pragma unroll
        for (int i = 0; i < N; ++i) dw[p][i] = db[p][i] = 0.0f;
    }
    uint4 next_x[P], next_dy[P];
    float next_mean = 0.0f, next_rstd = 0.0f;
    // (16384 values of 16 bits to a row leave no registers for another one)
    constexpr bool kAhead = !(THREADS == 1024 && P == 2 && N == 8);
    const auto fetch = [&](uint32_t row) __attribute__((always_inline)) {
        if (row >= last) return;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            next_x[p] = load_whole(x + row * x_stride + at(p).col);
            next_dy[p] = load_whole(dy + row * dy_stride + at(p).col);
        }
        next_mean = mean[row], next_rstd = rstd[row];
    };
    if (kAhead) fetch(first + mine);
    for (uint32_t row = first + mine; row < last; row += kTurn) {
        if (!kAhead) fetch(row);
        float u[P][N], g[P][N];
        const float r = next_rstd, m = mean_for(next_mean, r);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            values_of<T>(next_x[p], u[p]);
#pragma unroll
            for (int i = 0; i < N; ++i) u[p][i] = (u[p][i] - m) * r;
        }
        if (is_far(m, r)) {
            float off = 0.0f;
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < N; ++i) off += at(p).counts(i) ? u[p][i] : 0.0f;
            off = sums(off, 0.0f).x * s.per_col;
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < N; ++i) u[p][i] -= off;
        }
        float along = 0.0f, plain = 0.0f;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            values_of<T>(next_dy[p], g[p]);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                dw[p][i] = __builtin_fmaf(g[p][i], u[p][i], dw[p][i]);
                db[p][i] += g[p][i];
                g[p][i] *= w[p][i];
                plain += at(p).counts(i) ? g[p][i] : 0.0f;
                along += at(p).counts(i) ? g[p][i] * u[p][i] : 0.0f;
            }
        }
        if (kAhead) fetch(row + kTurn);
        const float2 t = sums(plain, along);
        const float a = t.x * s.per_col, b = t.y * s.per_col;
        T* to = dx + row * dx_stride;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (!at(p).there) continue;
#pragma unroll
            for (int i = 0; i < N; ++i) g[p][i] = r * (g[p][i] - __builtin_fmaf(u[p][i], b, a));
            store_piece<false>(to + at(p).col, N, g[p]);
        }
    }
    if (s.parts == nullptr && s.first == nullptr) return;
    if constexpr (THREADS == 64) {
        __shared__ float shared[2][64 * P * N];
        // wavefront after wavefront, in their order
        for (uint32_t turn = 0; turn < 3; ++turn) {
            if (mine == turn) {
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        float& a = shared[0][(p * N + i) * 64 + thread];
                        float& b = shared[1][(p * N + i) * 64 + thread];
                        a = turn == 0 ? dw[p][i] : a + dw[p][i];
                        b = turn == 0 ? db[p][i] : b + db[p][i];
                    }
            }
            __syncthreads();
        }
        if (mine != 3) return;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                dw[p][i] += shared[0][(p * N + i) * 64 + thread];
                db[p][i] += shared[1][(p * N + i) * 64 + thread];
            }
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (!at(p).there) continue;
        if (s.parts == nullptr) {
            store_only(s.first + at(p).col, s.accumulate, dw[p], [&](int i) { return at(p).counts(i); });
            store_only(s.second + at(p).col, s.accumulate, db[p], [&](int i) { return at(p).counts(i); });
            continue;
        }
        float* out = s.parts + (uint64_t)this_block() * 2 * s.pitch;
        memcpy(out + at(p).col, dw[p], sizeof dw[p]);
        memcpy(out + s.pitch + at(p).col, db[p], sizeof db[p]);
    }
}

// Rows of any length: the gradient of x by a workgroup for each row, which reads it twice; or, where there are sums over the rows too, only what the gradient takes from the whole row.
template <class T>
__global__ __launch_bounds__(1024) void layer_norm_backward_long_kernel(const T* dy, uint64_t dy_stride, const T* x, uint64_t x_stride, uint32_t rows, uint32_t cols, float per_col,
                                                                      const float* weight, const float* mean, const float* rstd, T* dx, uint64_t dx_stride, RowMeans* means)
{
    constexpr int N = kPiece<T>;
    __shared__ float2 space[2][16];
    BlockSums<16> sums{space};
    const uint64_t row = this_block();
    if (row >= rows) return;
    const float r = rstd[row], m = mean_for(mean[row], r);
    RowMeans t{};
    if (is_far(m, r)) {
        float off = 0.0f, v[N];
        for (uint32_t col = threadIdx.x * N; col < cols; col += 1024 * N) {
            const int valid = valid_of<T>(col, cols);
            load_piece<false>(x + row * x_stride + col, valid, v);
            float c = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) c += i < valid ? (v[i] - m) * r : 0.0f;
            off += c;
        }
        t.off = sums(off, 0.0f).x * per_col;
    }
    float u[N], g[N], w[N];
    const auto piece = [&](uint32_t col, int valid) __attribute__((always_inline)) {
        load_piece<false>(x + row * x_stride + col, valid, u);
        load_piece<false>(dy + row * dy_stride + col, valid, g);
        load_vector<T>(weight == nullptr ? nullptr : weight + col, valid, 1.0f, w);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            u[i] = i < valid ? (u[i] - m) * r - t.off : 0.0f;
            g[i] *= w[i];
        }
    };
    float along = 0.0f, plain = 0.0f;
    for (uint32_t col = threadIdx.x * N; col < cols; col += 1024 * N) {
        piece(col, valid_of<T>(col, cols));
        float a = 0.0f, b = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) a += g[i], b = __builtin_fmaf(g[i], u[i], b);
        plain += a, along += b;
    }
    const float2 all = sums(plain, along);
    t.plain = all.x * per_col, t.along = all.y * per_col;
    if (means != nullptr) {
        if (threadIdx.x == 0) means[row] = t;
        return;
    }
    for (uint32_t col = threadIdx.x * N; col < cols; col += 1024 * N) {
        const int valid = valid_of<T>(col, cols);
        piece(col, valid);
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] = r * (g[i] - __builtin_fmaf(u[i], t.along, t.plain));
        store_piece<false>(dx + row * dx_stride + col, valid, g);
    }
}

enum class Columns { kNorm, kActivation, kSums };

// Sums down the columns: a workgroup has 64 pieces of its columns and `part` rows, which its four wavefronts take in turn, and whose sums they add in LDS.
//   kNorm        the gradient of x, stored in dz, and the sums of dy * u and dy, of rows that no workgroup holds whole, from the rows' means
//   kActivation  dz = dy * act'(z), stored, and the sums of dz (s.parts may be null)
//   kSums        the sums of dy
// Bound by memory, and by the latency of four rows under way in a wavefront: kActivation (gelu by tanh) of 4096 x 4096 bf16 30 us with what the caches hold, 3.4 TB/s; of slopes that only a 16-bit dz needs 28,
// so that the vector unit's work is not all hidden.  kNorm of 2000 x 20000 fp32, with the rows' means before it, 162 us, 4.9 TB/s of x and dy read twice and dx written.
template <class T, Columns WHAT>
__global__ __launch_bounds__(kBlock) void columns_kernel(const T* dy, uint64_t dy_stride, const T* x, uint64_t x_stride, RowParts s, uint32_t blocks, const float* weight,
                                                       const float* mean, const float* rstd, const RowMeans* means, uint32_t act, T* dz, uint64_t dz_stride)
{
    constexpr int N = kPiece<T>, kVectors = WHAT == Columns::kNorm ? 2 : 1, kAhead = 4;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t block = this_block(), part = block / blocks, col = (block % blocks * 64 + lane) * N;
    const uint64_t first = (uint64_t)part * s.part, last = min((uint64_t)s.rows, first + s.part);
    if (first >= s.rows) return;  // (behind the last part, in the last row of a large grid)
    const int valid = valid_of<T>(col, s.cols);
    float sum[kVectors][N];
#pragma unroll
    for (int k = 0; k < kVectors; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) sum[k][i] = 0.0f;
    if (valid != 0) {
        float w[N];
        if constexpr (WHAT == Columns::kNorm) load_vector<T>(weight == nullptr ? nullptr : weight + col, valid, 1.0f, w);
        for (uint64_t at = first + wave; at < last; at += 4 * kAhead) {
            uint4 g_raw[kAhead], x_raw[kAhead];
            float m[kAhead], r[kAhead];
            RowMeans t[kAhead];
#pragma unroll
            for (int n = 0; n < kAhead; ++n) {
                const uint64_t row = min(at + 4 * n, last - 1);
                g_raw[n] = load_raw(dy + row * dy_stride + col, valid);
                if constexpr (WHAT != Columns::kSums) x_raw[n] = load_raw(x + row * x_stride + col, valid);
                if constexpr (WHAT == Columns::kNorm) r[n] = rstd[row], m[n] = mean_for(mean[row], r[n]), t[n] = means[row];
            }
#pragma unroll
            for (int n = 0; n < kAhead; ++n) {
                const uint64_t row = at + 4 * n;
                if (row >= last) break;
                float g[N], v[N];
                values_of<T>(g_raw[n], g);
                if constexpr (WHAT != Columns::kSums) values_of<T>(x_raw[n], v);
                if constexpr (WHAT == Columns::kNorm) {
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const float u = i < valid ? (v[i] - m[n]) * r[n] - t[n].off : 0.0f;
                        v[i] = r[n] * (g[i] * w[i] - __builtin_fmaf(u, t[n].along, t[n].plain));
                        sum[0][i] = __builtin_fmaf(g[i], u, sum[0][i]);
                        sum[1][i] += g[i];
                    }
                    store_piece<false>(dz + row * dz_stride + col, valid, v);
                    continue;
                }
                if constexpr (WHAT == Columns::kActivation) {
                    // (a z beyond fp16 was finite for the forward pass: its slope is the one far out, not infinity times 0)
                    if constexpr (__is_same(T, _Float16)) {
#pragma unroll
                        for (int i = 0; i < N; ++i) v[i] = fabsf(v[i]) == INFINITY ? copysignf(0x1p100f, v[i]) : v[i];
                    }
                    each_as<true>(act, v, [&](int i, float, float slope) { g[i] *= slope; });  // (16-bit types too: the sums are of 32 bits)
                    store_piece<false>(dz + row * dz_stride + col, valid, g);
                }
#pragma unroll
                for (int i = 0; i < N; ++i) sum[0][i] += g[i];
            }
        }
    }
    if (s.parts == nullptr && s.first == nullptr) return;
    __shared__ float shared[kVectors][N][3][64];
    if (wave != 0) {
#pragma unroll
        for (int k = 0; k < kVectors; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) shared[k][i][wave - 1][lane] = sum[k][i];
    }
    __syncthreads();
    if (wave != 0 || valid == 0) return;
#pragma unroll
    for (int k = 0; k < kVectors; ++k) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int w = 0; w < 3; ++w) sum[k][i] += shared[k][i][w][lane];
        if (s.parts == nullptr) store_only((k == 0 ? s.first : s.second) + col, s.accumulate, sum[k], [&](int i) { return i < valid; });
        else memcpy(s.parts + ((uint64_t)part * kVectors + k) * s.pitch + col, sum[k], sizeof sum[k]);
    }
}

// The parts' sums: 32 neighbouring columns (a line) to a workgroup, eight lanes with four columns each, and 128 threads to them that take the parts in turn, whose sums are then added two by two.  Bound by latency: 512 parts of 4096 columns, two vectors, about 5 us, a launch of which is 2.
__global__ __launch_bounds__(1024) void add_vectors_kernel(const float* parts, uint32_t number, uint32_t cols, uint32_t pitch, uint32_t vectors, uint32_t blocks, float* first,
                                                         float* second, bool accumulate)
{
    constexpr uint32_t kTurns = 128;
    __shared__ f32x4 shared[kTurns / 2][8];
    const uint32_t lane = threadIdx.x & 7, turn = threadIdx.x >> 3, vector = this_block() / blocks, col = (this_block() % blocks * 8 + lane) * 4;
    if (vector >= vectors) return;
    f32x4 v = {};
    if (col < cols) {
        const float* from = parts + (uint64_t)vector * pitch + col;
#pragma unroll 8
        for (uint32_t n = turn; n < number; n += kTurns) {
            f32x4 t;
            memcpy(&t, from + (uint64_t)n * vectors * pitch, sizeof t);
            v += t;
        }
    }
    for (uint32_t half = kTurns / 2; half != 0; half /= 2) {
        if (turn >= half && turn < 2 * half) shared[turn - half][lane] = v;
        __syncthreads();
        if (turn < half) v += shared[turn][lane];
        __syncthreads();
    }
    if (turn != 0 || col >= cols) return;
    float* out = (vector == 0 ? first : second) + col;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (col + i < cols) out[i] = accumulate ? out[i] + v[i] : v[i];
}

// Sums over no rows.
__global__ __launch_bounds__(kBlock) void zero_kernel(float* first, float* second, uint32_t cols)
{
    const uint32_t col = blockIdx.x * kBlock + threadIdx.x;
    if (col >= cols) return;
    first[col] = 0.0f;
    if (second != nullptr) second[col] = 0.0f;
}

uint32_t pitch_of(size_t cols) { return (uint32_t)((cols + 7) / 8 * 8); }

// Threads to a row and pieces to a thread.
struct RowShape {
    uint32_t threads, pieces;  // 0: a row that is longer than the registers or shorter than a piece
};

RowShape shape_of(size_t cols, uint32_t dtype, uint32_t most_pieces)
{
    const uint32_t piece = dtype == OGQ_FP32 ? 4 : 8;
    const uint64_t pieces = ceil_div(cols, piece);
    if (cols < piece) return {0, 0};
    for (const uint32_t threads : {64u, 256u, 1024u})
        for (uint32_t p = 1; p <= most_pieces; p *= 2)
            if (pieces <= threads * p) return {threads, p};
    return {0, 0};
}

// Rows of a workgroup of the backward pass, whose sums go to the workspace.
struct Cut {
    uint32_t part, parts;
};

Cut rows_cut(size_t rows, uint32_t most, uint32_t multiple)
{
    const uint32_t part = (uint32_t)(ceil_div(ceil_div(rows, most), multiple) * multiple);
    return {part, (uint32_t)ceil_div(rows, part)};
}

// bf16, 256 and 512 parts: 8192 x 4096 52.3 us and 42.3 (768 parts 42.4), 2048 x 4096 19.8 and 20.2; of rows that take all of a CU's threads 4096 x 8192 40.1 and 46.2.
Cut backward_cut(size_t rows, const RowShape& shape) { return rows_cut(rows, shape.threads == 1024 ? 256 : 512, shape.threads == 64 ? 4 : 1); }

// Columns' blocks and rows' parts of columns_kernel.
Cut columns_cut(size_t rows, size_t cols, uint32_t dtype)
{
    const uint64_t blocks = ceil_div(cols, dtype == OGQ_FP32 ? 256 : 512), most = blocks < 1024 ? 1024 / blocks : 1;
    return rows_cut(rows, (uint32_t)most, 16);
}

template <class T, Columns WHAT>
void launch_columns(const Values& dy, const Values& x, const RowParts& s, const Cut& cut, const float* weight, const float* mean, const float* rstd, const RowMeans* means, uint32_t act,
                    const Result& dz, hipStream_t st)
{
    const uint32_t blocks = (uint32_t)ceil_div(s.cols, 64 * kPiece<T>);
    launch_kernel(columns_kernel<T, WHAT>, grid_of((uint64_t)blocks * cut.parts), dim3(kBlock), st, static_cast<const T*>(dy.data), dy.stride,
                  static_cast<const T*>(x.data), x.stride, s, blocks, weight, mean, rstd, means, act, static_cast<T*>(dz.data), dz.stride);
}

}  // namespace

void launch_add_vectors(const float* parts, uint32_t number, size_t cols, size_t pitch, float* first, float* second, bool accumulate, hipStream_t st)
{
    const uint32_t blocks = (uint32_t)ceil_div(cols, 32), vectors = second != nullptr ? 2 : 1;
    launch_kernel(add_vectors_kernel, grid_of((uint64_t)blocks * vectors), dim3(1024), st, parts, number, (uint32_t)cols, (uint32_t)pitch, vectors, blocks, first, second, accumulate);
}

void launch_layer_norm_forward(const Values& x, size_t rows, size_t cols, uint32_t dtype, const float* weight, const float* bias, float eps, const Result& y, float* mean,
                               float* rstd, hipStream_t st)
{
    const RowShape shape = shape_of(cols, dtype, 4);
    const float per_col = (float)(1.0 / (double)cols);
    with_type(dtype, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        auto kernel = layer_norm_forward_long_kernel<T>;
        uint64_t blocks = rows;
        uint32_t threads = 1024;
        const auto pick = [&](auto n) {
            constexpr int kThreads = decltype(n)::value;
            if (shape.threads != kThreads) return;
            kernel = shape.pieces == 2 ? layer_norm_forward_kernel<T, kThreads, 2> : layer_norm_forward_kernel<T, kThreads, 4>;
            if constexpr (kThreads == 64)  // (more threads have one piece each only where fewer have four)
                if (shape.pieces == 1) kernel = layer_norm_forward_kernel<T, kThreads, 1>;
            threads = block_of(kThreads);
            if (kThreads == 64) blocks = ceil_div(rows, 4);
        };
        pick(std::integral_constant<int, 64>{}), pick(std::integral_constant<int, 256>{}), pick(std::integral_constant<int, 1024>{});
        launch_kernel(kernel, grid_of(blocks), dim3(threads), st, static_cast<const T*>(x.data), x.stride, (uint32_t)rows, (uint32_t)cols, weight, bias, eps, per_col,
                      static_cast<T*>(y.data), y.stride, mean, rstd);
    });
}

// The workspace of a norm's sums: the parts' and, behind them, the means of rows that no workgroup holds whole.
size_t parts_bytes(const Cut& cut, size_t cols) { return cut.parts > 1 ? (size_t)cut.parts * 2 * pitch_of(cols) * sizeof(float) : 0; }

size_t layer_norm_backward_workspace(size_t rows, size_t cols, uint32_t dtype)
{
    const RowShape shape = shape_of(cols, dtype, 2);
    const Cut cut = shape.threads != 0 ? backward_cut(rows, shape) : columns_cut(rows, cols, dtype);
    return parts_bytes(cut, cols) + (shape.threads != 0 ? 0 : rows * sizeof(RowMeans));
}

// The sums of a call's parts: to the workspace, and from there added up, or those of the only part straight to where they belong.
RowParts parts_of(size_t rows, size_t cols, const Cut& cut, float per_col, void* workspace, float* first, float* second, bool accumulate)
{
    return {(uint32_t)rows, (uint32_t)cols, cut.part, pitch_of(cols), per_col, first != nullptr && cut.parts > 1 ? static_cast<float*>(workspace) : nullptr, first, second, accumulate};
}

void launch_layer_norm_backward(const Values& dy, const Values& x, size_t rows, size_t cols, uint32_t dtype, const float* weight, const float* mean, const float* rstd,
                                const Result& dx, float* dweight, float* dbias, bool accumulate, void* workspace, hipStream_t st)
{
    if (rows == 0) {
        launch_kernel(zero_kernel, dim3((uint32_t)ceil_div(cols, kBlock)), dim3(kBlock), st, dweight, dbias, (uint32_t)cols);
        return;
    }
    const RowShape shape = shape_of(cols, dtype, 2);
    const float per_col = (float)(1.0 / (double)cols);
    const Cut cut = shape.threads != 0 ? backward_cut(rows, shape) : columns_cut(rows, cols, dtype);
    const RowParts s = parts_of(rows, cols, cut, per_col, workspace, dweight, dbias, accumulate);
    with_type(dtype, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        if (shape.threads == 0) {
            RowMeans* means = dweight != nullptr ? reinterpret_cast<RowMeans*>(static_cast<char*>(workspace) + parts_bytes(cut, cols)) : nullptr;
            launch_kernel(layer_norm_backward_long_kernel<T>, grid_of(rows), dim3(1024), st, static_cast<const T*>(dy.data), dy.stride, static_cast<const T*>(x.data),
                          x.stride, (uint32_t)rows, (uint32_t)cols, per_col, weight, mean, rstd, static_cast<T*>(dx.data), dx.stride, means);
            if (means != nullptr) launch_columns<T, Columns::kNorm>(dy, x, s, cut, weight, mean, rstd, means, 0, dx, st);
            return;
        }
        const auto pick = [&](auto n) {
            constexpr int kThreads = decltype(n)::value;
            if (shape.threads != kThreads) return;
            const auto kernel = shape.pieces == 1 ? layer_norm_backward_kernel<T, kThreads, 1> : layer_norm_backward_kernel<T, kThreads, 2>;
            launch_kernel(kernel, grid_of(cut.parts), dim3(block_of(kThreads)), st, static_cast<const T*>(dy.data), dy.stride, static_cast<const T*>(x.data), x.stride, s,
                          weight, mean, rstd, static_cast<T*>(dx.data), dx.stride);
        };
        pick(std::integral_constant<int, 64>{}), pick(std::integral_constant<int, 256>{}), pick(std::integral_constant<int, 1024>{});
    });
    if (s.parts != nullptr) launch_add_vectors(s.parts, cut.parts, cols, s.pitch, dweight, dbias, accumulate, st);
}

size_t linear_backward_workspace(size_t tokens, size_t outs, uint32_t dtype)
{
    const uint32_t parts = columns_cut(tokens, outs, dtype).parts;
    return parts > 1 ? (size_t)parts * pitch_of(outs) * sizeof(float) : 0;
}

void launch_linear_backward(const Values& dy, size_t tokens, size_t outs, uint32_t dtype, uint32_t act, const Values& before, const Result& dz, float* dbias, bool accumulate,
                            void* workspace, hipStream_t st)
{
    if (tokens == 0) {
        launch_kernel(zero_kernel, dim3((uint32_t)ceil_div(outs, kBlock)), dim3(kBlock), st, dbias, static_cast<float*>(nullptr), (uint32_t)outs);
        return;
    }
    const Cut cut = columns_cut(tokens, outs, dtype);
    const RowParts s = parts_of(tokens, outs, cut, 0.0f, workspace, dbias, nullptr, accumulate);
    with_type(dtype, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        if (act == OGQ_IDENTITY) launch_columns<T, Columns::kSums>(dy, before, s, cut, nullptr, nullptr, nullptr, nullptr, act, dz, st);
        else launch_columns<T, Columns::kActivation>(dy, before, s, cut, nullptr, nullptr, nullptr, nullptr, act, dz, st);
    });
    if (s.parts != nullptr) launch_add_vectors(s.parts, cut.parts, outs, s.pitch, dbias, nullptr, accumulate, st);
}

}  // namespace ogq
