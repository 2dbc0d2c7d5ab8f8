// libogq_layers: products of tokens with a layer's weights on the matrix cores, y[t][o] = sum over k of x[t][k] * W[o][k], or of x[t][k] * W[k][o], with what happens to the sums on
// their way out.
//
// A workgroup holds a tile of sums in registers and goes along k in steps.  Values go to LDS in the pieces that the matrix cores take: as they are in 16 bits, fp32 in three pieces of
// bf16.  Rows along k (x, and W as it is) are read back as they lie, eight values of k to a lane; rows across k (W transposed) come back transposed (ds_read_b64_tr_b16: 16
// lanes read four rows of 16 values and receive four values of one column each).  The weights are the instruction's first factor, so that a lane holds four neighbouring outputs of a token.
#include "layers_linear.h"

namespace ogq {

namespace {

typedef short s16x8 __attribute__((ext_vector_type(8)));

template <class T>
constexpr int kPlanes = sizeof(T) == 4 ? 3 : 1;
// Values of k in a step: 128 bytes of a row in 16 bits, whole lines of memory, and in fp32.
template <class T>
constexpr int kDepth = sizeof(T) == 4 ? 32 : 64;

// Eight values of a row in the pieces that the matrix cores take.
template <class T>
struct Chunk {
    uint32_t raw[2 * sizeof(T)];
    __device__ __forceinline__ void load(const T* from) { memcpy(raw, from, sizeof raw); }
    __device__ __forceinline__ void load(const T* from, int valid)
    {
        if (valid >= 8) load(from);
        else load_some<T, 8>(from, valid, raw);
    }
    __device__ __forceinline__ void store(char* to, int plane) const
    {
        if constexpr (sizeof(T) == 2) {
            memcpy(__builtin_assume_aligned(to, 16), raw, 16);
        } else {
            uint32_t w[3][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t a[3], b[3];
                split3(__uint_as_float(raw[2 * i]), a[0], a[1], a[2]);
                split3(__uint_as_float(raw[2 * i + 1]), b[0], b[1], b[2]);
#pragma unroll
                for (int p = 0; p < 3; ++p) w[p][i] = __builtin_amdgcn_perm(b[p], a[p], 0x07060302u);  // the upper halves
            }
#pragma unroll
            for (int p = 0; p < 3; ++p) memcpy(__builtin_assume_aligned(to + p * plane, 16), w[p], 16);
        }
    }
};

// ROWS rows along k of a factor: a step of each is a row in LDS, chunk c of row r at place(r, c), so that sixteen lanes that read chunk c of sixteen rows meet all banks.
template <class T, int ROWS, int THREADS = 256>
struct Along {
    static constexpr int kChunks = kDepth<T> / 8, kRowBytes = kDepth<T> * 2, kPlane = ROWS * kRowBytes, kUnits = ROWS * kChunks / THREADS, kUnitRows = THREADS / kChunks;
    static_assert(kUnits * THREADS == ROWS * kChunks);
    const T* rows[kUnits];
    uint32_t last, mine;
    char* to;
    Chunk<T> held[kUnits];

    static __device__ __forceinline__ uint32_t place(uint32_t row, uint32_t chunk) { return row * kRowBytes + ((chunk ^ (row / (256 / kRowBytes) & (kChunks - 1))) * 16); }

    // Rows `first` ... of `number`; what lies behind the last row is any row that is there: its sums are not stored.
    __device__ __forceinline__ Along(const T* data, uint64_t stride, uint32_t first, uint32_t number, uint32_t last_, uint32_t thread, char* lds) : last(last_)
    {
        const uint32_t row = thread / kChunks, chunk = thread % kChunks;
        mine = chunk * 8;
#pragma unroll
        for (int u = 0; u < kUnits; ++u) rows[u] = data + (uint64_t)min(first + row + u * kUnitRows, number - 1) * stride + mine;
        static_assert(kUnitRows % 16 == 0);  // (then place moves the chunks of all of a thread's rows alike)
        to = lds + place(row, chunk);
    }
    __device__ __forceinline__ void fetch(uint32_t k)
    {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) held[u].load(rows[u] + k);
    }
    __device__ __forceinline__ void fetch_asking(uint32_t k)
    {
        const int valid = k + mine >= last ? 0 : (int)min(8u, last - k - mine);
#pragma unroll
        for (int u = 0; u < kUnits; ++u) held[u].load(rows[u] + k, valid);
    }
    __device__ __forceinline__ void bring(uint32_t stage_bytes)
    {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) held[u].store(to + stage_bytes + u * kUnitRows * kRowBytes, kPlane);
    }
    // Where a lane finds its part of an operand: 32 rows from `row`, k = 16 h + lane / 32 * 8 ...
    static __device__ __forceinline__ s16x8 read(const char* plane, uint32_t row, int h, uint32_t lane)
    {
        return *reinterpret_cast<const s16x8*>(plane + place(row + (lane & 31), 2 * h + (lane >> 5)));
    }
};

// The same for rows across k: a step is kDepth rows of COLS values, of which the columns are the operand's rows.  Chunk c (32 bytes) of row k lies at c ^ twist(k).
template <class T, int COLS, int THREADS = 256>
struct Across {
    static constexpr int kChunks = COLS / 16, kRowBytes = COLS * 2, kPlane = kDepth<T> * kRowBytes, kUnits = kDepth<T> * kChunks / THREADS, kUnitRows = THREADS / kChunks;
    static_assert(kUnits * THREADS == kDepth<T> * kChunks && kUnitRows % 4 == 0);
    const T* data;
    uint64_t stride;
    uint32_t last, row, mine;
    int valid;
    char* to;
    Chunk<T> held[kUnits][2];

    static __device__ __forceinline__ uint32_t twist(uint32_t k) { return (k & (kChunks >= 8 ? 3u : 1u)) * 2u; }

    // Columns `first` ... of `number`; what lies behind the last one is 0.
    __device__ __forceinline__ Across(const T* data_, uint64_t stride_, uint32_t first, uint32_t number, uint32_t last_, uint32_t thread, char* lds)
        : data(data_), stride(stride_), last(last_)
    {
        const uint32_t chunk = thread % kChunks;
        row = thread / kChunks;
        mine = first + chunk * 16;
        valid = mine >= number ? 0 : (int)min(16u, number - mine);
        to = lds + row * kRowBytes + ((chunk ^ twist(row)) * 32);
    }
    __device__ __forceinline__ void load(int u, uint32_t k)
    {
        const T* from = data + (uint64_t)k * stride + mine;
        held[u][0].load(from, valid);
        held[u][1].load(from + 8, valid - 8);
    }
    __device__ __forceinline__ void fetch(uint32_t k)
    {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) load(u, k + row + u * kUnitRows);
    }
    __device__ __forceinline__ void fetch_asking(uint32_t k)
    {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const uint32_t at = k + row + u * kUnitRows;
            if (at < last) {
                load(u, at);
            } else {
#pragma unroll
                for (int i = 0; i < (int)(2 * sizeof(T)); ++i) held[u][0].raw[i] = held[u][1].raw[i] = 0;
            }
        }
    }
    __device__ __forceinline__ void bring(uint32_t stage_bytes)
    {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            held[u][0].store(to + stage_bytes + u * kUnitRows * kRowBytes, kPlane);
            held[u][1].store(to + stage_bytes + u * kUnitRows * kRowBytes + 16, kPlane);
        }
    }
    static __device__ __forceinline__ s16x8 read(const char* plane, uint32_t col, int h, uint32_t lane)
    {
        typedef __attribute__((address_space(3))) s16x4* Lds;
        const uint32_t k = (lane >> 5) * 8 + ((lane >> 2) & 3), chunk = col / 16 + ((lane >> 4) & 1);
        const char* at = plane + (h * 16 + k) * kRowBytes + ((chunk ^ twist(k)) * 32) + (lane & 3) * 8;
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)at), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + 4 * kRowBytes));
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

template <class T>
__device__ __forceinline__ f32x16 multiply_add(s16x8 a, s16x8 b, f32x16 c)
{
    if constexpr (__is_same(T, _Float16)) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ void wavefront_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The sums of a wavefront, 32 * NO outputs from `out` and 32 * NT tokens from `token`, on their way out.  A lane holds pieces of 16 bytes of 32 tokens; through LDS (`space`, kTurn<NO>
// bytes of the wavefront's own) neighbouring lanes get neighbouring pieces of one token, so that lines are written whole.
template <int NO>
constexpr int kTurnRow = NO * 128 + 16;  // (16 bytes between rows: eight rows' pieces in different banks)
template <int NO>
constexpr int kTurn = 32 * kTurnRow<NO>;

template <class T, int NO, int NT>
__device__ __forceinline__ void finish_tile(const f32x16 (&sum)[NO][NT], uint32_t out, uint32_t token, uint32_t lane, const LinearShape& s, uint32_t part, const Epilogue<T>& e,
                                            char* space)
{
    constexpr int N = kPiece<T>, kPieces = NO * 32 / N;
#pragma unroll
    for (int b = 0; b < NT; ++b) {
#pragma unroll
        for (int a = 0; a < NO; ++a)
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const f32x4 v = {sum[a][b][4 * m], sum[a][b][4 * m + 1], sum[a][b][4 * m + 2], sum[a][b][4 * m + 3]};
                *reinterpret_cast<f32x4*>(space + (lane & 31) * kTurnRow<NO> + a * 128 + 32 * m + (lane >> 5) * 16) = v;
            }
        wavefront_sync();
#pragma unroll 1
        for (int i = 0; i < 32 * kPieces / 64; ++i) {
            const uint32_t row = (i * 64 + lane) / kPieces, piece = (i * 64 + lane) % kPieces, t = token + 32 * b + row, o = out + piece * N;
            float v[N];
            memcpy(v, __builtin_assume_aligned(space + row * kTurnRow<NO> + piece * N * 4, 16), sizeof v);
            const int valid = valid_of<T>(o, s.outs);
            if (t >= s.tokens || valid == 0) continue;
            if (s.sums == nullptr) e(t, o, valid, v);
            else memcpy(s.sums + ((uint64_t)part * s.tokens + t) * s.pitch + o, v, sizeof v);
        }
        wavefront_sync();
    }
}

// fp32: an infinity is its first piece alone, and its products with pieces that are 0 are NaN.  Sums that are NaN are made again, one product after the other: few, or those of a program that
// has gone wrong already.
template <bool TRANSPOSED, int NO, int NT>
__device__ __forceinline__ void mend_sums(const float* x, const float* weight, const LinearShape& s, uint32_t out, uint32_t token, uint32_t first, uint32_t last, uint32_t lane,
                                          f32x16 (&sum)[NO][NT])
{
    bool any = false;
#pragma unroll
    for (int a = 0; a < NO; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) any |= sum[a][b][i] != sum[a][b][i];
    if (__builtin_amdgcn_ballot_w64(any) == 0) return;
#pragma unroll
    for (int a = 0; a < NO; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            const uint32_t t = token + 32 * b + (lane & 31);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t o = out + 32 * a + 8 * (i / 4) + 4 * (lane >> 5) + i % 4;
                if (sum[a][b][i] == sum[a][b][i] || t >= s.tokens || o >= s.outs) continue;
                float v = 0.0f;
#pragma unroll 1
                for (uint32_t k = first; k < last; ++k)
                    v = __builtin_fmaf(x[t * s.x_stride + k], TRANSPOSED ? weight[k * s.weight_stride + o] : weight[o * s.weight_stride + k], v);
                sum[a][b][i] = v;
            }
        }
}

// The pairs of pieces whose products count: all but those below 2^-24 of the largest.
template <class T, class F>
__device__ __forceinline__ void each_pair(F f)
{
    if constexpr (kPlanes<T> == 1) {
        f(0, 0);
    } else {
        f(2, 0), f(0, 2), f(1, 1), f(1, 0), f(0, 1), f(0, 0);
    }
}

// Tiles of OUT outputs by TOKENS tokens, a quarter in each of four wavefronts.
template <class T, int OUT, int TOKENS, bool TRANSPOSED>
__global__ __launch_bounds__(256) void linear_kernel(const T* x, const T* weight, LinearShape s, Epilogue<T> e)
{
    using FeedW = std::conditional_t<TRANSPOSED, Across<T, OUT>, Along<T, OUT>>;
    using FeedX = Along<T, TOKENS>;
    constexpr int kBytesW = kPlanes<T> * FeedW::kPlane, kStage = kBytesW + kPlanes<T> * FeedX::kPlane, NO = OUT / 64, NT = TOKENS / 64;
    constexpr int kBytes = kStage > 4 * kTurn<NO> ? kStage : 4 * kTurn<NO>;
    __shared__ __align__(16) char lds[kBytes];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t tiles = s.tiles_out * s.tiles_token, tile = blockIdx.x % tiles, part = blockIdx.x / tiles;
    const uint32_t out = tile % s.tiles_out * OUT, token = tile / s.tiles_out * TOKENS, out_wave = (wave & 1) * (OUT / 2), token_wave = (wave >> 1) * (TOKENS / 2);
    const uint32_t first = part * s.part, last = min(s.cols, first + s.part);
    FeedW feed_w(weight, s.weight_stride, out, s.outs, last, threadIdx.x, lds);
    FeedX feed_x(x, s.x_stride, token, s.tokens, last, threadIdx.x, lds + kBytesW);
    f32x16 sum[NO][NT] = {};
    const auto fetch = [&](uint32_t k) __attribute__((always_inline)) {
        if (k + kDepth<T> <= last) {
            feed_w.fetch(k);
            feed_x.fetch(k);
        } else if (k < last) {
            feed_w.fetch_asking(k);
            feed_x.fetch_asking(k);
        }
    };
    fetch(first);
    for (uint32_t k = first; k < last; k += kDepth<T>) {
        __syncthreads();
        feed_w.bring(0);
        feed_x.bring(0);
        __syncthreads();
        fetch(k + kDepth<T>);
#pragma unroll
        for (int h = 0; h < kDepth<T> / 16; ++h)
            each_pair<T>([&](int p, int q) __attribute__((always_inline)) {
                s16x8 a[NO], b[NT];
#pragma unroll
                for (int i = 0; i < NO; ++i) a[i] = FeedW::read(lds + p * FeedW::kPlane, out_wave + 32 * i, h, lane);
#pragma unroll
                for (int j = 0; j < NT; ++j) b[j] = FeedX::read(lds + kBytesW + q * FeedX::kPlane, token_wave + 32 * j, h, lane);
#pragma unroll
                for (int i = 0; i < NO; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) sum[i][j] = multiply_add<T>(a[i], b[j], sum[i][j]);
            });
    }
    __syncthreads();
    if constexpr (sizeof(T) == 4) mend_sums<TRANSPOSED>(x, weight, s, out + out_wave, token + token_wave, first, last, lane, sum);
    finish_tile<T>(sum, out + out_wave, token + token_wave, lane, s, part, e, lds + wave * kTurn<NO>);
}

// The parts' sums of a piece of a token's outputs.
template <class T>
__global__ __launch_bounds__(kBlock) void join_parts_kernel(LinearShape s, Epilogue<T> e, uint32_t per_token)
{
    constexpr int N = kPiece<T>;
    const uint64_t piece = (uint64_t)block_number() * kBlock + threadIdx.x;
    const uint64_t token = piece / per_token;
    if (token >= s.tokens) return;
    const uint32_t out = (uint32_t)(piece % per_token) * N;
    float v[N] = {};
    const float* from = s.sums + token * s.pitch + out;
#pragma unroll 4
    for (uint32_t n = 0; n < s.parts; ++n) {
        float t[N];
        memcpy(t, __builtin_assume_aligned(from + (uint64_t)n * s.tokens * s.pitch, 16), sizeof t);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += t[i];
    }
    e(token, out, valid_of<T>(out, s.outs), v);
}

struct Plan {
    uint32_t tile_out, tile_token, tiles_out, tiles_token, part, parts;
};

Plan plan_of(size_t tokens, size_t outs, size_t cols, uint32_t dtype)
{
    Plan p;
    const uint32_t depth = dtype == OGQ_FP32 ? 32 : 64;
    p.tile_out = 128;
    p.tile_token = tokens <= 64 ? 64 : 128;
    p.tiles_out = (uint32_t)ceil_div(outs, p.tile_out), p.tiles_token = (uint32_t)ceil_div(tokens, p.tile_token);
    const uint64_t tiles = (uint64_t)p.tiles_out * p.tiles_token, steps = ceil_div(cols, depth);
    uint64_t parts = 1;
    if (tiles < 512) {
        parts = 512 / tiles;
        if (parts > steps / 4) parts = steps / 4;
        if (parts < 1) parts = 1;
    }
    p.part = steps == 0 ? depth : (uint32_t)(ceil_div(steps, parts) * depth);
    p.parts = steps == 0 ? 1 : (uint32_t)ceil_div(cols, p.part);
    return p;
}

uint32_t pitch_of(size_t outs) { return (uint32_t)(ceil_div(outs, 8) * 8); }

}  // namespace

template <class T>
void launch_join_parts(const LinearShape& s, const Epilogue<T>& e, hipStream_t st)
{
    const uint32_t per_token = (uint32_t)ceil_div(s.outs, kPiece<T>);
    launch_kernel(join_parts_kernel<T>, grid_of_blocks(ceil_div((uint64_t)s.tokens * per_token, kBlock)), dim3(kBlock), st, s, e, per_token);
}

template void launch_join_parts<float>(const LinearShape&, const Epilogue<float>&, hipStream_t);
template void launch_join_parts<__bf16>(const LinearShape&, const Epilogue<__bf16>&, hipStream_t);
template void launch_join_parts<_Float16>(const LinearShape&, const Epilogue<_Float16>&, hipStream_t);

size_t linear_workspace(size_t tokens, size_t outs, size_t cols, uint32_t dtype, bool transposed)
{
    const uint32_t parts = tokens <= kFewTokens ? few_plan(tokens, outs, cols, dtype, transposed).parts : plan_of(tokens, outs, cols, dtype).parts;
    return parts > 1 ? (size_t)parts * tokens * pitch_of(outs) * sizeof(float) : 0;
}

void launch_linear(const Values& x, const Values& weight, bool transposed, size_t tokens, size_t outs, size_t cols, uint32_t dtype, const float* bias, uint32_t act,
                   const Values& residual, const Result& y, const Result& before, void* workspace, hipStream_t st)
{
    LinearShape s{};
    s.tokens = (uint32_t)tokens, s.outs = (uint32_t)outs, s.cols = (uint32_t)cols, s.x_stride = x.stride, s.weight_stride = weight.stride, s.pitch = pitch_of(outs);
    with_type(dtype, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const Epilogue<T> e{bias,          static_cast<const T*>(residual.data), static_cast<T*>(y.data), static_cast<T*>(before.data), residual.stride, y.stride,
                            before.stride, s.outs,                               act};
        const auto from = static_cast<const T*>(x.data), w = static_cast<const T*>(weight.data);
        if (tokens <= kFewTokens) {
            const FewPlan plan = few_plan(tokens, outs, cols, dtype, transposed);
            s.tiles_out = (uint32_t)ceil_div(outs, 64 * kPiece<T>), s.part = plan.part, s.parts = plan.parts;
            s.sums = plan.parts > 1 ? static_cast<float*>(workspace) : nullptr;
            launch_few(plan, from, w, transposed, s, e, st);
            return;
        }
        const Plan plan = plan_of(tokens, outs, cols, dtype);
        s.tiles_out = plan.tiles_out, s.tiles_token = plan.tiles_token, s.part = plan.part, s.parts = plan.parts;
        s.sums = plan.parts > 1 ? static_cast<float*>(workspace) : nullptr;
        auto kernel = transposed ? linear_kernel<T, 128, 128, true> : linear_kernel<T, 128, 128, false>;
        if (plan.tile_token == 64) kernel = transposed ? linear_kernel<T, 128, 64, true> : linear_kernel<T, 128, 64, false>;
        launch_kernel(kernel, dim3(s.tiles_out * s.tiles_token * s.parts), dim3(256), st, from, w, s, e);
        if (s.sums != nullptr) launch_join_parts(s, e, st);
    });
}

}  // namespace ogq
