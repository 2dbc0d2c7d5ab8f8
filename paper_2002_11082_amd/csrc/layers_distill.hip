// libogq_layers: the divergence of a row's distribution from a teacher's, known at a few places, and its gradient.
//
// One workgroup (or wavefront) to a row, which it reads once: largest logit, sum of exponentials and the gradient come from registers.  Bound by memory; rows too long for
// the registers are read again, from the caches.
#include "layers_common.h"

namespace ogq {

namespace {

struct Distill {
    uint32_t rows, cols, top;
    bool wide;                      // places are of 64 bits
    float per_temperature, temperature;
    uint64_t stride, out_stride;
    const void* places;
    const float *values, *row_weight;
    float* loss;
};

// exp(x - most), x and most over the temperature: in fp32 to a few roundings of 32 bits, for 16-bit results to 2^-19 of it.
template <class T>
__device__ __forceinline__ float exp_below(float x, float most)
{
    if constexpr (sizeof(T) == 4) {
        const float d = x - most;
        // (-infinity has no fraction, NaN none either: the instruction takes both)
        return d < -200.0f ? 0.0f : exp_of(d, 0.0f);
    } else {
        return __builtin_amdgcn_exp2f((x - most) * kLog2e);
    }
}

// A workgroup of THREADS to a row, P pieces to each, or P = 0: the row, of any length, is read for each of its passes.  The teacher's places are shared out over the threads, and are in
// LDS for the places that are the same.
template <class T, int THREADS, int P, bool GRADIENT>
__global__ __launch_bounds__(THREADS) void distill_kernel(const T* logits, Distill s, T* dlogits)
{
    constexpr int N = kPiece<T>, kWaves = THREADS / 64, kMostTop = 1024, kSlots = kMostTop / THREADS, kHeld = P == 0 ? 1 : P;
    __shared__ float2 space[2][kWaves];
    // a row's places and what the teacher has there: exp(value - largest)
    __shared__ uint32_t place_of[GRADIENT ? kMostTop : 1];
    __shared__ float weight_of[GRADIENT ? kMostTop : 1];
    BlockSums<kWaves> sums{space};
    const uint32_t thread = threadIdx.x;
    const uint64_t row = this_block();
    if (row >= s.rows) return;
    const T* from = logits + row * s.stride;
    T* to = GRADIENT ? dlogits + row * s.out_stride : nullptr;
    const float row_weight = s.row_weight == nullptr ? 1.0f : s.row_weight[row];
    uint4 held[kHeld];
    // f(values, i -> whether value i counts) for all pieces of the thread, which it may change; STORE: and they go to the gradient
    const auto each_piece = [&](auto store, auto f) __attribute__((always_inline)) {
        float v[N];
        if constexpr (P != 0) {
            uint32_t t = thread;  // (places are made again too)
#pragma unroll
            for (int p = 0; p < P; ++p) {
                asm volatile("" : "+v"(t));
                // (the values are made again from what is held, piece after piece: otherwise the compiler keeps them from one pass to the next, in registers that there are not)
                asm volatile("" : "+v"(held[p].x), "+v"(held[p].y), "+v"(held[p].z), "+v"(held[p].w));
                const PieceAt<T> at = piece_at<T, THREADS, P>(p, t, s.cols);
                values_of<T>(held[p], v);
                f(v, [&](int i) { return at.counts(i); });
                if constexpr (decltype(store)::value)
                    if (at.there) store_piece<false>(to + at.col, N, v);
            }
        } else {
            for (uint32_t col = thread * N; col < s.cols; col += THREADS * N) {
                const int valid = valid_of<T>(col, s.cols);
                load_piece<false>(from + col, valid, v);
                f(v, [&](int i) { return i < valid; });
                if constexpr (decltype(store)::value) store_piece<false>(to + col, valid, v);
            }
        }
    };
    constexpr std::true_type kStore{};
    constexpr std::false_type kOnly{};
    const auto finish_without = [&]() __attribute__((always_inline)) {
        if (thread == 0 && s.loss != nullptr) s.loss[row] = 0.0f;
        if constexpr (GRADIENT) {
            float v[N] = {};
            for (uint32_t col = thread * N; col < s.cols; col += THREADS * N) store_piece<false>(to + col, valid_of<T>(col, s.cols), v);
        }
    };
    if (row_weight == 0.0f) {
        finish_without();
        return;
    }
    if constexpr (P != 0) {
#pragma unroll
        for (int p = 0; p < P; ++p) held[p] = load_whole(from + piece_at<T, THREADS, P>(p, thread, s.cols).col);
    }
    // The teacher's places of this thread, their values and the student's logits there.
    uint32_t place[kSlots];
    float value[kSlots], logit[kSlots];
    float most_value = -INFINITY, most = -INFINITY;
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
        const uint32_t slot = k * THREADS + thread;
        place[k] = 0xFFFFFFFFu, value[k] = -INFINITY, logit[k] = 0.0f;
        if (slot < s.top) {
            const uint64_t at = row * s.top + slot;
            const int64_t c = s.wide ? static_cast<const int64_t*>(s.places)[at] : (int64_t)static_cast<const int32_t*>(s.places)[at];
            if (c >= 0 && c < (int64_t)s.cols) {
                place[k] = (uint32_t)c;
                value[k] = s.values[at] * s.per_temperature;
                logit[k] = (float)from[c] * s.per_temperature;
                most_value = fmaxf(most_value, value[k]);
            }
        }
    }
    each_piece(kOnly, [&](const float(&v)[N], auto counts) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < N; ++i) most = fmaxf(most, P != 0 || counts(i) ? v[i] : -INFINITY);  // (twice is no harm)
    });
    {
        const float2 t = sums.largest(most * s.per_temperature, most_value);
        most = t.x, most_value = t.y;
    }
    float total = 0.0f, teacher = 0.0f;
    each_piece(kOnly, [&](const float(&v)[N], auto counts) __attribute__((always_inline)) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) t += counts(i) ? exp_below<T>(v[i] * s.per_temperature, most) : 0.0f;
        total += t;
    });
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
        const bool there = place[k] != 0xFFFFFFFFu;
        // (the largest of values that are all -infinity or NaN is -infinity: of the first the row has none, the second are NaN)
        value[k] = there && value[k] != -INFINITY ? value[k] - most_value : -INFINITY;
        const float e = there ? exp_below<float>(value[k], 0.0f) : 0.0f;
        teacher += e;
        if constexpr (GRADIENT) {
            const uint32_t slot = k * THREADS + thread;
            if (slot < s.top) place_of[slot] = place[k], weight_of[slot] = e;
        }
    }
    {
        const float2 t = sums(total, teacher);
        total = t.x, teacher = t.y;
    }
    if (teacher == 0.0f) {  // no place, or none with a value
        finish_without();
        return;
    }
    const float per_teacher = 1.0f / teacher, log_teacher = logf(teacher), log_total = logf(total);
    float divergence = 0.0f;
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
        const float p = place[k] != 0xFFFFFFFFu ? exp_below<float>(value[k], 0.0f) * per_teacher : 0.0f;
        // (not equal to 0: a NaN stays)
        if (p != 0.0f) divergence += p * ((value[k] - log_teacher) - ((logit[k] - most) - log_total));
    }
    const float2 sum = sums(divergence, 0.0f);
    if (thread == 0 && s.loss != nullptr) s.loss[row] = row_weight * s.temperature * s.temperature * sum.x;
    if constexpr (GRADIENT) {
        // (a NaN of the teacher's is everywhere, one of the student's is in `total`)
        const float factor = row_weight * s.temperature, per_total = 1.0f / total, scale = factor * per_total, none = teacher != teacher ? teacher : 0.0f;
        each_piece(kStore, [&](float(&v)[N], auto) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = exp_below<T>(v[i] * s.per_temperature, most) * scale + none;
        });
        // Behind the row's other values: the places, each with the shares of all that are the same.
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kSlots; ++k) {
            if (place[k] == 0xFFFFFFFFu) continue;
            float p = 0.0f;
            for (uint32_t n = 0; n < s.top; ++n) p += place_of[n] == place[k] ? weight_of[n] : 0.0f;
            to[place[k]] = (T)(factor * (exp_below<T>(logit[k], most) * per_total - p * per_teacher));
        }
    }
}

// Threads to a row and pieces to a thread; no pieces: more than the registers hold, or less than a piece.
struct RowShape {
    int threads, pieces;
};

RowShape shape_of(size_t cols, uint32_t dtype)
{
    const uint32_t piece = dtype == OGQ_FP32 ? 4 : 8;
    const uint64_t pieces = ceil_div(cols, piece);
    for (const int threads : {256, 1024})
        for (int p = 1; p <= (threads == 1024 ? 16 : 4); p *= 2)
            if (cols >= piece && pieces <= (uint64_t)threads * p) return {threads, p};
    return {1024, 0};
}

template <class T, bool GRADIENT, int THREADS>
auto kernel_of(int pieces)
{
    if constexpr (THREADS == 256) {
        return pieces == 1 ? distill_kernel<T, 256, 1, GRADIENT> : pieces == 2 ? distill_kernel<T, 256, 2, GRADIENT> : distill_kernel<T, 256, 4, GRADIENT>;
    } else {
        return pieces == 2   ? distill_kernel<T, 1024, 2, GRADIENT>
               : pieces == 4 ? distill_kernel<T, 1024, 4, GRADIENT>
               : pieces == 8 ? distill_kernel<T, 1024, 8, GRADIENT>
               : pieces == 16 ? distill_kernel<T, 1024, 16, GRADIENT>
                              : distill_kernel<T, 1024, 0, GRADIENT>;
    }
}

}  // namespace

void launch_distill(const Values& logits, size_t rows, size_t cols, uint32_t dtype, const Integers& places, const float* values, size_t top, float temperature,
                    const float* row_weight, float* loss, const Result& dlogits, hipStream_t st)
{
    const Distill s{(uint32_t)rows, (uint32_t)cols, (uint32_t)top, places.type == OGQ_INT64, 1.0f / temperature, temperature, logits.stride, dlogits.stride,
                    places.data,    values,         row_weight,    loss};
    const RowShape shape = shape_of(cols, dtype);
    with_type(dtype, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const auto go = [&](auto gradient) {
            constexpr bool kGradient = decltype(gradient)::value;
            const auto kernel = shape.threads == 256 ? kernel_of<T, kGradient, 256>(shape.pieces) : kernel_of<T, kGradient, 1024>(shape.pieces);
            launch_kernel(kernel, grid_of(rows), dim3(shape.threads), st, static_cast<const T*>(logits.data), s, static_cast<T*>(dlogits.data));
        };
        if (dlogits.data != nullptr) go(std::true_type{});
        else go(std::false_type{});
    });
}

}  // namespace ogq
