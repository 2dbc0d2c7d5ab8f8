// libogq_layers: the divergence of a row's distribution from a teacher's, known at a few places, and its gradient.
//
// One workgroup to a row, which it reads once: largest logit, sum of exponentials and the gradient come from registers.  Bound by memory, with the vector unit close behind (an exponential twice
// for each logit: keeping the first one's results would take the registers that the logits are in): 4096 x 32768 bf16 with its gradient 107 us, 5.0 TB/s, vector instructions issued in nearly all cycles.
// Rows too long for the registers are read again, from the caches.  61 x 131071 fp16, several workgroups to a row: 6.1 + 12.7 us, of which 6.6 are the bytes' and the rest two chains of latencies.
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
    uint32_t slices;                // of a row, where several workgroups share it
    float2* parts;                  // [rows][slices]: a slice's largest logit, as Below has it, and the sum of its exponentials
    float* logits_there;            // [rows][top]: the logits at the teacher's places
};

// exp(d) for d that are at most 0 but for a rounding.
__device__ __forceinline__ float exp_of_share(float d) { return d < -200.0f ? 0.0f : exp_of(d, 0.0f); }

// (x - most) / temperature for the logits x of a row, most being the largest, times 1 (fp32) or log2(e) (16 bits), and exp of it: in fp32 to a few roundings of 32 bits, for 16-bit results to 2^-17 of it.  The largest logit
// is held times the factor, `held`, rounded.  All differences, those of the loss too, are one rounding from that same number, so that its own rounding, which grows with an offset of the logits,
// is in none of the results: it cancels between a logit and the sum of exponentials.
template <class T>
struct Below {
    static constexpr bool kWide = sizeof(T) == 4;
    float factor, held;
    static __device__ __forceinline__ float factor_of(float per_temperature) { return kWide ? per_temperature : per_temperature * kLog2e; }
    __device__ __forceinline__ float difference(float x) const { return __builtin_fmaf(x, factor, -held); }
    // exp of a difference.  (-infinity has no fraction, NaN none either: the instruction takes both)
    static __device__ __forceinline__ float power(float d) { return kWide ? exp_of_share(d) : __builtin_amdgcn_exp2f(d); }
    __device__ __forceinline__ float exp(float x) const { return power(difference(x)); }
    __device__ __forceinline__ float natural(float x) const { return kWide ? difference(x) : difference(x) * 0.693147180559945f; }
};

// Place n of a row, -1 where it stands for none.
__device__ __forceinline__ int64_t place_at(const Distill& s, uint64_t n)
{
    const int64_t c = s.wide ? static_cast<const int64_t*>(s.places)[n] : (int64_t)static_cast<const int32_t*>(s.places)[n];
    return c >= 0 && c < (int64_t)s.cols ? c : -1;
}

// What a row's workgroup is to do.
//   kLoss      the loss
//   kGradient  the loss and the gradient
//   kPart      of rows that several workgroups share: largest logit and sum of exponentials of a slice; the first slice's also puts the logits at the teacher's places aside
//   kRest      and then the loss and, where it is wanted, a slice of the gradient
enum class Pass { kLoss, kGradient, kPart, kRest };

// A workgroup of THREADS to a row (or a slice of it), P pieces to each, or P = 0: the row, of any length, is read for each of its passes.  The teacher's places are shared out over the threads, and
// are in LDS for the places that are the same.
template <class T, int THREADS, int P, Pass PASS>
__global__ __launch_bounds__(THREADS) void distill_kernel(const T* logits, Distill s, T* dlogits)
{
    constexpr int N = kPiece<T>, kWaves = THREADS / 64, kMostTop = 1024, kSlots = kMostTop / THREADS, kHeld = P == 0 ? 1 : P;
    constexpr bool kSliced = PASS == Pass::kPart || PASS == Pass::kRest, kGradient = PASS == Pass::kGradient || PASS == Pass::kRest;
    static_assert(!kSliced || P != 0);
    __shared__ float2 space[2][kWaves];
    // a row's places and what the teacher has there: exp(value - largest)
    __shared__ __align__(16) uint32_t place_of[kGradient ? kMostTop : 1];
    __shared__ __align__(16) float weight_of[kGradient ? kMostTop : 1];
    BlockSums<kWaves> sums{space};
    const uint32_t thread = threadIdx.x;
    const uint64_t row = kSliced ? this_block() / s.slices : this_block();
    if (row >= s.rows) return;
    const uint32_t slice = kSliced ? (uint32_t)(this_block() - row * s.slices) : 0;
    if (PASS == Pass::kRest && dlogits == nullptr && slice != 0) return;
    // the slice's first column, and one behind its last
    const uint32_t first = slice * (uint32_t)(THREADS * P * N), last = kSliced ? min(s.cols, first + (uint32_t)(THREADS * P * N)) : s.cols;
    const T* from = logits + row * s.stride;
    T* to = kGradient ? dlogits + row * s.out_stride : nullptr;
    const float row_weight = s.row_weight == nullptr ? 1.0f : s.row_weight[row];
    const auto at = [&](int p, uint32_t t) __attribute__((always_inline)) {
        // (the last piece of the row's last slice ends with the row)
        if constexpr (kSliced) return PieceAt<T>(first + (p * THREADS + t) * N, s.cols);
        else return piece_at<T, THREADS, P == 0 ? 1 : P>(p, t, s.cols);
    };
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
                const PieceAt<T> piece = at(p, t);
                values_of<T>(held[p], v);
                f(v, [&](int i) { return piece.counts(i); });
                if constexpr (decltype(store)::value) {
                    if (!piece.there) continue;
                    if (!kSliced || piece.again == 0) {
                        store_piece<false>(to + piece.col, N, v);
                    } else {  // (what the last piece has of the one before it may be another workgroup's)
#pragma unroll
                        for (int i = 0; i < N; ++i)
                            if (piece.counts(i)) to[piece.col + i] = (T)v[i];
                    }
                }
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
        if (PASS == Pass::kPart) return;
        if (thread == 0 && slice == 0 && s.loss != nullptr) s.loss[row] = 0.0f;
        if constexpr (kGradient) {
            if (dlogits == nullptr) return;
            float v[N] = {};
            for (uint32_t col = first + thread * N; col < last; col += THREADS * N) store_piece<false>(to + col, valid_of<T>(col, last), v);
        }
    };
    if (row_weight == 0.0f) {
        finish_without();
        return;
    }
    if constexpr (P != 0) {
#pragma unroll
        for (int p = 0; p < P; ++p) held[p] = load_whole(from + at(p, thread).col);
    }
    // The teacher's places of this thread, their values and the student's logits there.
    uint32_t place[kSlots];
    float value[kSlots], logit[kSlots];
    float most_value = -INFINITY, most = -INFINITY, total = 0.0f, teacher = 0.0f;
    const float factor = Below<T>::factor_of(s.per_temperature);
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
        const uint32_t slot = k * THREADS + thread;
        place[k] = 0xFFFFFFFFu, value[k] = -INFINITY, logit[k] = 0.0f;
        if (slot < s.top && !(PASS == Pass::kPart && slice != 0)) {
            const uint64_t n = row * s.top + slot;
            const int64_t c = place_at(s, n);
            if (c >= 0) {
                place[k] = (uint32_t)c;
                value[k] = s.values[n];
                logit[k] = PASS == Pass::kRest ? s.logits_there[n] : (float)from[c];
                most_value = fmaxf(most_value, value[k]);
                if (PASS == Pass::kPart) s.logits_there[n] = logit[k];
            }
        }
    }
    if constexpr (PASS == Pass::kRest) {
        // the slices' parts, a few to a lane: all of them scaled to the largest
        const float2* parts = s.parts + row * s.slices;
        for (uint32_t n = thread; n < s.slices; n += THREADS) most = fmaxf(most, parts[n].x);
        const float2 t = sums.largest(most, most_value);
        most = t.x, most_value = t.y;
        for (uint32_t n = thread; n < s.slices; n += THREADS) total += parts[n].y * Below<T>::power(parts[n].x - most);
    } else {
        each_piece(kOnly, [&](const float(&v)[N], auto counts) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < N; ++i) most = fmaxf(most, P != 0 || counts(i) ? v[i] : -INFINITY);  // (twice is no harm)
        });
        const float2 t = sums.largest(most * factor, most_value);
        most = t.x, most_value = t.y;
        const Below<T> below{factor, most};
        if (PASS == Pass::kPart && most == -INFINITY) {  // nothing but -infinities, of which the row may have others, and NaN
            each_piece(kOnly, [&](const float(&v)[N], auto) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < N; ++i) total += v[i] != v[i] ? v[i] : 0.0f;
            });
        } else {
            each_piece(kOnly, [&](const float(&v)[N], auto counts) __attribute__((always_inline)) {
                float t = 0.0f;
#pragma unroll
                for (int i = 0; i < N; ++i) t += counts(i) ? below.exp(v[i]) : 0.0f;
                total += t;
            });
        }
    }
    const Below<float> below_teacher{s.per_temperature, most_value * s.per_temperature};
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
        const bool there = place[k] != 0xFFFFFFFFu;
        // (the largest of values that are all -infinity or NaN is -infinity: of the first the row has none, the second are NaN)
        value[k] = there && value[k] != -INFINITY ? below_teacher.difference(value[k]) : -INFINITY;
        const float e = there ? exp_of_share(value[k]) : 0.0f;
        teacher += e;
        if constexpr (kGradient) {
            const uint32_t slot = k * THREADS + thread;
            if (slot < (s.top + 7) / 8 * 8) place_of[slot] = place[k], weight_of[slot] = e;  // (behind the last place: none)
        }
    }
    {
        const float2 t = sums(total, teacher);
        total = t.x, teacher = t.y;
    }
    if constexpr (PASS == Pass::kPart) {
        if (thread == 0) s.parts[row * s.slices + slice] = make_float2(most, total);
        return;
    }
    if (teacher == 0.0f) {  // no place, or none with a value
        finish_without();
        return;
    }
    const Below<T> below{factor, most};
    const float per_teacher = 1.0f / teacher, log_teacher = logf(teacher), log_total = logf(total);
    float divergence = 0.0f;
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
        const float p = place[k] != 0xFFFFFFFFu ? exp_of_share(value[k]) * per_teacher : 0.0f;
        // (not equal to 0: a NaN stays)
        if (p != 0.0f) divergence += p * ((value[k] - log_teacher) - (below.natural(logit[k]) - log_total));
    }
    const float2 sum = sums(divergence, 0.0f);
    if (thread == 0 && slice == 0 && s.loss != nullptr) s.loss[row] = row_weight * s.temperature * s.temperature * sum.x;
    if constexpr (kGradient) {
        // (a NaN of the teacher's is in `teacher`, one of the student's in `total`)
        if (PASS == Pass::kRest && dlogits == nullptr) return;
        const float out = row_weight * s.temperature, per_total = 1.0f / total, scale = teacher != teacher ? teacher : out * per_total;
        each_piece(kStore, [&](float(&v)[N], auto) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = below.exp(v[i]) * scale;
        });
        // Behind the row's other values: the places, each with the shares of all that are the same.
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kSlots; ++k) {
            if (place[k] < first || place[k] >= last) continue;  // (none is above all)
            float p = 0.0f;
            for (uint32_t n = 0; n < s.top; n += 8) {
                const uint4 a = *reinterpret_cast<const uint4*>(place_of + n), b = *reinterpret_cast<const uint4*>(place_of + n + 4);
                const float4 c = *reinterpret_cast<const float4*>(weight_of + n), d = *reinterpret_cast<const float4*>(weight_of + n + 4);
                p += a.x == place[k] ? c.x : 0.0f, p += a.y == place[k] ? c.y : 0.0f, p += a.z == place[k] ? c.z : 0.0f, p += a.w == place[k] ? c.w : 0.0f;
                p += b.x == place[k] ? d.x : 0.0f, p += b.y == place[k] ? d.y : 0.0f, p += b.z == place[k] ? d.z : 0.0f, p += b.w == place[k] ? d.w : 0.0f;
            }
            to[place[k]] = (T)(out * (below.exp(logit[k]) * per_total - p * per_teacher));
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

template <class T, Pass PASS, int THREADS>
auto kernel_of(int pieces)
{
    if constexpr (THREADS == 256) {
        return pieces == 1 ? distill_kernel<T, 256, 1, PASS> : pieces == 2 ? distill_kernel<T, 256, 2, PASS> : distill_kernel<T, 256, 4, PASS>;
    } else {
        return pieces == 2   ? distill_kernel<T, 1024, 2, PASS>
               : pieces == 4 ? distill_kernel<T, 1024, 4, PASS>
               : pieces == 8 ? distill_kernel<T, 1024, 8, PASS>
               : pieces == 16 ? distill_kernel<T, 1024, 16, PASS>
                              : distill_kernel<T, 1024, 0, PASS>;
    }
}

// Several workgroups to a row, of 256 threads with four pieces each, where rows of eight such slices or more leave CUs without work: a second launch and reading the row again cost less than what one
// CU takes for the row's exponentials.  fp16, a gradient of one workgroup to a row and of several: 16 rows x 32768 8.3 us and 9.2, 16 x 65536 12.1 and 9.0, 64 x 65536 12.9 and 11.4, 64 x 131072 21.6 and
// 15.3, 128 x 131072 25.8 and 25.3, 192 x 131072 28.2 and 36.6.  1: none.
constexpr uint32_t kSliceThreads = 256, kSlicePieces = 4;
uint32_t slices_of(size_t rows, size_t cols, uint32_t dtype)
{
    const uint64_t slices = ceil_div(cols, (uint64_t)kSliceThreads * kSlicePieces * (dtype == OGQ_FP32 ? 4 : 8));
    return rows <= 96 && slices >= 8 ? (uint32_t)slices : 1;
}

}  // namespace

size_t distill_workspace(size_t rows, size_t cols, uint32_t dtype, size_t top)
{
    const uint32_t slices = slices_of(rows, cols, dtype);
    return slices > 1 ? rows * (slices * sizeof(float2) + top * sizeof(float)) : 0;
}

void launch_distill(const Values& logits, size_t rows, size_t cols, uint32_t dtype, const Integers& places, const float* values, size_t top, float temperature,
                    const float* row_weight, float* loss, const Result& dlogits, void* workspace, hipStream_t st)
{
    Distill s{};
    s.rows = (uint32_t)rows, s.cols = (uint32_t)cols, s.top = (uint32_t)top, s.wide = places.type == OGQ_INT64;
    s.per_temperature = 1.0f / temperature, s.temperature = temperature, s.stride = logits.stride, s.out_stride = dlogits.stride;
    s.places = places.data, s.values = values, s.row_weight = row_weight, s.loss = loss;
    s.slices = slices_of(rows, cols, dtype);
    s.parts = static_cast<float2*>(workspace), s.logits_there = reinterpret_cast<float*>(s.parts + rows * s.slices);
    const RowShape shape = shape_of(cols, dtype);
    with_type(dtype, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const auto from = static_cast<const T*>(logits.data);
        const auto to = static_cast<T*>(dlogits.data);
        if (s.slices > 1) {
            const dim3 grid = grid_of((uint64_t)rows * s.slices), block(kSliceThreads);
            launch_kernel(distill_kernel<T, kSliceThreads, kSlicePieces, Pass::kPart>, grid, block, st, from, s, to);
            launch_kernel(distill_kernel<T, kSliceThreads, kSlicePieces, Pass::kRest>, grid, block, st, from, s, to);
            return;
        }
        const auto go = [&](auto pass) {
            constexpr Pass kPass = decltype(pass)::value;
            const auto kernel = shape.threads == 256 ? kernel_of<T, kPass, 256>(shape.pieces) : kernel_of<T, kPass, 1024>(shape.pieces);
            launch_kernel(kernel, grid_of(rows), dim3(shape.threads), st, from, s, to);
        };
        if (to != nullptr) go(std::integral_constant<Pass, Pass::kGradient>{});
        else go(std::integral_constant<Pass, Pass::kLoss>{});
    });
}

}  // namespace ogq
