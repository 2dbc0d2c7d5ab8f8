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
// NEAR: the rows of a tile lie within 2^32 bytes, and are held as one address and 32 bits to each.
template <class T, int ROWS, bool NEAR>
struct Along {
    static constexpr int THREADS = 256;
    static constexpr int kChunks = kDepth<T> / 8, kRowBytes = kDepth<T> * 2, kPlane = ROWS * kRowBytes, kUnits = ROWS * kChunks / THREADS, kUnitRows = THREADS / kChunks;
    static_assert(kUnits * THREADS == ROWS * kChunks);
    using Offset = std::conditional_t<NEAR, uint32_t, uint64_t>;
    const T* data;          // the tile's first row
    Offset offset[kUnits];  // of a thread's values in a step, in bytes
    uint32_t last, mine;
    char* to;
    Chunk<T> held[kUnits];

    static __device__ __forceinline__ uint32_t place(uint32_t row, uint32_t chunk) { return row * kRowBytes + ((chunk ^ (row / (256 / kRowBytes) & (kChunks - 1))) * 16); }

    // Rows `first` ... of `number`; what lies behind the last row is any row that is there: its sums are not stored.
    __device__ __forceinline__ Along(const T* data_, uint64_t stride, uint32_t first, uint32_t number, uint32_t, uint32_t last_, uint32_t thread, char* lds)
        : data(data_ + first * stride), last(last_)
    {
        const uint32_t row = thread / kChunks, chunk = thread % kChunks;
        mine = chunk * 8;
#pragma unroll
        for (int u = 0; u < kUnits; ++u) offset[u] = ((Offset)min(row + u * kUnitRows, number - 1 - first) * (Offset)stride + mine) * sizeof(T);
        static_assert(kUnitRows % 16 == 0);  // (then place moves the chunks of all of a thread's rows alike)
        to = lds + place(row, chunk);
    }
    // How many whole steps from `first` on can be fetched without asking.
    __device__ __forceinline__ uint32_t readable(uint32_t first) const { return (last - first) / kDepth<T>; }
    __device__ __forceinline__ const T* at(uint32_t k, int u) const { return reinterpret_cast<const T*>(reinterpret_cast<const char*>(data + k) + offset[u]); }
    __device__ __forceinline__ void fetch_unit(uint32_t k, int u)
    {
        if constexpr (NEAR) asm volatile("" : "+v"(offset[u]));  // (an address in scalar registers and 32 bits: the compiler makes 64 bits of these ahead of the loop)
        held[u].load(at(k, u));
    }
    __device__ __forceinline__ void fetch(uint32_t k)
    {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) fetch_unit(k, u);
    }
    __device__ __forceinline__ void fetch_unit_asking(uint32_t k, int u) { held[u].load(at(k, u), k + mine >= last ? 0 : (int)min(8u, last - k - mine)); }
    __device__ __forceinline__ void fetch_asking(uint32_t k)
    {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) fetch_unit_asking(k, u);
    }
    __device__ __forceinline__ void bring_unit(uint32_t stage_bytes, int u) { held[u].store(to + stage_bytes + u * kUnitRows * kRowBytes, kPlane); }
    __device__ __forceinline__ void bring(uint32_t stage_bytes)
    {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) bring_unit(stage_bytes, u);
    }
    // Where a lane finds its part of the first operand in 32 rows from `row` (a multiple of 32): the others lie kOperand bytes apart, and those of k = 16 h ... at this place ^ 32 h.
    static constexpr int kOperand = 32 * kRowBytes;
    static __device__ __forceinline__ uint32_t operand(uint32_t row, uint32_t lane) { return place(row + (lane & 31), lane >> 5); }
    static __device__ __forceinline__ s16x8 read_operand(const char* lds, uint32_t at, uint32_t bytes, int n, int h)
    {
        return *reinterpret_cast<const s16x8*>(lds + (at ^ (32 * h)) + bytes + n * kOperand);
    }
    // Where a lane finds its part of an operand: 32 rows from `row`, k = 16 h + lane / 32 * 8 ...
    static __device__ __forceinline__ s16x8 read(const char* plane, uint32_t row, int h, uint32_t lane)
    {
        return *reinterpret_cast<const s16x8*>(plane + place(row + (lane & 31), 2 * h + (lane >> 5)));
    }
};

// The same for rows across k: a step is kDepth rows of COLS values, of which the columns are the operand's rows.  Chunk c (32 bytes) of row k lies at c ^ twist(k).
template <class T, int COLS, bool NEAR>
struct Across {
    static constexpr int THREADS = 256;
    static constexpr int kChunks = COLS / 16, kRowBytes = COLS * 2, kPlane = kDepth<T> * kRowBytes, kUnits = kDepth<T> * kChunks / THREADS, kUnitRows = THREADS / kChunks;
    static_assert(kUnits * THREADS == kDepth<T> * kChunks && kUnitRows % 4 == 0);
    const T* data;
    uint64_t stride;
    std::conditional_t<NEAR, uint32_t, uint64_t> offset;  // of a thread's values in a step, in bytes
    uint32_t last, row, mine;
    int valid;
    bool partial, whole_factor;
    char* to;
    Chunk<T> held[kUnits][2];

    static __device__ __forceinline__ uint32_t twist(uint32_t k) { return (k & (kChunks >= 8 ? 3u : 1u)) * 2u; }

    // Columns `first` ... of `number`, rows below `last`, of which the factor has `rows`.  What lies behind the last column is any value that is there: its sums are not stored.
    __device__ __forceinline__ Across(const T* data_, uint64_t stride_, uint32_t first, uint32_t number, uint32_t rows, uint32_t last_, uint32_t thread, char* lds)
        : data(data_), stride(stride_), last(last_)
    {
        const uint32_t chunk = thread % kChunks;
        row = thread / kChunks;
        mine = first + chunk * 16;
        valid = mine >= number ? 0 : (int)min(16u, number - mine);
        partial = first + COLS > number && number % 16 != 0;
        whole_factor = last_ == rows;
        offset = (row * (decltype(offset))stride + (valid == 0 ? first : mine)) * sizeof(T);
        to = lds + row * kRowBytes + ((chunk ^ twist(row)) * 32);
    }
    // How many whole steps from `first` on can be fetched without asking: a thread whose sixteen columns reach beyond the last one reads on into the next row, which the last row does not have.
    __device__ __forceinline__ uint32_t readable(uint32_t first) const
    {
        const uint32_t whole = (last - first) / kDepth<T>;
        if (!partial || whole == 0) return whole;
        if (stride < 16) return 0;
        return whole_factor && first + whole * kDepth<T> == last ? whole - 1 : whole;
    }
    __device__ __forceinline__ void fetch_unit(uint32_t k, int u)
    {
        const T* from = reinterpret_cast<const T*>(reinterpret_cast<const char*>(data + (uint64_t)(k + u * kUnitRows) * stride) + offset);
        held[u][0].load(from);
        held[u][1].load(from + 8);
    }
    __device__ __forceinline__ void fetch(uint32_t k)
    {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) fetch_unit(k, u);
    }
    __device__ __forceinline__ void fetch_unit_asking(uint32_t k, int u)
    {
        const uint32_t at = k + row + u * kUnitRows;
        const T* from = data + (uint64_t)at * stride + mine;
        held[u][0].load(from, at < last ? valid : 0);
        held[u][1].load(from + 8, at < last ? valid - 8 : 0);
    }
    __device__ __forceinline__ void fetch_asking(uint32_t k)
    {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) fetch_unit_asking(k, u);
    }
    __device__ __forceinline__ void bring_unit(uint32_t stage_bytes, int u)
    {
        held[u][0].store(to + stage_bytes + u * kUnitRows * kRowBytes, kPlane);
        held[u][1].store(to + stage_bytes + u * kUnitRows * kRowBytes + 16, kPlane);
    }
    __device__ __forceinline__ void bring(uint32_t stage_bytes)
    {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) bring_unit(stage_bytes, u);
    }
    // (`at` of operands has no part for the columns: these move the chunks)
    static __device__ __forceinline__ uint32_t operand(uint32_t col, uint32_t lane) { return col << 16 | lane; }
    static __device__ __forceinline__ s16x8 read_operand(const char* lds, uint32_t at, uint32_t bytes, int n, int h) { return read(lds + bytes, (at >> 16) + 32 * n, h, at & 63); }
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

// fp32: an infinity is its first piece alone, and its products with pieces that are 0 are NaN.  Sums that are NaN are made again, one product after the other, where a factor is infinite or may make a product that is:
// a wavefront looks at all of its rows for one first, 64 values at a time.  Without it NaN come from NaN, and stay.  256 x 4096 to 4096, 63 us: with a NaN in each row 3895 us, now 147; with
// an infinity in each row 306, 354; 2048 x 2048 to 2048, 112: all NaN 15405, now 258.
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
    bool large = false;
    const auto look = [&](float v) __attribute__((always_inline)) { large |= fabsf(v) >= 0x1p64f; };  // (a product of others is within fp32)
    const auto look_along = [&](const float* rows, uint64_t stride, uint32_t row, uint32_t behind) __attribute__((always_inline)) {
        for (; row < behind && __builtin_amdgcn_ballot_w64(large) == 0; ++row)
#pragma unroll 4
            for (uint32_t k = first + lane; k < last; k += 64) look(rows[row * stride + k]);
    };
    look_along(x, s.x_stride, token, min(s.tokens, token + 32 * NT));
    if constexpr (TRANSPOSED) {
        static_assert(NO <= 2);
        if (__builtin_amdgcn_ballot_w64(large) == 0 && out + lane < min(s.outs, out + 32 * NO)) {
#pragma unroll 8
            for (uint32_t k = first; k < last; ++k) look(weight[k * s.weight_stride + out + lane]);
        }
    } else {
        look_along(weight, s.weight_stride, out, min(s.outs, out + 32 * NO));
    }
    if (__builtin_amdgcn_ballot_w64(large) == 0) return;
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
                for (uint32_t k = first; k < last && v == v; ++k)
                    v = __builtin_fmaf(x[t * s.x_stride + k], TRANSPOSED ? weight[k * s.weight_stride + o] : weight[o * s.weight_stride + k], v);
                sum[a][b][i] = v;
            }
        }
}

// Tiles of OUT outputs by TOKENS tokens, a quarter in each of four wavefronts.  In 16 bits two stages of LDS and one barrier a step: while one step is multiplied the next one waits in registers,
// goes to LDS behind the products, and the one behind it sets off.  fp32, whose three pieces fill LDS, has one stage and two barriers, and more workgroups to a CU.
// Where there are too few tiles for the chip, two teams of four wavefronts take a tile's steps in turn and add what they have in LDS.
// 16 bits: bound by a step's latency where tiles are few (37 x 1001 to 2589 9 us, sixteen steps), else by LDS: a product of 32 cycles takes two operands of 16 bytes a lane, of which a 128 x 128 tile uses each
// twice (2000 x 2048 to 2048 fp16 30 us, 560 TFLOP/s).  fp32: six bf16 products, 256 x 25088 to 4096 300 us, 1.05 PFLOP/s of them; matrix cores busy for 0.62 of the cycles.
template <class T, int OUT, int TOKENS, bool TRANSPOSED, int TEAMS = 1>
__global__ __launch_bounds__(256 * TEAMS) void linear_kernel(const T* x, const T* weight, LinearShape s, Epilogue<T> e)
{
    using FeedW = std::conditional_t<TRANSPOSED, Across<T, OUT, false>, Along<T, OUT, false>>;
    using FeedX = Along<T, TOKENS, false>;
    constexpr int kBytesW = kPlanes<T> * FeedW::kPlane, kStage = kBytesW + kPlanes<T> * FeedX::kPlane, NO = OUT / 64, NT = TOKENS / 64, kStages = sizeof(T) == 2 ? 2 : 1, D = kDepth<T>;
    constexpr int kBytes = kStages * kStage > 4 * kTurn<NO> ? kStages * kStage : 4 * kTurn<NO>;
    static_assert(TEAMS == 1 || (TEAMS == 2 && kStages == 2 && kBytes >= 1024 * NO * NT * 16));
    __shared__ __align__(16) char all_lds[TEAMS * kBytes];
    const uint32_t lane = threadIdx.x & 63, all_waves = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = all_waves & 3, team = TEAMS == 1 ? 0 : all_waves >> 2;
    const uint32_t thread = TEAMS == 1 ? threadIdx.x : threadIdx.x & 255;
    char* lds = all_lds + team * kBytes;
    const uint32_t tiles = s.tiles_out * s.tiles_token, tile = this_block() % tiles, part = this_block() / tiles;
    if (part >= s.parts) return;  // (behind the last tile, in the last row of a large grid)
    const uint32_t out = tile % s.tiles_out * OUT, token = tile / s.tiles_out * TOKENS, out_wave = (wave & 1) * (OUT / 2), token_wave = (wave >> 1) * (TOKENS / 2);
    const uint32_t first = part * s.part, last = min(s.cols, first + s.part);
    FeedW feed_w(weight, s.weight_stride, out, s.outs, s.cols, last, thread, lds);
    FeedX feed_x(x, s.x_stride, token, s.tokens, s.cols, last, thread, lds + kBytesW);
    f32x16 sum[NO][NT] = {};
    const uint32_t whole = first + (first < last ? feed_w.readable(first) : 0) * kDepth<T>;  // the first column of a step that asks
    const auto fetch = [&](uint32_t k) __attribute__((always_inline)) {
        if (k < whole) {
            feed_w.fetch(k);
            feed_x.fetch(k);
        } else if (k < last) {
            feed_w.fetch_asking(k);
            feed_x.fetch_asking(k);
        }
    };
    const auto bring = [&](uint32_t stage) __attribute__((always_inline)) {
        feed_w.bring(stage * kStage);
        feed_x.bring(stage * kStage);
    };
    // The pairs of pieces of a step's slices of 16, one behind the other; the operands of one are read while the one before it is multiplied.
    constexpr int kPairs = kPlanes<T> == 1 ? 1 : 6, kSlices = D / 16;
    struct Operands {
        s16x8 w[NO], x[NT];
    };
    const auto read = [&](Operands& r, const char* at, int n) __attribute__((always_inline)) {
        constexpr int kW[6] = {2, 0, 1, 1, 0, 0}, kX[6] = {0, 2, 1, 0, 1, 0};  // (the smallest first.  The second piece is below 2^-7 of the first, the third below 2^-15: the three pairs left out are below 2^-21 of a product, with its sign)
        const int h = n / kPairs, p = kPairs == 1 ? 0 : kW[n % 6], q = kPairs == 1 ? 0 : kX[n % 6];
#pragma unroll
        for (int i = 0; i < NO; ++i) r.w[i] = FeedW::read(at + p * FeedW::kPlane, out_wave + 32 * i, h, lane);
#pragma unroll
        for (int j = 0; j < NT; ++j) r.x[j] = FeedX::read(at + kBytesW + q * FeedX::kPlane, token_wave + 32 * j, h, lane);
    };
    const auto products = [&](uint32_t stage) __attribute__((always_inline)) {
        const char* at = lds + stage * kStage;
        Operands r[2];
        read(r[0], at, 0);
#pragma unroll
        for (int n = 0; n < kSlices * kPairs; ++n) {
            if (n + 1 < kSlices * kPairs) read(r[(n + 1) & 1], at, n + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                asm volatile("" : "+v"(r[n & 1].x[j]));  // (a product has no other order than that of what it takes)
#pragma unroll
                for (int i = 0; i < NO; ++i) sum[i][j] = multiply_add<T>(r[n & 1].w[i], r[n & 1].x[j], sum[i][j]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const uint32_t begin = first + team * D;
    fetch(begin);
    if constexpr (kStages == 2) {
        if (begin < last) bring(0);
        fetch(begin + TEAMS * D);
        uint32_t stage = 0;
        // (the teams meet at the same barriers: the last step may be one team's alone)
        for (uint32_t k = begin; k < last + team * D; k += TEAMS * D) {
            __syncthreads();
            if (TEAMS == 1 || k < last) products(stage);
            stage ^= 1;
            if (k + TEAMS * D < last) bring(stage);
            fetch(k + 2 * TEAMS * D);
        }
    } else {
        for (uint32_t k = first; k < last; k += kDepth<T>) {
            __syncthreads();
            bring(0);
            __syncthreads();
            fetch(k + kDepth<T>);
            products(0);
        }
    }
    __syncthreads();
    if constexpr (sizeof(T) == 4) mend_sums<TRANSPOSED>(x, weight, s, out + out_wave, token + token_wave, first, last, lane, sum);
    if constexpr (TEAMS == 2) {
        // the second team's sums, 16 bytes of a lane at a time
        f32x4* const exchange = reinterpret_cast<f32x4*>(all_lds + kBytes) + wave * (NO * NT * 256) + lane;
#pragma unroll
        for (int a = 0; a < NO; ++a)
#pragma unroll
            for (int b = 0; b < NT; ++b)
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    f32x4& place = exchange[((a * NT + b) * 4 + m) * 64];
                    if (team == 1) place = f32x4{sum[a][b][4 * m], sum[a][b][4 * m + 1], sum[a][b][4 * m + 2], sum[a][b][4 * m + 3]};
                }
        __syncthreads();
        if (team == 1) return;
#pragma unroll
        for (int a = 0; a < NO; ++a)
#pragma unroll
            for (int b = 0; b < NT; ++b)
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    const f32x4 v = exchange[((a * NT + b) * 4 + m) * 64];
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[a][b][4 * m + i] += v[i];
                }
    }
    finish_tile<T>(sum, out + out_wave, token + token_wave, lane, s, part, e, lds + wave * kTurn<NO>);
}

// Workgroups go to the eight XCDs in turn, each with an L2 of its own: an XCD takes neighbouring tiles, four along the outputs by eight along the tokens at a time.
__device__ __forceinline__ uint2 tile_of(uint32_t id, uint32_t tiles_out, uint32_t tiles_token)
{
    constexpr uint32_t kXcds = 8, kWide = 4;
    const uint32_t tiles = tiles_out * tiles_token, each = tiles / kXcds, more = tiles % kXcds, xcd = id % kXcds;
    const uint32_t n = xcd * each + min(xcd, more) + id / kXcds;
    const uint32_t panel = n / (kWide * tiles_token), rest = n % (kWide * tiles_token), width = min(kWide, tiles_out - panel * kWide);
    return make_uint2(panel * kWide + rest % width, rest / width);
}

// Tiles of 256 x 256 sums of 16-bit products, 128 x 128 in each of four wavefronts, one to a SIMD, which has all of its registers: 256 hold the sums.  A step of 64 columns is multiplied in four
// quarters; while one is, the next one's operands come from LDS.  Two stages of LDS: the step behind the next one goes where the last one was, and the one behind that sets off from
// memory.  One barrier a step, in front of the last quarter, which reads the next step's first operands.
template <class T, bool TRANSPOSED>
__global__ __launch_bounds__(256, 1) void large_linear_kernel(const T* x, const T* weight, LinearShape s, Epilogue<T> e)
{
    static_assert(kPlanes<T> == 1);
    using FeedW = std::conditional_t<TRANSPOSED, Across<T, 256, true>, Along<T, 256, true>>;
    using FeedX = Along<T, 256, true>;
    constexpr int kStage = FeedW::kPlane + FeedX::kPlane, kW = FeedW::kUnits, kX = FeedX::kUnits;
    static_assert(kX == 8 && (kW == 8 || kW == 4) && 2 * kStage >= 4 * kTurn<4>);
    __shared__ __align__(256) char lds[2 * kStage];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (this_block() >= s.tiles_out * s.tiles_token) return;  // (in the last row of a large grid)
    const uint2 tile = tile_of(this_block(), s.tiles_out, s.tiles_token);
    const uint32_t out = tile.x * 256, token = tile.y * 256, out_wave = (wave & 1) * 128, token_wave = (wave >> 1) * 128;
    FeedW feed_w(weight, s.weight_stride, out, s.outs, s.cols, s.cols, threadIdx.x, lds);
    FeedX feed_x(x, s.x_stride, token, s.tokens, s.cols, s.cols, threadIdx.x, lds + FeedW::kPlane);
    const uint32_t whole = feed_w.readable(0);
    f32x16 sum[4][4] = {};
    struct Operands {
        s16x8 w[4], x[4];
    };
    uint32_t w_at = FeedW::operand(out_wave, lane), x_at = FeedX::operand(token_wave, lane);
    // Operand m of the eight, in the order in which they are needed first: w0, x0 ... x3, w1 ... w3.
    const auto read = [&](Operands& r, uint32_t stage, int h, int m) __attribute__((always_inline)) {
        if (m >= 1 && m < 5) r.x[m - 1] = FeedX::read_operand(lds, x_at, stage * kStage + FeedW::kPlane, m - 1, h);
        else r.w[m == 0 ? 0 : m - 4] = FeedW::read_operand(lds, w_at, stage * kStage, m == 0 ? 0 : m - 4, h);
    };
    const auto product = [&](const Operands& r, int m) __attribute__((always_inline)) { sum[m / 4][m % 4] = multiply_add<T>(r.w[m / 4], r.x[m % 4], sum[m / 4][m % 4]); };
    // (one behind the last whole step is the last one again, and not used)
    const auto column = [&](uint32_t n) __attribute__((always_inline)) { return min(n, whole - 1) * kDepth<T>; };
    // Unit u of both factors' sixteen (two of W's to a unit of 32 bytes): to stage `stage`, and its place in step n sets off.
    const auto pass_on = [&](uint32_t stage, uint32_t n, int u) __attribute__((always_inline)) {
        if (u < 8) {
            feed_x.bring_unit(stage * kStage, u);
            feed_x.fetch_unit(column(n), u);
        } else if (kW == 8 || (u & 1) == 0) {
            feed_w.bring_unit(stage * kStage, (u - 8) * kW / 8);
            feed_w.fetch_unit(column(n), (u - 8) * kW / 8);
        }
    };
    Operands a, b;
    // A quarter of a step: sixteen products, which the matrix core takes 32 cycles for each.  Behind each of the first eight an operand of the next quarter is read, behind the others units
    // first ... last are passed on.  The order is as written: the compiler's own has the reads waited for where they are issued (8192 x 8192 sums of 8192 products 904 us)
    const auto quarter = [&](Operands& now, Operands& then, uint32_t stage, int h, uint32_t to, uint32_t n, int first, int last, bool meet) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < 16; ++m) {
            asm volatile("" : "+v"(now.x[m % 4]));  // (a product has no other order than that of what it takes)
            product(now, m);
            if (m < 8) read(then, stage, h, m);
            else if (first + m - 8 < last) pass_on(to, n, first + m - 8);
            __builtin_amdgcn_sched_barrier(0);
            if (meet && m == 13) {
                __syncthreads();
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    // Step n, of which `a` holds the first quarter's operands, in stage `here`; step n + 1 is in registers on its way to the other stage ...
    const auto step = [&](uint32_t n, uint32_t here) __attribute__((always_inline)) {
        const uint32_t next = here ^ 1;
        if constexpr (!TRANSPOSED) asm volatile("" : "+v"(w_at));  // (places are made again every step: there are no registers to hold all of them)
        asm volatile("" : "+v"(x_at));
        quarter(a, b, here, 1, next, n + 2, 0, 6, false);
        quarter(b, a, here, 2, next, n + 2, 6, 12, false);
        quarter(a, b, here, 3, next, n + 2, 12, 16, true);
        quarter(b, a, next, 0, next, n + 2, 0, 0, false);
    };
    if (whole != 0) {
        feed_x.fetch(0), feed_w.fetch(0);
        feed_x.bring(0), feed_w.bring(0);
        feed_x.fetch(column(1)), feed_w.fetch(column(1));
        __syncthreads();
#pragma unroll
        for (int m = 0; m < 8; ++m) read(a, 0, 0, m);
        uint32_t n = 0;
        for (; n + 2 <= whole; n += 2) {
            step(n, 0);
            step(n + 1, 1);
        }
        if (n < whole) step(n, 0);
    }
    for (uint32_t k = whole * kDepth<T>; k < s.cols; k += kDepth<T>) {
        __syncthreads();
        // (unit after unit: together they would need more registers than there are)
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            feed_x.fetch_unit_asking(k, u);
            feed_x.bring_unit(0, u);
            __builtin_amdgcn_sched_barrier(0);
            if (u < kW) {
                feed_w.fetch_unit_asking(k, u);
                feed_w.bring_unit(0, u);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 4; ++h) {
#pragma unroll
            for (int m = 0; m < 8; ++m) read(a, 0, h, m);
#pragma unroll
            for (int m = 0; m < 16; ++m) product(a, m);
        }
    }
    __syncthreads();
    finish_tile<T>(sum, out + out_wave, token + token_wave, lane, s, 0, e, lds + wave * kTurn<4>);
}

// The same tiles where the rows of both factors begin at multiples of 16 bytes: memory goes to LDS without a way through registers (16 bytes to a lane: lane n of a wavefront's load writes
// bytes 16 n ... of 1 KB), in the places that Along and Across read.
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t offset, uint32_t lds)
{
    // (in assembly because the compiler would have every read of LDS wait for all such loads; nothing is returned in registers.  One wait state between m0 and its use)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}

// Units of 4 KB of a step of 256 rows along k, 32 rows each, or of 64 rows across k, 8 rows each.
template <class T, bool ACROSS>
struct Direct {
    static constexpr int kUnits = 8, kRowPieces = ACROSS ? 32 : 8, kUnitRows = 256 / kRowPieces;
    const T* data;
    uint64_t stride;
    uint32_t offset[ACROSS ? 1 : kUnits], lds;

    Direct() = default;
    // `at`: where the factor's plane of the first stage begins.
    __device__ __forceinline__ Direct(const T* data_, uint64_t stride_, uint32_t first, uint32_t number, uint32_t thread, uint32_t at) : data(data_), stride(stride_)
    {
        const uint32_t row = thread / kRowPieces, piece = thread % kRowPieces;
        lds = at + __builtin_amdgcn_readfirstlane(thread / 64) * 1024;
        if constexpr (ACROSS) {
            const uint32_t column = first + ((piece / 2) ^ Across<T, 256, true>::twist(row)) * 16 + piece % 2 * 8;
            offset[0] = (row * (uint32_t)stride + (column < number ? column : first)) * sizeof(T);
        } else {
            data += first * stride;
#pragma unroll
            for (int u = 0; u < kUnits; ++u) offset[u] = (min(row + u * kUnitRows, number - 1 - first) * (uint32_t)stride + (piece ^ (row / 2 & 7)) * 8) * sizeof(T);
        }
    }
    __device__ __forceinline__ void load(uint32_t k, uint32_t stage_bytes, int u)
    {
        if constexpr (ACROSS) load_to_lds(data + (uint64_t)(k + u * kUnitRows) * stride, offset[0], lds + stage_bytes + u * 4096);
        else load_to_lds(data + k, offset[u], lds + stage_bytes + u * 4096);
    }
};

// The sums of a wavefront, 128 outputs from `out` and 128 tokens from `token`, on their way out in eight parts of 64 by 32.  A lane holds four neighbouring outputs of a token; through LDS (8 KB of the
// wavefront's own, 16 bytes of row r in place of those 16 (r % 16) bytes away, for the banks' sake) eight lanes get the 64 of one, so that whole lines are written.
template <class T>
__device__ __forceinline__ void finish_large(const f32x16 (&sum)[4][4], uint32_t out, uint32_t token, uint32_t lane, const LinearShape& s, const Epilogue<T>& e, char* space)
{
    const uint32_t column = lane % 8 * 8;
    float bias[8];
#pragma unroll 1
    for (int part = 0; part < 8; ++part) {  // (one code for all parts: only what reads the sums' registers is there for each)
#pragma unroll
        for (int p = 0; p < 8; ++p)
            if (p == part) {
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        const f32x16& v = sum[p / 4 * 2 + a][p % 4];
                        *reinterpret_cast<f32x4*>(space + (lane & 31) * 256 + (((a * 8 + 2 * m + (lane >> 5)) ^ (lane & 15)) * 16)) = f32x4{v[4 * m], v[4 * m + 1], v[4 * m + 2], v[4 * m + 3]};
                    }
            }
        wavefront_sync();
        const uint32_t o = out + part / 4 * 64 + column;
        const int valid = valid_of<T>(o, s.outs);
        float v[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t row = lane / 8 + 8 * i;
#pragma unroll
            for (int h = 0; h < 2; ++h) memcpy(v[i] + 4 * h, __builtin_assume_aligned(space + row * 256 + (((lane % 8 * 2 + h) ^ (row & 15)) * 16), 16), 16);
        }
        wavefront_sync();
        if (valid == 0) continue;
        if (part % 4 == 0) load_vector<T>(e.bias == nullptr ? nullptr : e.bias + o, valid, 0.0f, bias);
        const uint32_t first = token + part % 4 * 32 + lane / 8;
        e.template rows<4>(first, 8, s.tokens, o, valid, bias, v);
    }
}

// A step's four quarters, sixteen products each; behind a product an operand of the next quarter is read or a load to LDS sets off.  LDS holds five planes of 32 KB: the step's two, the next
// one's, and one to which the next plane is on its way: x two steps ahead in the first two quarters, W in the last, when the step's own operands have been read by all: one barrier a step.  A workgroup
// stays and takes tile after tile; the next one's first two steps come in while the last one's sums leave, through the plane that is free.
// Bound by the matrix cores and the power that they draw: 8192 x 4096 to 16384 bf16 880 to 930 us plain (1.18 to 1.25 PFLOP/s, the library's product 786 to 907), 925 to 975 with gelu and what goes into it (the first twenty launches 1000 to 1270, until the card's power has settled);
// 8192 x 8192 sums of 8192 products 770 to 806 (1.36 to 1.43, library 676 to 728); transposed, 4096 x 4096 to 16384, 462 to 467 (library 504).  Matrix cores are busy for 0.63 to 0.71 of the cycles; products
// alone, of random values in registers, reach 1.7 PFLOP/s.  No gain: a second set of operands a step ahead, all operands read in the first two quarters.
template <class T, bool TRANSPOSED>
__global__ __launch_bounds__(256, 1) void direct_linear_kernel(const T* x, const T* weight, LinearShape s, Epilogue<T> e)
{
    using FeedW = std::conditional_t<TRANSPOSED, Across<T, 256, true>, Along<T, 256, true>>;
    using FeedX = Along<T, 256, true>;
    constexpr uint32_t kPlane = FeedX::kPlane;
    static_assert(kPlanes<T> == 1 && FeedW::kPlane == 32768 && kPlane == 32768);
    __shared__ __align__(256) char lds[5 * kPlane];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t tiles = s.tiles_out * s.tiles_token, out_wave = (wave & 1) * 128, token_wave = (wave >> 1) * 128, steps = s.cols / kDepth<T>;
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    // where loads are: the tile that is multiplied, or the next one
    Direct<T, TRANSPOSED> load_w;
    Direct<T, false> load_x;
    const auto turn_to = [&](uint32_t id) __attribute__((always_inline)) {
        const uint2 tile = tile_of(id < tiles ? id : blockIdx.x, s.tiles_out, s.tiles_token);  // (behind the last tile the first one again, which is not used)
        load_w = Direct<T, TRANSPOSED>(weight, s.weight_stride, tile.x * 256, s.outs, threadIdx.x, base);
        load_x = Direct<T, false>(x, s.x_stride, tile.y * 256, s.tokens, threadIdx.x, base);
    };
    f32x16 sum[4][4];
    struct Operands {
        s16x8 w[4], x[4];
    };
    uint32_t w_at = FeedW::operand(out_wave, lane), x_at = FeedX::operand(token_wave, lane);
    // Operand m of the eight, in the order in which they are needed first: w0, x0 ... x3, w1 ... w3.
    const auto read = [&](Operands& r, uint32_t x_plane, uint32_t w_plane, int h, int m) __attribute__((always_inline)) {
        if (m >= 1 && m < 5) r.x[m - 1] = FeedX::read_operand(lds, x_at, x_plane, m - 1, h);
        else r.w[m == 0 ? 0 : m - 4] = FeedW::read_operand(lds, w_at, w_plane, m == 0 ? 0 : m - 4, h);
    };
    // The planes, by where they begin: this step's, the next one's, and the one that is free.
    uint32_t x_here = 0, w_here = kPlane, x_next = 2 * kPlane, w_next = 3 * kPlane, free = 4 * kPlane;
    Operands a, b;
    turn_to(blockIdx.x);
#pragma unroll
    for (int u = 0; u < 8; ++u) load_x.load(0, x_here, u), load_w.load(0, w_here, u);
#pragma unroll
    for (int u = 0; u < 8; ++u) load_x.load(kDepth<T>, x_next, u), load_w.load(kDepth<T>, w_next, u);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int m = 0; m < 8; ++m) read(a, x_here, w_here, 0, m);
    uint32_t stores = 0;  // of the last tile, at least, that may be under way
    for (uint32_t id = blockIdx.x; id < tiles; id += gridDim.x) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[i][j] = f32x16{};
        for (uint32_t n = 0; n < steps; ++n) {
            if (n + 2 == steps) turn_to(id + gridDim.x);
            const uint32_t k = (n + 2 < steps ? n + 2 : n + 2 - steps) * kDepth<T>;
            if constexpr (!TRANSPOSED) asm volatile("" : "+v"(w_at));  // (places are made again every step: there are no registers to hold all of them)
            asm volatile("" : "+v"(x_at));
            const auto quarter = [&](int q, Operands& now, Operands& then, uint32_t x_plane, uint32_t w_plane) __attribute__((always_inline)) {
#pragma unroll
                for (int m = 0; m < 16; ++m) {
                    asm volatile("" : "+v"(now.x[m % 4]));  // (a product has no other order than that of what it takes)
                    sum[m / 4][m % 4] = multiply_add<T>(now.w[m / 4], now.x[m % 4], sum[m / 4][m % 4]);
                    if (q == 2 ? m < 8 : m % 2 == 0) read(then, x_plane, w_plane, (q + 1) % 4, q == 2 ? m : m / 2);
                    if (q < 2 && m % 4 == 1) load_x.load(k, free, q * 4 + m / 4);
                    if (q == 3 && m % 2 == 1) load_w.load(k, x_here, m / 2);
                    __builtin_amdgcn_sched_barrier(0);
                    if (q == 2 && m == 13) {
                        // This wavefront's share of the next step has arrived, all but the eight loads of the one behind it.  (In front of these, in a tile's first step, the last tile's stores:
                        // 32 of a tile that is full, or twice as many.  They complete in the order in which they were issued.)
                        if (n != 0) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
                        else if (stores == 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                        else if (stores == 32) asm volatile("s_waitcnt vmcnt(40)" ::: "memory");
                        else asm volatile("s_waitcnt vmcnt(63)" ::: "memory");
                        __syncthreads();
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            };
            quarter(0, a, b, x_here, w_here);
            quarter(1, b, a, x_here, w_here);
            quarter(2, a, b, x_here, w_here);
            quarter(3, b, a, x_next, w_next);
            const uint32_t w_last = w_here, x_last = x_here;
            x_here = x_next, w_here = w_next, x_next = free, w_next = x_last, free = w_last;
        }
        const uint2 tile = tile_of(id, s.tiles_out, s.tiles_token);
        finish_large<T>(sum, tile.x * 256 + out_wave, tile.y * 256 + token_wave, lane, s, e, lds + free + wave * (kPlane / 4));
        stores = (tile.x + 1) * 256 <= s.outs && (tile.y + 1) * 256 <= s.tokens ? (e.before != nullptr ? 64 : 32) : 0;
        __syncthreads();
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (nothing is on its way to LDS that is no longer this workgroup's)
    __syncthreads();
}

// The parts' sums of a piece of a token's outputs.
template <class T>
__global__ __launch_bounds__(kBlock) void join_parts_kernel(LinearShape s, Epilogue<T> e, uint32_t per_token)
{
    constexpr int N = kPiece<T>;
    const uint64_t piece = (uint64_t)this_block() * kBlock + threadIdx.x;
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
    uint32_t tile_out, tile_token, tiles_out, tiles_token, part, parts, teams;
};

// Which tiles, and into how many parts a sum is cut: what takes least by this account, in us.  With c workgroups on a CU a step (64 columns in 16 bits, 32 in fp32) takes a + b c, of which
// a CU holds up to `most`; parts cost a launch of 3.5 us, 0.3 us each, and 8 bytes for each of their sums, written and read, at 4 TB/s.  Where there is up
// to one workgroup to a CU, the tiles of 64 tokens have two teams in 16 bits, and a step takes 0.7 of the time (64 x 4096 to 16384 27.6 us without, 24.3 with; 128 x 128 are no faster with them: 1733 x 1216 to 1249 19.7 without, 20.5 with).
//   16 bits: 64 x 64 0.28 + 0.17 c, 128 x 64 0.27 + 0.26 c, 128 x 128 0.52 + 0.26 c, 256 x 256 (no parts) 1.6 and 10 a tile;  fp32: 128 x 64 0.5 + 0.63 c, 128 x 128 1.0 + 0.8 c.
// Measured for x [tokens, cols] to outs (fp16; by tile and parts): 1000 x 1000 to 1000: 64 x 64 9.0 in one part, 14.8 in two, 128 x 128 16.9; 128 x 4096 to 4096: 64 x 64 29.3 in one, 16.5 in 4, 18.7 in 8,
// 128 x 128 50.7 in one, 19.4 in 6; 256 x 25088 to 4096: 128 x 128 148 in 2, 74.9 in 8, 92.4 in 12, 64 x 64 98.8 in 2; 2000 x 2048 to 2048: 64 x 64 33.5, 128 x 64 28.3, 128 x 128 30.4, in two parts 36.8; 4096
// x 512 to 512: 64 x 64 7.8, 128 x 128 11.3.  fp32: 128 x 4096 to 4096: 128 x 64 148 in one, 46.3 in 4, 38.5 in 8, 128 x 128 38.6 in 16; 256 x 25088 to 4096: 128 x 128 301 in 8, 297 in 12, 128 x 64 341 in 8; 2000 x
// 2048 to 2048: 128 x 128 123 in one, 106 in 2.
// near: whether a tile's rows of both factors lie within 2^32 bytes.
struct Tile {
    uint32_t out, token, most;
    double a, b;
};

Plan plan_of(size_t tokens, size_t outs, size_t cols, uint32_t dtype, bool near)
{
    static constexpr Tile kHalf[] = {{64, 64, 5, 0.28, 0.17}, {128, 64, 3, 0.27, 0.26}, {128, 128, 2, 0.52, 0.26}}, kFull[] = {{128, 64, 4, 0.5, 0.63}, {128, 128, 3, 1.0, 0.8}};
    const bool fp32 = dtype == OGQ_FP32;
    const uint32_t depth = fp32 ? 32 : 64, kinds = fp32 ? 2 : 3;
    const uint64_t steps = ceil_div(cols, depth);
    Plan p{};
    double least = 1e300;
    if (!fp32 && near && cols >= 512 && tokens > 128 && outs > 128) {
        const uint64_t tiles = ceil_div(outs, 256) * ceil_div(tokens, 256);
        least = (double)ceil_div(tiles, 256) * ((double)steps * 1.6 + 10.0);
        p = {256, 256, (uint32_t)ceil_div(outs, 256), (uint32_t)ceil_div(tokens, 256), (uint32_t)cols, 1, 1};
    }
    for (uint32_t n = 0; n < kinds; ++n) {
        const Tile& t = fp32 ? kFull[n] : kHalf[n];
        const uint64_t tiles = ceil_div(outs, t.out) * ceil_div(tokens, t.token);
        for (uint64_t parts = 1; parts <= 32 && (parts == 1 || (parts <= steps / 2 && tiles * parts <= 1024)); ++parts) {
            const uint64_t each = ceil_div(steps, parts), slots = 256 * t.most, full = tiles * parts / slots, rest = tiles * parts % slots;
            const bool teams = !fp32 && t.token == 64 && tiles * parts <= 256 && each >= 4;
            const double step = ((double)full * (t.a + t.b * (double)t.most) + (rest != 0 ? t.a + t.b * (double)ceil_div(rest, 256) : 0.0)) * (teams ? 0.7 : 1.0);
            const double join = parts > 1 ? 3.5 + 0.3 * (double)parts + 2e-6 * (double)parts * (double)tokens * (double)outs : 0.0, cost = step * (double)each + join;
            if (cost >= least) continue;
            least = cost;
            p = {t.out, t.token, (uint32_t)ceil_div(outs, t.out), (uint32_t)ceil_div(tokens, t.token), steps == 0 ? depth : (uint32_t)(each * depth), 1, teams ? 2u : 1u};
            p.parts = steps == 0 ? 1 : (uint32_t)ceil_div(cols, p.part);
        }
    }
    return p;
}

uint32_t pitch_of(size_t outs) { return (uint32_t)(ceil_div(outs, 8) * 8); }

}  // namespace

template <class T>
void launch_join_parts(const LinearShape& s, const Epilogue<T>& e, hipStream_t st)
{
    const uint32_t per_token = (uint32_t)ceil_div(s.outs, kPiece<T>);
    launch_kernel(join_parts_kernel<T>, grid_of(ceil_div((uint64_t)s.tokens * per_token, kBlock)), dim3(kBlock), st, s, e, per_token);
}

template void launch_join_parts<float>(const LinearShape&, const Epilogue<float>&, hipStream_t);
template void launch_join_parts<__bf16>(const LinearShape&, const Epilogue<__bf16>&, hipStream_t);
template void launch_join_parts<_Float16>(const LinearShape&, const Epilogue<_Float16>&, hipStream_t);

size_t linear_workspace(size_t tokens, size_t outs, size_t cols, uint32_t dtype, bool transposed)
{
    const uint32_t parts = !few_tokens(tokens, outs, cols, dtype, transposed) ? plan_of(tokens, outs, cols, dtype, true).parts : transposed ? few_parts(outs, cols).parts : 1;
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
        if (few_tokens(tokens, outs, cols, dtype, transposed)) {
            if constexpr (sizeof(T) == 4)
                if (transposed) {
                    launch_few_across(from, w, s, e, static_cast<float*>(workspace), st);
                    return;
                }
            launch_few(from, w, s, e, st);
            return;
        }
        // (with rows that are not near, what takes large tiles elsewhere takes others in one part: the workspace is what the sizes say)
        const bool near = x.stride < ((size_t)1 << 23) && weight.stride < ((size_t)1 << 23) && outs < ((size_t)1 << 30);
        Plan plan = plan_of(tokens, outs, cols, dtype, true);
        if (plan.tile_out == 256 && !near) {
            plan = plan_of(tokens, outs, cols, dtype, false);
            plan.part = (uint32_t)cols, plan.parts = 1;
        }
        s.tiles_out = plan.tiles_out, s.tiles_token = plan.tiles_token, s.part = plan.part, s.parts = plan.parts;
        s.sums = plan.parts > 1 ? static_cast<float*>(workspace) : nullptr;
        auto kernel = transposed ? linear_kernel<T, 128, 128, true> : linear_kernel<T, 128, 128, false>;
        if (plan.tile_token == 64) kernel = transposed ? linear_kernel<T, 128, 64, true> : linear_kernel<T, 128, 64, false>;
        if constexpr (sizeof(T) == 2)
            if (plan.tile_out == 64) kernel = transposed ? linear_kernel<T, 64, 64, true> : linear_kernel<T, 64, 64, false>;
        if constexpr (sizeof(T) == 2)
            if (plan.tile_out == 256) {
                const bool whole = cols % 64 == 0 && ((reinterpret_cast<uintptr_t>(from) | reinterpret_cast<uintptr_t>(w) | x.stride * 2 | weight.stride * 2) & 15) == 0 && (!transposed || outs % 8 == 0);
                if (whole) {
                    launch_kernel(transposed ? direct_linear_kernel<T, true> : direct_linear_kernel<T, false>, dim3(s.tiles_out * s.tiles_token < 256 ? s.tiles_out * s.tiles_token : 256),
                                  dim3(256), st, from, w, s, e);
                    return;
                }
                kernel = transposed ? large_linear_kernel<T, true> : large_linear_kernel<T, false>;
            }
        if constexpr (sizeof(T) == 2) {
            if (plan.teams == 2) {
                kernel = transposed ? linear_kernel<T, 128, 64, true, 2> : linear_kernel<T, 128, 64, false, 2>;
                if (plan.tile_out == 64) kernel = transposed ? linear_kernel<T, 64, 64, true, 2> : linear_kernel<T, 64, 64, false, 2>;
            }
        }
        launch_kernel(kernel, grid_of((uint64_t)s.tiles_out * s.tiles_token * s.parts), dim3(256 * plan.teams), st, from, w, s, e);
        if (s.sums != nullptr) launch_join_parts(s, e, st);
    });
}

}  // namespace ogq
