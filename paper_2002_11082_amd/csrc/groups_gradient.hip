// libogq_groups: the gradient of a linear layer's weights from the gradient of its outputs and its 8-bit inputs,
//   dw[o][i] = sum over t of dy[t][o] * x^[t][i].
//
// A workgroup holds a tile of sums in registers and goes along t in steps of 32 rows.  In memory both factors have the summed index
// outside; the matrix instruction wants eight of it per lane.  The rows go to LDS as they are and come back transposed (ds_read_b64_tr_b16: 16
// lanes read four rows of 16 values and receive four values of one column each).  The codes become 16-bit values on the way to LDS, exactly.
#include "groups_common.h"

namespace ogq {

namespace {

constexpr int kDepth = 32;   // rows of a step
constexpr int kSmall = 128, kLarge = 256;  // inputs and outputs of a workgroup's sums

typedef short s16x8 __attribute__((ext_vector_type(8)));

// A row of a tile in LDS is 8 or 16 chunks of 32 bytes (16 values); chunk c of row k lies at c ^ twist(k): what half a wavefront reads at once, two neighbouring chunks of
// four rows, lies in different banks.
__device__ __forceinline__ uint32_t twist(uint32_t k) { return (k & 3u) * 2u; }

// Sixteen values of a row of dy in the pieces that the matrix cores take: one for 16-bit types, three for fp32.
template <class T>
struct Rows16 {
    static constexpr int kPieces = 1;
    uint32_t raw[8];
    __device__ __forceinline__ void load(const T* from) { memcpy(raw, from, 32); }
    __device__ __forceinline__ void load(const T* from, int valid)
    {
        if (valid >= 16) load(from);
        else load_some<T, 16>(from, valid, raw);
    }
    __device__ __forceinline__ void store(char* to, int) const { memcpy(to, raw, 32); }
    // fp16 in two pieces of bf16, whose sum each value is.
    __device__ __forceinline__ void store_split(char* to, int plane) const
    {
        T v[16];
        memcpy(v, raw, 32);
        uint32_t w[2][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t a[3], b[3];
            split3((float)v[2 * i], a[0], a[1], a[2]);
            split3((float)v[2 * i + 1], b[0], b[1], b[2]);
#pragma unroll
            for (int p = 0; p < 2; ++p) w[p][i] = __builtin_amdgcn_perm(b[p], a[p], 0x07060302u);
        }
#pragma unroll
        for (int p = 0; p < 2; ++p) memcpy(to + p * plane, w[p], 32);
    }
};
template <>
struct Rows16<float> {
    static constexpr int kPieces = 3;
    uint32_t raw[16];
    __device__ __forceinline__ void load(const float* from) { memcpy(raw, from, 64); }
    __device__ __forceinline__ void load(const float* from, int valid)
    {
        if (valid >= 16) load(from);
        else load_some<float, 16>(from, valid, raw);
    }
    __device__ __forceinline__ void store(char* to, int plane) const
    {
        uint32_t w[3][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t a[3], b[3];
            split3(__uint_as_float(raw[2 * i]), a[0], a[1], a[2]);
            split3(__uint_as_float(raw[2 * i + 1]), b[0], b[1], b[2]);
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
    uint32_t w[8];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        float v[4];
        decode8(h == 0 ? codes.x : h == 1 ? codes.y : h == 2 ? codes.z : codes.w, byte, v);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if constexpr (__is_same(T, _Float16)) {
                const auto a = __builtin_amdgcn_cvt_pkrtz(v[2 * i], v[2 * i + 1]);
                memcpy(&w[2 * h + i], &a, 4);
            } else {  // the upper halves, exactly
                w[2 * h + i] = __builtin_amdgcn_perm(__float_as_uint(v[2 * i + 1]), __float_as_uint(v[2 * i]), 0x07060302u);
            }
        }
    }
    memcpy(to, w, 32);
}

// An fp16 tensor's exponents as bytes: the lowest, and how far behind it the others are.  What a group with another one holds (NaN among it) may lie outside of fp16.
constexpr uint32_t kHalfLow = ExponentLimits<_Float16, 8>::kLow + 127, kHalfSpan = ExponentLimits<_Float16, 8>::kHigh - ExponentLimits<_Float16, 8>::kLow;

template <int ROW_BYTES>
__device__ __forceinline__ s16x8 read_transposed(const char* at)
{
    typedef __attribute__((address_space(3))) s16x4* Lds;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)at), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + 4 * ROW_BYTES));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

template <class T>
__device__ __forceinline__ f32x16 multiply_add32(s16x8 a, s16x8 b, f32x16 c)
{
    if constexpr (__is_same(T, _Float16)) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

struct GradientShape {
    uint32_t rows, outs, cols, groups, group_log2;
    uint32_t tiles_in, tiles_out;  // tiles along the inputs and the outputs
    uint32_t part;                 // rows of a part of the sum, a multiple of kDepth
    bool stream;                   // whether the caches need not keep the sums
    uint64_t dy_stride, out_stride, out_part;
};

// Four neighbouring sums into a row of dw, or added to it, at once where the row has all four (the hardware takes 16 bytes at any value's address: rows of 2589 sums
// 20.7 us and 12.8).
__device__ __forceinline__ void store_sums(float* row, uint32_t at, uint32_t cols, bool accumulate, bool stream, f32x4 v)
{
    float* p = row + at;
    if (at + 4 <= cols) {
        if (accumulate) {
            f32x4 held;
            memcpy(&held, p, sizeof held);
            v += held;
        }
        if (stream) __builtin_nontemporal_store(__builtin_bit_cast(Words, v), reinterpret_cast<Words*>(p));
        else memcpy(p, &v, sizeof v);
        return;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (at + r < cols) p[r] = accumulate ? p[r] + v[r] : v[r];
}

// What a workgroup's 256 threads bring of both factors to LDS, a step (kDepth rows) at a time: sixteen values of a row to a thread and unit, on their way in SETS sets
// of registers.  Tiles of IN inputs and OUT outputs.
template <class T, int IN, int OUT, int SETS>
struct Feeder {
    static constexpr int kInUnits = IN / 128, kOutUnits = OUT / 128;
    static constexpr int kInRows = kDepth / kInUnits, kOutRows = kDepth / kOutUnits;  // of a unit
    static constexpr int kInBytes = IN * 2, kOutBytes = OUT * 2;                      // of a row in LDS
    static constexpr int kInPlane = kDepth * kInBytes, kOutPlane = kDepth * kOutBytes;
    static constexpr int kStage = kInPlane + Rows16<T>::kPieces * kOutPlane;  // of LDS: the codes as values, then the pieces of dy
    const T* dy;
    const uint8_t *codes, *exponents;
    uint64_t dy_stride, pitch;
    uint32_t groups, group_log2, first, last, in_row, out_row, i_mine, o_mine;
    uint32_t at_codes, at_byte, at_dy;
    uint32_t whole;  // steps that are there in all rows
    bool readable;   // whether these can be read without asking
    bool has_codes;
    uint64_t outside = 0;  // fp16: the lanes that have brought a group whose exponent is none of an fp16 tensor (in scalar registers)
    int valid;
    char *in_to, *out_to;
    Rows16<T> g[SETS][kOutUnits];
    uint4 q[SETS][kInUnits];
    uint32_t byte[SETS][kInUnits];

    __device__ __forceinline__ Feeder(const T* dy_, const uint8_t* codes_, const uint8_t* exponents_, const GradientShape& s, uint32_t i0, uint32_t o0, uint32_t first_,
                                      uint32_t last_, uint32_t thread, char* lds)
        : dy(dy_), codes(codes_), exponents(exponents_), dy_stride(s.dy_stride), pitch((uint64_t)s.groups << s.group_log2), groups(s.groups),
          group_log2(s.group_log2), first(first_), last(last_)
    {
        const uint32_t in_chunk = thread % (IN / 16), out_chunk = thread % (OUT / 16);
        in_row = thread / (IN / 16), out_row = thread / (OUT / 16);
        i_mine = i0 + in_chunk * 16, o_mine = o0 + out_chunk * 16;
        has_codes = i_mine < pitch;
        valid = o_mine >= s.outs ? 0 : (int)min(16u, s.outs - o_mine);
        // (a unit's rows are a multiple of 16, which twist does not see)
        in_to = lds + in_row * kInBytes + ((in_chunk ^ twist(in_row)) * 32);
        out_to = lds + kInPlane + out_row * kOutBytes + ((out_chunk ^ twist(out_row)) * 32);
        // What lies behind the last input or output is any value that is there: its sums are not stored.  A thread whose sixteen outputs reach beyond the
        // last reads on into the next row; the tensor's last rows are then left to the steps that ask.
        const bool partial = o0 + OUT > s.outs && s.outs % 16 != 0;
        whole = first < last ? (last - first) / kDepth : 0;
        if (partial && whole != 0 && first + whole * kDepth == s.rows) --whole;
        // (a thread's place in a unit's rows is held in 32 bits; reading on needs a next row.  `whole` stays what the sizes make it: two teams share the rows by it.)
        readable = (dy_stride | pitch) < (1u << 24) && !(partial && dy_stride < 16);
        const uint32_t i = has_codes ? i_mine : i0, o = valid != 0 ? o_mine : o0;
        at_codes = in_row * (uint32_t)pitch + i;
        at_byte = in_row * groups + (i >> group_log2);
        at_dy = out_row * (uint32_t)dy_stride + o;
    }
    // Of step n, of the whole ones.  (One behind the last of them is the last one again, and not used.)
    __device__ __forceinline__ void fetch_codes(uint32_t n, int set, int u)
    {
        const uint32_t t = first + min(n, whole - 1) * kDepth + kInRows * u;
        q[set][u] = *reinterpret_cast<const uint4*>(codes + t * pitch + at_codes);
        byte[set][u] = (exponents + (uint64_t)t * groups)[at_byte];
    }
    __device__ __forceinline__ void fetch_dy(uint32_t n, int set, int u)
    {
        const uint32_t t = first + min(n, whole - 1) * kDepth + kOutRows * u;
        g[set][u].load(dy + t * dy_stride + at_dy);
    }
    __device__ __forceinline__ void bring_codes(uint32_t stage, int set, int u)
    {
        store_codes<T>(q[set][u], byte[set][u], in_to + stage * kStage + u * kInRows * kInBytes);
        if constexpr (__is_same(T, _Float16)) outside |= __builtin_amdgcn_ballot_w64(byte[set][u] - kHalfLow > kHalfSpan);
    }
    __device__ __forceinline__ void bring_dy(uint32_t stage, int set, int u) { g[set][u].store(out_to + stage * kStage + u * kOutRows * kOutBytes, kOutPlane); }
    __device__ __forceinline__ void fetch(uint32_t n, int set)
    {
#pragma unroll
        for (int u = 0; u < kOutUnits; ++u) fetch_dy(n, set, u);
#pragma unroll
        for (int u = 0; u < kInUnits; ++u) fetch_codes(n, set, u);
    }
    __device__ __forceinline__ void bring(uint32_t stage, int set)
    {
#pragma unroll
        for (int u = 0; u < kOutUnits; ++u) bring_dy(stage, set, u);
#pragma unroll
        for (int u = 0; u < kInUnits; ++u) bring_codes(stage, set, u);
    }
    // Rows t ... of any step, what is not there as 0, on their way.
    __device__ __forceinline__ void fetch_asking(uint32_t t)
    {
#pragma unroll
        for (int u = 0; u < kInUnits; ++u) {
            const uint32_t mine = t + in_row + kInRows * u;
            q[0][u] = make_uint4(0, 0, 0, 0);
            byte[0][u] = 127;
            if (mine < last && has_codes) {
                q[0][u] = *reinterpret_cast<const uint4*>(codes + mine * pitch + i_mine);
                byte[0][u] = exponents[(uint64_t)mine * groups + (i_mine >> group_log2)];
            }
        }
#pragma unroll
        for (int u = 0; u < kOutUnits; ++u) {
            const uint32_t mine = t + out_row + kOutRows * u;
            g[0][u].load(dy + mine * dy_stride + o_mine, mine < last ? valid : 0);
        }
    }
    __device__ __forceinline__ void bring_asking(uint32_t t)
    {
        fetch_asking(t);
        bring(0, 0);
    }
    // The same for fp16 gradients and any checkpoint: both factors as bf16, dy in two pieces.
    static_assert(kInPlane + 2 * kOutPlane <= SETS * kStage || !__is_same(T, _Float16));
    __device__ __forceinline__ void bring_split(uint32_t t)
    {
        fetch_asking(t);
#pragma unroll
        for (int u = 0; u < kOutUnits; ++u) g[0][u].store_split(out_to + u * kOutRows * kOutBytes, kOutPlane);
#pragma unroll
        for (int u = 0; u < kInUnits; ++u) store_codes<__bf16>(q[0][u], byte[0][u], in_to + u * kInRows * kInBytes);
    }
};

// Where a lane finds its part of the operands of v_mfma_f32_32x32x16: lane l holds k = l / 32 * 8 ... of column l % 32.  Operand n begins at chunk first + 2 n of a row.
template <int N, int ROW_BYTES>
struct OperandPlaces {
    const char* at[N];
    __device__ __forceinline__ OperandPlaces(const char* plane, uint32_t lane, uint32_t first)
    {
        const uint32_t k = (lane >> 5) * 8 + ((lane >> 2) & 3), f = twist(k), side = (lane >> 4) & 1;
#pragma unroll
        for (int n = 0; n < N; ++n) at[n] = plane + k * ROW_BYTES + (lane & 3) * 8 + (((first + 2 * n + side) ^ f) * 32);
    }
    // Operand n of the upper or lower 16 rows of a step, `bytes` behind the plane that the places are in.
    __device__ __forceinline__ s16x8 read(int n, int half, uint32_t bytes) const { return read_transposed<ROW_BYTES>(at[n] + bytes + half * 16 * ROW_BYTES); }
};

// The sums of a wavefront again, for fp16 gradients and a checkpoint that holds what fp16 does not (one of a bf16 or fp32 tensor): as products of bf16, of which dy takes two.  All of the
// workgroup's threads call it where one has met such a group; nothing of what they hold but the tile is needed, so that the usual way keeps its registers.  4096 x 4096 sums of 4096 rows 129 us, and 545
// where every tile is made again.
template <class FEED, int TEAMS, int NI, int NO>
__device__ __forceinline__ void sums_of_any_checkpoint(const _Float16* dy, const uint8_t* codes, const uint8_t* exponents, const GradientShape& s, uint32_t i0, uint32_t o0,
                                                       uint32_t first, uint32_t last, uint32_t thread, uint32_t team, char* lds, f32x16 (&sum)[NI][NO])
{
    asm("" : "+v"(thread));  // (the places below are made here, not held since the start)
    FEED feed(dy, codes, exponents, s, i0, o0, first, last, thread, lds);
    const OperandPlaces<NI, FEED::kInBytes> from_in(lds, thread & 63, (thread >> 6 & 1) * NI * 2);
    const OperandPlaces<NO, FEED::kOutBytes> from_out(lds + FEED::kInPlane, thread & 63, (thread >> 7) * NO * 2);
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NO; ++j) sum[i][j] = f32x16{};
    for (uint32_t t = first + team * kDepth; t < last + team * kDepth; t += TEAMS * kDepth) {
        if (t < last) feed.bring_split(t);
        __syncthreads();
        if (t < last) {
#pragma unroll 1
            for (int h = 0; h < 2; ++h)
#pragma unroll 1
                for (int p = 1; p >= 0; --p)
#pragma unroll
                    for (int j = 0; j < NO; ++j) {
                        const s16x8 b = from_out.read(j, h, p * FEED::kOutPlane);
#pragma unroll
                        for (int i = 0; i < NI; ++i) sum[i][j] = multiply_add32<__bf16>(from_in.read(i, h, 0), b, sum[i][j]);
                    }
        }
        __syncthreads();
    }
}

// The sums of a wavefront, 32 * NI inputs from i and 32 * NO outputs from o, to dw or the workspace.  A lane holds pieces of 16 bytes of one row; through LDS (`space`, 4608
// bytes of the wavefront's own) eight lanes get the 128 bytes of one, so that lines are written whole.
constexpr int kTurnRow = 144, kTurnBytes = 32 * kTurnRow;  // (16 bytes between rows: eight rows' pieces in different banks)

__device__ __forceinline__ void wavefront_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <int NI, int NO>
__device__ __forceinline__ void store_tile(const f32x16 (&sum)[NI][NO], uint32_t i, uint32_t o, uint32_t lane, const GradientShape& s, bool accumulate, float* out, char* space)
{
#pragma unroll
    for (int b = 0; b < NO; ++b)
#pragma unroll
        for (int a = 0; a < NI; ++a) {
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const f32x4 v = {sum[a][b][4 * m], sum[a][b][4 * m + 1], sum[a][b][4 * m + 2], sum[a][b][4 * m + 3]};
                *reinterpret_cast<f32x4*>(space + (lane & 31) * kTurnRow + 32 * m + (lane >> 5) * 16) = v;
            }
            wavefront_sync();
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const uint32_t row = 8 * m + (lane >> 3);
                const f32x4 v = *reinterpret_cast<const f32x4*>(space + row * kTurnRow + (lane & 7) * 16);
                if (o + 32 * b + row < s.outs) store_sums(out + (o + 32 * b + row) * s.out_stride, i + 32 * a + (lane & 7) * 4, s.cols, accumulate, s.stream, v);
            }
            wavefront_sync();
        }
}

// Tiles of IN x OUT sums, a quarter in each of a team's four wavefronts; two teams have half of the rows each.  `out` is dw, or the workspace where the sum is cut into parts (out_part
// values from one part to the next).  Bound by LDS, to which every step goes and from which each factor is read twice, where a CU has two workgroups, and by a step's latency where it has
// one: 2048 x 2048 sums of 8192 rows in bf16 91 us, 755 TFLOP/s; fp32, whose three products count: the same 250 us, 825 TFLOP/s, and 4096 x 4096 of 4096 rows in tiles of 256 x 128 345 us, 1190 TFLOP/s;
// 4096 x 25088 of 256 rows 180 us, 870 TFLOP/s beside 2.3 TB/s of sums written.
template <class T, int IN, int OUT, int GROUPS, int TEAMS>
__global__ __launch_bounds__(256 * TEAMS, GROUPS * TEAMS) void weight_gradient_kernel(const T* dy, const uint8_t* codes, const uint8_t* exponents, GradientShape s,
                                                                              bool accumulate, float* out)
{
    constexpr int kPieces = Rows16<T>::kPieces, kSets = kPieces == 1 || IN == kSmall ? 2 : 1, kIn = IN / 64, kOut = OUT / 64;
    using Feed = Feeder<T, IN, OUT, kSets>;
    __shared__ __align__(16) char all_lds[TEAMS * kSets * Feed::kStage];
    __shared__ uint32_t any_outside;
    if (__is_same(T, _Float16) && threadIdx.x == 0) any_outside = 0;
    const uint32_t tiles = s.tiles_in * s.tiles_out, tile = blockIdx.x % tiles, part = blockIdx.x / tiles;
    const uint32_t i0 = tile % s.tiles_in * IN, o0 = tile / s.tiles_in * OUT;  // (neighbours along a row of sums: 8192 x 16384 of 32 rows 97 us, 131 in tile_of's order)
    const uint32_t first = part * s.part, last = min(s.rows, first + s.part);
    const uint32_t wave = TEAMS == 1 ? threadIdx.x >> 6 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = TEAMS == 1 ? 0 : wave >> 2;
    const uint32_t lane = threadIdx.x & 63, i_wave = (wave & 1) * (IN / 2), o_wave = (wave >> 1 & 1) * (OUT / 2);
    char* lds = all_lds + team * kSets * Feed::kStage;
    Feed feed(dy, codes, exponents, s, i0, o0, first, last, TEAMS == 1 ? threadIdx.x : threadIdx.x & 255, lds);
    const uint32_t share = feed.whole / TEAMS;  // steps of a team, one behind the other; what is left goes round
    feed.first += team * share * kDepth;
    feed.whole = feed.readable ? share : 0;
    const OperandPlaces<kIn, Feed::kInBytes> from_in(lds, lane, i_wave / 16);
    const OperandPlaces<kOut, Feed::kOutBytes> from_out(lds + Feed::kInPlane, lane, o_wave / 16);
    f32x16 sum[kIn][kOut] = {};
    const auto products = [&](uint32_t stage) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            s16x8 a[kIn];
#pragma unroll
            for (int i = 0; i < kIn; ++i) a[i] = from_in.read(i, h, stage * Feed::kStage);
#pragma unroll
            for (int p = kPieces - 1; p >= 0; --p)
#pragma unroll
                for (int j = 0; j < kOut; ++j) {
                    const s16x8 b = from_out.read(j, h, stage * Feed::kStage + p * Feed::kOutPlane);
#pragma unroll
                    for (int i = 0; i < kIn; ++i) sum[i][j] = multiply_add32<T>(a[i], b, sum[i][j]);
                }
        }
    };
    // Two stages of LDS and one barrier a step: while one step is multiplied, the next comes to LDS and two more are on their way (1733 x 1216 sums of 1249 rows in bf16 23.4 us;
    // 25.0 with the step itself brought ahead of the barrier, 24.6 with the next one brought ahead of the products).  fp32 in tiles of 256 x 128: one stage, since a second would
    // fill LDS (4096 x 4096 sums of 4096 rows 364 us, 414 with two; in tiles of 128 x 128, of which a CU has one or two, 2048 x 2048 of 512 rows 33.0 us with one and 27.0 with two).
    const auto step = [&](uint32_t n, int set) __attribute__((always_inline)) {
        if constexpr (kSets == 1) {
            __syncthreads();
            feed.bring(0, 0);
            __syncthreads();
            feed.fetch(n + 1, 0);
            products(0);
        } else {
            __syncthreads();
            products(set);
            feed.bring(set ^ 1, set ^ 1);
            feed.fetch(n + 3, set ^ 1);
        }
    };
    if (feed.whole != 0) {
#pragma unroll
        for (int n = 0; n < kSets; ++n) feed.fetch(n, n);
        if constexpr (kSets == 2) {
            feed.bring(0, 0);
            feed.fetch(2, 0);
        }
        uint32_t n = 0;
        for (; n + kSets <= feed.whole; n += kSets) {
            step(n, 0);
            if constexpr (kSets == 2) step(n + 1, 1);
        }
        if (n < feed.whole) step(n, 0);
    }
    for (uint32_t n = feed.whole; first + TEAMS * n * kDepth < last; ++n) {
        const uint32_t t = n < share ? feed.first + n * kDepth : first + (TEAMS * n + team) * kDepth;
        __syncthreads();
        if (t < last) feed.bring_asking(t);
        __syncthreads();
        if (t < last) products(0);
    }
    if (__is_same(T, _Float16) && feed.outside != 0) any_outside = 1;
    __syncthreads();
    if constexpr (__is_same(T, _Float16))
        if (any_outside != 0) sums_of_any_checkpoint<Feed, TEAMS>(dy, codes, exponents, s, i0, o0, first, last, (wave & 3) * 64 + lane, team, lds, sum);
    char* space = all_lds + wave * kTurnBytes;
    if constexpr (TEAMS == 1) {
        store_tile(sum, i0 + i_wave, o0 + o_wave, lane, s, accumulate, out + part * s.out_part, space);
    } else {
        // each team stores the sums of one half of the outputs, and has the other one's share of them through LDS
        static_assert(TEAMS == 2 && kOut == 2 && sizeof all_lds >= 2 * 256 * kIn * 64);
        f32x4* exchange = reinterpret_cast<f32x4*>(all_lds);
        const auto place = [&](uint32_t of, int i, int m) { return ((of * 4 + (wave & 3)) * kIn + i) * 256 + m * 64 + lane; };
        const auto send = [&](const f32x16& v, int i) __attribute__((always_inline)) {
#pragma unroll
            for (int m = 0; m < 4; ++m) exchange[place(team, i, m)] = f32x4{v[4 * m], v[4 * m + 1], v[4 * m + 2], v[4 * m + 3]};
        };
        f32x16 mine[kIn][1];
#pragma unroll
        for (int i = 0; i < kIn; ++i) {
            if (team == 0) send(sum[i][1], i), mine[i][0] = sum[i][0];
            else send(sum[i][0], i), mine[i][0] = sum[i][1];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kIn; ++i)
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const f32x4 v = exchange[place(team ^ 1, i, m)];
#pragma unroll
                for (int r = 0; r < 4; ++r) mine[i][0][4 * m + r] += v[r];
            }
        __syncthreads();
        store_tile(mine, i0 + i_wave, o0 + o_wave + 32 * team, lane, s, accumulate, out + part * s.out_part, space);
    }
}

// Workgroups go to the eight XCDs in turn, each with an L2 of its own: an XCD takes neighbouring tiles, four along the inputs by eight along the outputs at a
// time.
__device__ __forceinline__ uint2 tile_of(uint32_t id, uint32_t tiles_in, uint32_t tiles_out)
{
    constexpr uint32_t kXcds = 8, kWide = 4;
    const uint32_t tiles = tiles_in * tiles_out, each = tiles / kXcds, more = tiles % kXcds, xcd = id % kXcds;
    const uint32_t n = xcd * each + min(xcd, more) + id / kXcds;
    const uint32_t panel = n / (kWide * tiles_out), rest = n % (kWide * tiles_out), width = min(kWide, tiles_in - panel * kWide);
    return make_uint2(panel * kWide + rest % width, rest / width);
}

// The order of instructions around eight products, which the matrix core takes 32 cycles for each: behind each of them, reads of operands, a few vector
// instructions, and behind some a write to LDS and a load.
template <int READS, int VECTOR, int WRITES>
__device__ __forceinline__ void interleave()
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                          // matrix
        if (READS >= 8) __builtin_amdgcn_sched_group_barrier(0x100, READS / 8, 0);  // LDS read
        if (i < READS % 8) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        if (VECTOR != 0) __builtin_amdgcn_sched_group_barrier(0x002, VECTOR, 0);  // vector
        if (WRITES == 4 ? i % 2 == 1 : WRITES == 2 ? i >= 6 : false) {
            __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);  // LDS write
            __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);  // memory read
        }
    }
    __builtin_amdgcn_sched_barrier(0);
}

// Tiles of 256 x 256 sums, 128 x 128 in each of four wavefronts, one to a SIMD, which has all of its registers: 256 hold the sums.  While a wavefront
// multiplies what it holds of a step, it reads its share of the next one from LDS and brings the one after that there; the step behind that is on its
// way from memory.  One barrier a step, behind which all that the matrix cores need is in registers.
// 16384 x 4096 sums of 8192 rows in bf16 890 us, 1.24 PFLOP/s; the library's product of two bf16 matrices of these sizes takes 907.  The matrix cores are busy for 0.64 of the
// cycles, at a clock that is down to 1.7 GHz under their load.
template <class T>
__global__ __launch_bounds__(256, 1) void large_weight_gradient_kernel(const T* dy, const uint8_t* codes, const uint8_t* exponents, GradientShape s,
                                                                       bool accumulate, float* out)
{
    static_assert(Rows16<T>::kPieces == 1);
    using Feed = Feeder<T, kLarge, kLarge, 2>;
    __shared__ __align__(16) char lds[2 * Feed::kStage];
    __shared__ uint32_t any_outside;
    if (__is_same(T, _Float16) && threadIdx.x == 0) any_outside = 0;
    const uint32_t tiles = s.tiles_in * s.tiles_out, part = blockIdx.x / tiles;
    const uint2 tile = tile_of(blockIdx.x % tiles, s.tiles_in, s.tiles_out);
    const uint32_t i0 = tile.x * kLarge, o0 = tile.y * kLarge;
    const uint32_t first = part * s.part, last = min(s.rows, first + s.part);
    const uint32_t lane = threadIdx.x & 63, i_wave = (threadIdx.x >> 6 & 1) * 128, o_wave = (threadIdx.x >> 7) * 128;
    Feed feed(dy, codes, exponents, s, i0, o0, first, last, threadIdx.x, lds);
    if (!feed.readable) feed.whole = 0;
    const OperandPlaces<4, Feed::kInBytes> from_in(lds, lane, i_wave / 16);
    const OperandPlaces<4, Feed::kOutBytes> from_out(lds + Feed::kInPlane, lane, o_wave / 16);
    using Operands = s16x8[4][2];
    // Operand n of a factor.
    const auto read = [&](Operands& r, const auto& from, uint32_t stage, int n) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) r[n][h] = from.read(n, h, stage * Feed::kStage);
    };
    f32x16 sum[4][4] = {};
    // An eighth of a step's products.
    const auto products = [&](const Operands& in, const Operands& o, int eighth) __attribute__((always_inline)) {
        const int h = eighth / 4, i = eighth % 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[i][j] = multiply_add32<T>(in[i][h], o[j][h], sum[i][j]);
    };
    // One step: what it multiplies is held in `in` and `o`, the next one's goes to the others.  Step n + 1 is in LDS, step n + 2 goes where step n was, and
    // step n + 4 sets off.
    const auto step = [&](uint32_t n, uint32_t here, Operands& in, Operands& o, Operands& next_in, Operands& next_o) __attribute__((always_inline)) {
        const uint32_t next = here ^ 1;
        read(next_in, from_in, next, 0), read(next_o, from_out, next, 0), read(next_o, from_out, next, 1);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            feed.bring_dy(here, here, u);
            feed.fetch_dy(n + 4, here, u);
        }
        products(in, o, 0), products(in, o, 1);
        interleave<12, 2, 4>();
        read(next_o, from_out, next, 2), read(next_o, from_out, next, 3), read(next_in, from_in, next, 1);
        feed.bring_codes(here, here, 0);
        feed.fetch_codes(n + 4, here, 0);
        products(in, o, 2), products(in, o, 3);
        interleave<12, 6, 2>();
        read(next_in, from_in, next, 2), read(next_in, from_in, next, 3);
        feed.bring_codes(here, here, 1);
        feed.fetch_codes(n + 4, here, 1);
        products(in, o, 4), products(in, o, 5);
        interleave<8, 6, 2>();
        // the barrier between the last products: those before it give the writes time, those behind it the other wavefronts
        products(in, o, 6);
        __builtin_amdgcn_sched_barrier(0);
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
        products(in, o, 7);
        __builtin_amdgcn_sched_barrier(0);
    };
    Operands a, b, na, nb;
    if (feed.whole != 0) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                feed.fetch_dy(n, n, u);
                feed.fetch_codes(n, n, u);
            }
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                feed.bring_dy(n, n, u);
                feed.fetch_dy(n + 2, n, u);
                feed.bring_codes(n, n, u);
                feed.fetch_codes(n + 2, n, u);
            }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k) read(a, from_in, 0, k), read(b, from_out, 0, k);
        __syncthreads();
        uint32_t n = 0;
        for (; n + 2 <= feed.whole; n += 2) {
            step(n, 0, a, b, na, nb);
            step(n + 1, 1, na, nb, a, b);
        }
        if (n < feed.whole) step(n, 0, a, b, na, nb);
    }
    for (uint32_t t = first + feed.whole * kDepth; t < last; t += kDepth) {
        feed.bring_asking(t);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k) read(a, from_in, 0, k), read(b, from_out, 0, k);
#pragma unroll
        for (int eighth = 0; eighth < 8; ++eighth) products(a, b, eighth);
        __syncthreads();
    }
    if (__is_same(T, _Float16) && feed.outside != 0) any_outside = 1;
    __syncthreads();
    if constexpr (__is_same(T, _Float16))
        if (any_outside != 0) sums_of_any_checkpoint<Feed, 1>(dy, codes, exponents, s, i0, o0, first, last, threadIdx.x, 0, lds, sum);
    store_tile(sum, i0 + i_wave, o0 + o_wave, lane, s, accumulate, out + part * s.out_part, lds + (threadIdx.x >> 6) * kTurnBytes);
}

// The parts of the sums, added in an order that their number alone decides.  Four sums to a thread, and four threads to them: each adds every fourth part.
__global__ __launch_bounds__(kBlock) void add_parts_kernel(const f32x4* parts, uint32_t number, uint32_t quads, uint32_t row_quads, uint32_t cols, bool accumulate,
                                                           float* dw, uint64_t dw_stride)
{
    __shared__ f32x4 shared[3][64];
    const uint32_t lane = threadIdx.x & 63, fourth = threadIdx.x >> 6, quad = blockIdx.x * 64 + lane;
    f32x4 v = {};
    if (quad < quads) {
        const f32x4* from = parts + quad;
#pragma unroll 8
        for (uint32_t n = fourth; n < number; n += 4) v += from[(uint64_t)n * quads];
    }
    if (fourth != 0) shared[fourth - 1][lane] = v;
    __syncthreads();
    if (fourth != 0 || quad >= quads) return;
#pragma unroll
    for (int n = 0; n < 3; ++n) v += shared[n][lane];
    const uint32_t o = quad / row_quads, at = quad % row_quads * 4;
    store_sums(dw + o * dw_stride, at, cols, accumulate, false, v);
}

uint32_t ceil_div(uint64_t a, uint64_t b) { return (uint32_t)((a + b - 1) / b); }

// Which tiles, and into how many parts a sum is cut.
// 16-bit types: 256 x 256 where such tiles fill most of the chip and a tile's own costs (its first steps, 256 KB of sums to store, with one workgroup on a CU) are
// spread over 640 rows: 4096 x 4096 sums of 512 rows 27.9 us and 28.6 with 128 x 128, of 768 34.6 and 38.3, of 2048 68 and 86; 8192 x 8192 of 512 rows 114 and 99, of
// 1024 167 and 195; 2560 x 4096 (160 tiles) of 4096 rows 100 and 115, 2048 x 4096 (128) of 2048 rows 58 and 47.  256 x 128: not better than 128 x 128 anywhere.
// fp32: 256 x 128 where such tiles fill the chip, because LDS holds three pieces of dy beside one of the inputs: 4096 x 4096 of 2048 rows 179 us and 256 with 128 x
// 128, of 128 rows 24.5 and 27.5, 4096 x 25088 of 256 rows 201 and 235; 1024 x 1024 (32 tiles) of 8192 rows in the best parts 68 and 77, 1000 x 4096 (128) of 1000 rows 47
// and 48, 512 x 512 of 1024 rows 20 and 17.
// 16 bits in tiles of 128 x 128: two teams of four wavefronts share a tile's rows where there are up to two workgroups to a CU, which leave its latencies open: 2048 x 2048 of 2048
// rows 28.3 us and 32.2 with one team, 1733 x 1216 of 1249 19.7 and 23.4, 2500 x 2500 (400 tiles) of 3000 64.8 and 69.0; but 2560 x 4096 (640) of 1024 37.5 and 35.8, 4096 x 4096 of
// 256 22.7 and 19.5, 512 x 512 of 32 rows, one step, 5.4 and 5.0, and 128 x 128 of 1200 in 18 parts 10.4 and 9.8.  fp32: 1733 x 1216 of 1249 rows 47 us with two teams in the best parts, 38.6 with one.
// A part's sums are written and read once more, 8 bytes each at about 3 TB/s; a workgroup's step of 32 rows takes 1.1 us in fp32 and 0.28 in 16 bits where it has the CU alone.  As
// many parts as make the two together little, up to 512 workgroups (256 of two teams) and 64 rows, where the steps saved are worth the second launch (4 us and what it reads).  us of both launches,
// by parts, at outputs x inputs of rows; 16 bits: 512 x 512 of 8192: 8 20.2, 12 18.7, 16 18.2 (16 by this), 24 23.0; 1024 x 1024 of 4096: 1 40.8, 2 29.4, 4 24.0 (4), 6 28.4; 864 x 977 of
// 1689: 1 21.2, 3 18.6 (4), 4 17.3, 6 21.8; 1024 x 1024 of 1024: 1 14.2 (1), 2 18.0; 221 x 7969 of 2280: 1 28.8, 2 26.3 (2), 3 31.0; 2048 x 2048 of 8192: 1 90.9 (1), 2 96.7; 200 x 333 of
// 16385: 8 26.7, 16 18.8, 24 17.3, 32 16.8, 42 17.5 (42), 48 22.7.
// fp32: 512 x 512 of 8192: 8 48.4, 16 33.1, 24 33.2, 32 31.6 (27); 1024 x 1024 of 4096: 4 53.6, 8 46.8 (8), 12 53.7; 864 x 977 of 1689: 1 67.3, 3 33.6, 6 29.4 (7), 8 27.7; 2048 x 2048 of
// 2048: 1 87.8, 2 75.6 (2), 3 82.8; 237 x 5423 of 416: 1 21.7, 2 23.2 (2), 4 22.2; 1024 x 1024 of 256: 1 13.2 (1), 2 17.5.  16 bits, 128 x 128 of 1200: 1 15.4, 4 10.2, 18 10.5 (18).
struct Plan {
    uint32_t tile_in, tile_out, tiles_in, tiles_out, parts, part, teams;
};

Plan plan_of(size_t rows, size_t outs, size_t cols, uint32_t dtype)
{
    const auto tiles_of = [&](uint32_t in, uint32_t out) { return (uint64_t)ceil_div(cols, in) * ceil_div(outs, out); };
    Plan p;
    p.tile_in = p.tile_out = kSmall;
    if (dtype == OGQ_FP32) {
        if (tiles_of(kLarge, kSmall) >= 256) p.tile_in = kLarge;
    } else if (tiles_of(kLarge, kLarge) >= 160 && rows >= 640) {
        p.tile_in = p.tile_out = kLarge;
    }
    p.tiles_in = ceil_div(cols, p.tile_in), p.tiles_out = ceil_div(outs, p.tile_out);
    const uint64_t tiles = tiles_of(p.tile_in, p.tile_out);
    p.parts = 1;
    const bool fp32 = dtype == OGQ_FP32;
    const uint64_t fill = fp32 ? 512 : 256;
    if (p.tile_in == kSmall && tiles < fill) {
        const uint64_t squared = (uint64_t)rows * (fp32 ? 25000 : 9000) / (outs * cols);
        const uint64_t most = rows / 64 < fill / tiles ? rows / 64 : fill / tiles;
        uint32_t parts = 1;
        while (parts < most && (uint64_t)(parts + 1) * (parts + 1) <= squared) ++parts;
        const double saved = rows / 32.0 * (fp32 ? 1.1 : 0.28) * (1.0 - 1.0 / parts), cost = 4.0 + 1e-6 * parts * (double)outs * (double)cols;
        if (saved > cost) p.parts = parts;
    }
    p.teams = !fp32 && p.tile_in == kSmall && tiles * p.parts <= 512 && rows / p.parts >= (p.parts == 1 ? kDepth + 1 : 6 * kDepth) ? 2 : 1;
    const uint32_t steps = kDepth * p.teams;  // (a step more for one team would be one that asks)
    p.part = ceil_div(ceil_div(rows, p.parts), steps) * steps;
    return p;
}

uint64_t pitch_of(size_t cols) { return (cols + 3) / 4 * 4; }

}  // namespace

size_t weight_gradient_workspace(size_t rows, size_t outs, size_t cols, uint32_t dtype)
{
    const uint32_t parts = plan_of(rows, outs, cols, dtype).parts;
    return parts > 1 ? parts * outs * pitch_of(cols) * sizeof(float) : 0;
}

void launch_weight_gradient(const Values& dy, uint32_t dtype, const Groups& x, size_t rows, size_t outs, size_t cols, const ogq_group_params_t* p,
                            bool accumulate, float* dw, size_t dw_stride, void* workspace, hipStream_t st)
{
    GradientShape s;
    s.rows = (uint32_t)rows, s.outs = (uint32_t)outs, s.cols = (uint32_t)cols;
    s.groups = ceil_div(cols, p->group_size);
    s.group_log2 = p->group_size == 32 ? 5 : p->group_size == 64 ? 6 : 7;
    const Plan plan = plan_of(rows, outs, cols, dtype);
    const uint32_t parts = plan.parts;  // (the last ones may be empty: their sums are 0)
    s.tiles_in = plan.tiles_in, s.tiles_out = plan.tiles_out, s.part = plan.part;
    s.dy_stride = dy.stride;
    s.out_stride = parts > 1 ? pitch_of(cols) : dw_stride;
    s.out_part = parts > 1 ? outs * s.out_stride : 0;
    float* out = parts > 1 ? static_cast<float*>(workspace) : dw;
    // Past the caches: 32 MB of sums, more than those of the eight XCDs hold, in rows of whole lines (4096 x 25088 of 256 rows in bf16 136 us and 92 past them, in fp32
    // 202 and 194; but 2700 x 6890, whose lines two rows share, of 9 rows 48.4 and 18.9 through them).
    s.stream = parts == 1 && outs * cols >= ((size_t)8 << 20) && ((reinterpret_cast<uintptr_t>(out) | s.out_stride * 4) & 63) == 0;
    const bool add = accumulate && parts == 1;
    const dim3 grid(s.tiles_in * s.tiles_out * parts), block(256 * plan.teams);
    const auto codes = static_cast<const uint8_t*>(x.codes);
    const auto go = [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        auto kernel = weight_gradient_kernel<T, kSmall, kSmall, sizeof(T) == 4 ? 2 : 3, 1>;
        if constexpr (sizeof(T) == 4) {
            if (plan.tile_in == kLarge) kernel = weight_gradient_kernel<T, kLarge, kSmall, 2, 1>;
        } else {
            if (plan.teams == 2) kernel = weight_gradient_kernel<T, kSmall, kSmall, 2, 2>;
            if (plan.tile_in == kLarge) kernel = large_weight_gradient_kernel<T>;
        }
        launch_kernel(kernel, grid, block, st, static_cast<const T*>(dy.data), codes, x.exponents, s, add, out);
    };
    if (dtype == OGQ_FP32) go((float*)nullptr);
    else if (dtype == OGQ_BF16) go((__bf16*)nullptr);
    else go((_Float16*)nullptr);
    if (parts > 1)
        launch_kernel(add_parts_kernel, dim3(ceil_div(s.out_part / 4, 64)), dim3(kBlock), st, reinterpret_cast<const f32x4*>(out), parts, (uint32_t)(s.out_part / 4),
                      (uint32_t)(s.out_stride / 4), s.cols, accumulate, dw, (uint64_t)dw_stride);
}

}  // namespace ogq
