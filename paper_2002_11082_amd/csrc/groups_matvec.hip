// libogq_groups: tokens times the transpose of weights held in 4 bits,
//   y[t][o] = sum over i of x[t][i] * w^[o][i].
//
// group_matvec_kernel (a few tokens) on the vector unit, group_matmul_kernel (more) on the matrix cores.  Both read 32 weights (16 bytes) per lane and
// turn eight of them into bf16 with four conversions, which take the group's power along.
#include <cmath>

#include "groups_common.h"

namespace ogq {

namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kLaneCols = 32;  // weights of a lane's load: within one group

struct MatvecShape {
    uint32_t tokens, outs, cols, groups, group_log2, row_blocks, token_blocks;
    uint32_t steps;  // of a wavefront: chunks of columns, or of a part of the sum
    uint32_t team;   // wavefronts that share the columns of a row
    uint64_t x_stride, y_stride, y_part;
};

__device__ __forceinline__ uint32_t word_of(const uint4& w, int j) { return j == 0 ? w.x : j == 1 ? w.y : j == 2 ? w.z : w.w; }

// Pair n (0 .. 15) of a lane's 32 weights; the conversion's byte is a constant of the instruction.
#define OGQ_PAIR(cvt, w, n, unit) \
    ((n) % 4 == 0 ? cvt(word_of(w, (n) / 4), unit, 0) : (n) % 4 == 1 ? cvt(word_of(w, (n) / 4), unit, 1) : (n) % 4 == 2 ? cvt(word_of(w, (n) / 4), unit, 2) : cvt(word_of(w, (n) / 4), unit, 3))

// Two values summed over the two halves of the wavefront (of each pair of rows of 16 lanes): the lower one keeps the first's sum.
__device__ __forceinline__ float halves_sum(float a, float b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float rows_sum(float a, float b)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// One step of a sum of N values over the wavefront: while there are several, lanes and their partners at distance D share them, half each.
template <int D, int N>
__device__ __forceinline__ void sum_step(float* v, uint32_t lane, uint32_t& index)
{
    if constexpr (N > 1) {
        constexpr int H = N / 2;
#pragma unroll
        for (int i = 0; i < H; ++i) {
            if constexpr (D == 32) {
                v[i] = halves_sum(v[i], v[i + H]);
            } else if constexpr (D == 16) {
                v[i] = rows_sum(v[i], v[i + H]);
            } else {
                const bool upper = (lane & D) != 0;
                const float keep = upper ? v[i + H] : v[i], send = upper ? v[i] : v[i + H];
                v[i] = keep + __uint_as_float(lane_xor<D>(__float_as_uint(send), lane));
            }
        }
        index += (lane & D) ? H : 0;
    } else {
        v[0] += __uint_as_float(lane_xor<D>(__float_as_uint(v[0]), lane));
    }
}

// Sums N values (a power of two) over the wavefront.  A lane ends with the sums `index`, ... (as many as N / 64, at least one).
template <int N>
__device__ __forceinline__ uint32_t sum_over_lanes(float* v, uint32_t lane)
{
    uint32_t index = 0;
    sum_step<32, N>(v, lane, index);
    sum_step<16, (N > 2 ? N / 2 : 1)>(v, lane, index);
    sum_step<8, (N > 4 ? N / 4 : 1)>(v, lane, index);
    sum_step<4, (N > 8 ? N / 8 : 1)>(v, lane, index);
    sum_step<2, (N > 16 ? N / 16 : 1)>(v, lane, index);
    sum_step<1, (N > 32 ? N / 32 : 1)>(v, lane, index);
    return index;
}

// A lane's 32 values of a token, as they are in memory; `whole`: all lanes have 32, a branch of the scalar unit.
template <class T>
constexpr int kLaneWords = kLaneCols * sizeof(T) / 4;

template <class T, int N>
__device__ __forceinline__ void load_values(const T* from, int valid, bool whole, uint32_t (&to)[N * sizeof(T) / 4])
{
    if (whole || valid >= N) memcpy(to, from, sizeof to);
    else load_some<T, N>(from, valid, to);
}

// The same of 64 lanes' values: in the order of memory, 1 KB at once, and through LDS to the lane that wants them (a lane's own 32 values lie 64 or
// 128 bytes from its neighbour's, four times as many trips to the cache).  Sixteen bytes p of lane l lie at p ^ (l / 2 or l).
template <class T>
__device__ __forceinline__ void load_turned(const T* from, int valid, bool whole, uint32_t lane, uint4* turn, uint32_t (&to)[kLaneWords<T>])
{
    constexpr uint32_t kQuads = kLaneWords<T> / 4, kShift = kQuads == 4 ? 1 : 0;
    constexpr int kQuad = 16 / sizeof(T);
    uint32_t q[kQuads][4];
#pragma unroll
    for (uint32_t i = 0; i < kQuads; ++i) {
        const int at = (int)(i * 64 + lane) * kQuad;
        load_values<T, kQuad>(from + at, valid - at, whole, q[i]);
    }
#pragma unroll
    for (uint32_t i = 0; i < kQuads; ++i) {
        const uint32_t n = i * 64 + lane, of = n / kQuads;
        turn[of * kQuads + ((n ^ (of >> kShift)) & (kQuads - 1))] = make_uint4(q[i][0], q[i][1], q[i][2], q[i][3]);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (uint32_t p = 0; p < kQuads; ++p) {
        const uint4 w = turn[lane * kQuads + ((p ^ (lane >> kShift)) & (kQuads - 1))];
        memcpy(&to[4 * p], &w, 16);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The products of 32 weights with every token's values, added to the tokens' sums.
template <class T, int NT>
__device__ __forceinline__ void add_products(const uint32_t (&x)[NT][kLaneWords<T>], const uint4& w, float unit, float* sum)
{
    if constexpr (__is_same(T, __bf16)) {
#pragma unroll
        for (int n = 0; n < 16; ++n) {
            const bf16x2 q = OGQ_PAIR(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4, w, n, unit);
#pragma unroll
            for (int t = 0; t < NT; ++t) sum[t] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x[t][n]), q, sum[t], false);
        }
    } else if constexpr (__is_same(T, _Float16)) {
        // (a weight times its group's power may be outside of fp16: the power comes in behind the sum)
        float part[NT] = {};
#pragma unroll
        for (int n = 0; n < 16; ++n) {
            const f16x2 q = OGQ_PAIR(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4, w, n, 1.0f);
#pragma unroll
            for (int t = 0; t < NT; ++t) part[t] = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, x[t][n]), q, part[t], false);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) sum[t] = __builtin_fmaf(part[t], unit, sum[t]);
    } else {
#pragma unroll
        for (int n = 0; n < 16; ++n) {
            const f32x2 q = OGQ_PAIR(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4, w, n, unit);
#pragma unroll
            for (int t = 0; t < NT; ++t)
                sum[t] = __builtin_fmaf(q[1], __uint_as_float(x[t][2 * n + 1]), __builtin_fmaf(q[0], __uint_as_float(x[t][2 * n]), sum[t]));
        }
    }
}

constexpr int kFew = 4;  // rows of weights of a wavefront, and most wavefronts of a workgroup

// A few tokens: a lane keeps 32 of the values of each and multiplies them with the same columns of four rows of weights, whose loads are all under way at
// once, 1 KB of a row in a piece.  The wavefronts of a team share the columns of its rows; a workgroup has up to four wavefronts, in one team or several.
// Bound by memory behind 3 us of latency: one token in bf16 against 4096 x 25088 weights 11.0 us, 5.0 TB/s.  (Eight rows 14.1, sixteen 16.2, two 18.1 where four
// took 13.8; eight wavefronts 16.7; with the next piece's loads ahead of the products 14.3.)
// Values straight from memory or through LDS: one token in bf16 11.0 and 11.3 us, two 23.5 and 15.3, four against 4096 x 4096 8.8 and 5.6; one in fp32 15.6 and 15.0.
template <class T, int NT>
__global__ __launch_bounds__(64 * kFew) void group_matvec_kernel(const uint8_t* codes, const uint8_t* exponents, const T* x, MatvecShape s, T* y)
{
    constexpr bool kTurned = sizeof(T) == 4 || NT > 1;
    __shared__ float parts[kFew][kFew * NT];
    __shared__ uint4 turn[kTurned ? kFew : 1][kTurned ? 64 * kLaneWords<T> / 4 : 1];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), teams = blockDim.x / (64 * s.team);
    const uint32_t first_out = block_number() * teams * kFew, o0 = first_out + wave / s.team * kFew;
    if (first_out >= s.outs) return;
    const uint32_t pitch = s.groups << s.group_log2;
    float sum[kFew * NT] = {};
    for (uint32_t chunk = wave % s.team; chunk < s.steps; chunk += s.team) {
        const uint32_t first = chunk * (64 * kLaneCols), col = first + lane * kLaneCols;
        const bool whole = first + 64 * kLaneCols <= s.cols;
        uint4 w[kFew];
        uint32_t byte[kFew], v[NT][kLaneWords<T>];
#pragma unroll
        for (int r = 0; r < kFew; ++r) w[r] = make_uint4(0, 0, 0, 0), byte[r] = 127;
        if (col < pitch) {
#pragma unroll
            for (int r = 0; r < kFew; ++r) {
                const uint64_t row = min(o0 + r, s.outs - 1);  // (what is not there repeats the last)
                w[r] = *reinterpret_cast<const uint4*>(codes + row * (pitch / 2) + col / 2);
                byte[r] = exponents[row * s.groups + (col >> s.group_log2)];
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const T* of = x + min((uint32_t)t, s.tokens - 1) * s.x_stride;
            if constexpr (kTurned) {
                // (fp32: a check per piece costs registers, two tokens against 4096 x 25088 30.8 us for 24.5)
                if (sizeof(T) == 2) load_turned(of + first, (int)(s.cols - first), whole, lane, turn[wave], v[t]);
                else if (whole) load_turned(of + first, 0, true, lane, turn[wave], v[t]);
                else load_values<T, kLaneCols>(of + col, (int)(s.cols - col), false, v[t]);
            } else {
                load_values<T, kLaneCols>(of + col, (int)(s.cols - col), whole, v[t]);
            }
        }
#pragma unroll
        for (int r = 0; r < kFew; ++r) add_products<T, NT>(v, w[r], power(byte[r]), sum + r * NT);
    }
    const uint32_t index = sum_over_lanes<kFew * NT>(sum, lane);
    parts[wave][index] = sum[0];  // (several lanes write the same)
    __syncthreads();
    if (threadIdx.x < teams * kFew * NT) {
        const uint32_t r = threadIdx.x / NT, t = threadIdx.x % NT, o = first_out + r, first = r / kFew * s.team, at = threadIdx.x % (kFew * NT);
        if (o >= s.outs || t >= s.tokens) return;
        float all = parts[first][at];
        for (uint32_t k = 1; k < s.team; ++k) all += parts[first + k][at];
        y[t * s.y_stride + o] = (T)all;
    }
}

// ----------------------------------------------------------------------------------------------------------------------
// More tokens
// ----------------------------------------------------------------------------------------------------------------------
template <class T>
constexpr int kPiecesOf = __is_same(T, __bf16) ? 1 : __is_same(T, _Float16) ? 2 : 3;

// Eight values of a token as they are in memory, in pieces of bf16 whose sum they are.
template <class T>
__device__ __forceinline__ void pieces_of(const uint32_t* raw, bf16x8 (&out)[kPiecesOf<T>])
{
    if constexpr (__is_same(T, __bf16)) {
        memcpy(&out[0], raw, 16);
    } else {
        T v[8];
        memcpy(v, raw, sizeof v);
        uint32_t w[3][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t a[3], b[3];
            split3((float)v[2 * i], a[0], a[1], a[2]);
            split3((float)v[2 * i + 1], b[0], b[1], b[2]);
#pragma unroll
            for (int p = 0; p < 3; ++p) w[p][i] = __builtin_amdgcn_perm(b[p], a[p], 0x07060302u);
        }
#pragma unroll
        for (int p = 0; p < kPiecesOf<T>; ++p) memcpy(&out[p], w[p], 16);
    }
}

// Eight weights of a lane's 32.
__device__ __forceinline__ bf16x8 weights_of(const uint4& w, int q, float unit)
{
    const uint32_t word = word_of(w, q);
    const bf16x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, unit, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, unit, 1),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, unit, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, unit, 3)};
    bf16x8 a;
    memcpy(&a, p, 16);
    return a;
}

// Four neighbouring results of a token.
template <class OUT>
__device__ __forceinline__ void store_outs(OUT* row, uint32_t o, uint32_t outs, f32x4 v)
{
    OUT r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = (OUT)v[i];
    if (o + 4 <= outs) {
        memcpy(row + o, r, sizeof r);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (o + i < outs) row[o + i] = r[i];
}

constexpr int kStep = 4 * kLaneCols;  // columns of a wavefront's step

// Columns of a workgroup's stage, and how many stages it has in LDS: what leaves room for several workgroups on a CU.
constexpr uint32_t stage_cols(uint32_t value_bytes, uint32_t token_tiles) { return value_bytes == 4 || token_tiles == 4 ? 128 : 256; }
template <class T>
constexpr int stage_buffers(int token_tiles) { return stage_cols(sizeof(T), token_tiles) * 16 * token_tiles * kPiecesOf<T> * 2 <= 20480 ? 2 : 1; }


// Many weights: the wavefronts of a workgroup hold 32 rows each and share the tokens' values, which come to LDS a stage of columns at a time, in pieces and in the order
// of the matrix instruction's operands, while the weights and the values of the next stage are on their way.  Lane l has the columns l / 16 * STAGE / 4 ... of a stage.
// 16 tokens in bf16 against 4096 x 25088 weights 15.0 us and 3.9 for the parts (memory: 3.6 TB/s of weights); 64 tokens 33.7 and 5.2, in fp32 against 4096 x 16384 36.1 and 4.9, where a stage's
// latency and the values' way through LDS bound it: the matrix cores are busy for a third of the time.  64 rows to a wavefront, which halve the reads of LDS: 38.0 for 35.3.
template <class T, class OUT, int NT>
__global__ __launch_bounds__(256) void group_matmul_kernel(const uint8_t* codes, const uint8_t* exponents, const T* x, MatvecShape s, OUT* y)
{
    constexpr int kPieces = kPiecesOf<T>, kRb = 2, kStageCols = stage_cols(sizeof(T), NT), kLoads = kStageCols / kStep, kBuffers = stage_buffers<T>(NT);
    constexpr int kOctets = kStageCols / 8, kMine = 16 * NT * kOctets / 256, kFragments = 4 * kLoads * NT * kPieces;
    __shared__ uint4 operands[kBuffers][kFragments][64];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t block = blockIdx.x;
    const uint32_t o0 = block % s.row_blocks * (64 * kRb) + wave * (16 * kRb);
    block /= s.row_blocks;
    const uint32_t t0 = block % s.token_blocks * (16 * NT), part = block / s.token_blocks;
    const uint32_t pitch = s.groups << s.group_log2;
    const uint32_t first = part * s.steps * kStageCols, end = min(first + s.steps * kStageCols, pitch);
    const uint32_t mine = (lane >> 4) * (kStageCols / 4);
    const uint8_t* w_row[kRb];
    const uint8_t* e_row[kRb];
#pragma unroll
    for (int r = 0; r < kRb; ++r) {
        const uint64_t row = min(o0 + 16 * r + (lane & 15), s.outs - 1);  // (what is not there repeats the last)
        w_row[r] = codes + row * (pitch / 2);
        e_row[r] = exponents + row * s.groups;
    }
    uint4 w[kRb][kLoads], next_w[kRb][kLoads];
    uint32_t bytes[kRb], next_bytes[kRb];
    const auto fetch_weights = [&](uint32_t at, uint4 (&to)[kRb][kLoads], uint32_t (&to_bytes)[kRb]) __attribute__((always_inline)) {
        const uint32_t col = at + mine;
#pragma unroll
        for (int r = 0; r < kRb; ++r) {
            to_bytes[r] = 0x7F7F;
#pragma unroll
            for (int j = 0; j < kLoads; ++j) to[r][j] = make_uint4(0, 0, 0, 0);
        }
        if (col + kLoads * kLaneCols <= pitch) {
#pragma unroll
            for (int r = 0; r < kRb; ++r) {
#pragma unroll
                for (int j = 0; j < kLoads; ++j) to[r][j] = *reinterpret_cast<const uint4*>(w_row[r] + col / 2 + 16 * j);
                const uint8_t* e = e_row[r] + (col >> s.group_log2);
                if (kLoads == 2 && s.group_log2 == 5) {
                    uint16_t both;
                    memcpy(&both, e, 2);
                    to_bytes[r] = both;
                } else {
                    to_bytes[r] = *e * 0x0101u;
                }
            }
        } else if (col < pitch) {  // (the first 32 columns alone)
#pragma unroll
            for (int r = 0; r < kRb; ++r) {
                to[r][0] = *reinterpret_cast<const uint4*>(w_row[r] + col / 2);
                to_bytes[r] = e_row[r][col >> s.group_log2] | 0x7F00u;
            }
        }
    };
    // eight values of a token to a thread and pass
    uint32_t v[kMine][kLaneWords<T> / 4];
    const auto fetch_values = [&](uint32_t at) __attribute__((always_inline)) {
        const bool whole = at + kStageCols <= s.cols;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const uint32_t n = i * 256 + threadIdx.x, token = min(t0 + n / kOctets, s.tokens - 1), col = at + n % kOctets * 8;
            load_values<T, 8>(x + token * s.x_stride + col, (int)(s.cols - col), whole, v[i]);
        }
    };
    // (a fragment's 64 pieces of 16 bytes lie at lane ^ its number: neighbouring octets, which go to the same lane of eight fragments, in different banks)
    const auto bring_values = [&](uint32_t buffer) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const uint32_t n = i * 256 + threadIdx.x, token = n / kOctets, octet = n % kOctets;
            const uint32_t of = octet / (kOctets / 4) * 16 + token % 16, fragment = octet % (kOctets / 4);
            bf16x8 b[kPieces];
            pieces_of<T>(v[i], b);
#pragma unroll
            for (int p = 0; p < kPieces; ++p)
                operands[buffer][(fragment * NT + token / 16) * kPieces + p][of ^ (fragment & 7)] = __builtin_bit_cast(uint4, b[p]);
        }
    };
    f32x4 sum[kRb][NT] = {};
    if (first < end) {
        fetch_weights(first, w, bytes);
        fetch_values(first);
    }
    uint32_t buffer = 0;
    for (uint32_t at = first; at < end; at += kStageCols, buffer ^= kBuffers - 1) {
        if (kBuffers == 1) __syncthreads();
        bring_values(buffer);
        if (at + kStageCols < end) {
            fetch_weights(at + kStageCols, next_w, next_bytes);
            fetch_values(at + kStageCols);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                bf16x8 a[kRb];
#pragma unroll
                for (int r = 0; r < kRb; ++r) a[r] = weights_of(w[r][j], q, power(bytes[r] >> (8 * j) & 0xFFu));
                const int fragment = 4 * j + q;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int p = kPieces - 1; p >= 0; --p) {
                        const bf16x8 b = __builtin_bit_cast(bf16x8, operands[buffer][(fragment * NT + n) * kPieces + p][lane ^ (fragment & 7)]);
#pragma unroll
                        for (int r = 0; r < kRb; ++r) sum[r][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[r], b, sum[r][n], 0, 0, 0);
                    }
            }
#pragma unroll
        for (int r = 0; r < kRb; ++r) {
            bytes[r] = next_bytes[r];
#pragma unroll
            for (int j = 0; j < kLoads; ++j) w[r][j] = next_w[r][j];
        }
    }
    y += part * s.y_part;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint32_t t = t0 + 16 * n + (lane & 15);
        if (t >= s.tokens) continue;
#pragma unroll
        for (int r = 0; r < kRb; ++r) store_outs(y + t * s.y_stride, o0 + 16 * r + (lane >> 4) * 4, s.outs, sum[r][n]);
    }
}

// The parts of the sums, added in an order that their number alone decides: four sums to a thread, and four threads to them, which add every fourth part.
template <class T>
__global__ __launch_bounds__(kBlock) void add_token_parts_kernel(const float* parts, uint32_t number, uint32_t tokens, uint32_t outs, T* y, uint64_t y_stride)
{
    __shared__ f32x4 shared[3][64];
    const uint32_t lane = threadIdx.x & 63, fourth = threadIdx.x >> 6, row_quads = (outs + 3) / 4, quad = blockIdx.x * 64 + lane;
    const uint32_t t = quad / row_quads, o = quad % row_quads * 4;
    f32x4 v = {};
    if (t < tokens) {
        const float* from = parts + (uint64_t)t * row_quads * 4 + o;
        const uint64_t part = (uint64_t)tokens * row_quads * 4;
#pragma unroll 4
        for (uint32_t n = fourth; n < number; n += 4) v += *reinterpret_cast<const f32x4*>(from + n * part);
    }
    if (fourth != 0) shared[fourth - 1][lane] = v;
    __syncthreads();
    if (fourth != 0 || t >= tokens) return;
#pragma unroll
    for (int n = 0; n < 3; ++n) v += shared[n][lane];
    store_outs(y + t * y_stride, o, outs, v);
}

uint32_t ceil_div(uint64_t a, uint64_t b) { return (uint32_t)((a + b - 1) / b); }


// Which calls group_matvec_kernel takes: one launch for two, while what it reads of the tokens, once for four rows of weights, does not yet cost more.  Its us and the two launches'
// together.  Two tokens in bf16: 4096 x 25088 15.3 and 18.4, 4096 x 4096 4.4 and 7.4, 16384 x 1024 5.8 and 8.0, 2048 x 1024 4.0 and 7.3, 16384 x 500 6.4 and 5.2.  Four: 4096 x 4096 5.6
// and 7.6, 8192 x 1024 5.5 and 7.5, 8192 x 2816 9.7 and 9.0, 16384 x 1024 8.6 and 8.0, 4096 x 25088 26.4 and 18.4.  Two in fp32: 4096 x 16384 16.1 and 19.5, 4096 x 4096 6.0 and 9.1,
// 8192 x 1024 7.2 and 7.4, 4096 x 25088 24.5 and 23.6, 16384 x 1024 11.2 and 9.0; four: 4096 x 4096 8.6 and 9.4, 8192 x 1024 13.0 and 7.4.
bool few_tokens(size_t tokens, size_t outs, size_t cols, uint32_t dtype)
{
    if (tokens <= 1) return true;
    if (dtype == OGQ_FP32) return tokens == 2 && outs <= 8192 && cols <= 16384;
    if (tokens == 2) return outs <= 8192 || cols >= 1024;
    return tokens <= 4 && outs <= 8192 && outs * cols <= (1u << 24);
}

// How group_matmul_kernel is launched.
struct Plan {
    uint32_t token_tiles, row_blocks, token_blocks, parts, steps;
};

Plan plan_of(size_t tokens, size_t outs, size_t cols, uint32_t dtype)
{
    Plan p;
    p.token_tiles = tokens <= 16 ? 1 : tokens <= 32 ? 2 : 4;
    p.row_blocks = ceil_div(outs, 128);
    p.token_blocks = ceil_div(tokens, 16 * p.token_tiles);
    const uint64_t blocks = (uint64_t)p.row_blocks * p.token_blocks;
    const uint32_t steps = ceil_div(cols, stage_cols(dtype == OGQ_FP32 ? 4 : 2, p.token_tiles));
    // Parts of the sums, where they save more than the second launch (3 us).  `alone`: us of a workgroup that has all steps, 1.2, 1.8 or 2.2 each, which more parts share out;
    // `sums`: us for a part's sums on their way out and back.  Their sum is least at sqrt(alone / sums) parts.  Beyond one workgroup to a CU (`full`) only some two fifths of a
    // step's time is still shared out, and whole rounds of 256 workgroups count.  us of both launches, by parts: 64 tokens in bf16, 1000 x 4096: 1 51, 4 19.6, 8 11.9, 16 10.9,
    // 32 12.3; 2048 x 2048: 4 14.4, 8 10.6, 16 11.6; 4096 x 25088: 12 50.3, 16 42.5, 24 38.4, 32 38.0; in fp32, 4096 x 4096: 4 29.4, 8 22.0, 16 22.5, 32 28.2; 4096 x 16384: 8 54.9,
    // 16 42.2, 32 44.2; 16 tokens in bf16, 4096 x 25088: 8 25.5, 16 19.2, 32 19.2; 16384 x 1024: 1 8.2, 2 8.6; 32 tokens: 1 13.0, 2 11.9; 512 tokens, 4096 x 4096: 1 73.5, 4 45.6.
    const double alone = steps * (p.token_tiles == 1 ? 1.2 : p.token_tiles == 2 ? 1.8 : 2.2), sums = 1e-6 * (double)tokens * (double)outs;
    const double full = 256.0 / blocks;
    double parts = sqrt(alone / sums);
    if (parts > full) parts = full * fmax(1.0, floor(0.63 * parts / full + 0.25));
    p.parts = alone > 6.0 ? (uint32_t)fmax(1.0, fmin(parts, fmin(1024.0 / blocks, steps))) : 1;
    p.steps = ceil_div(steps, p.parts);
    return p;
}

uint64_t pitch_of(size_t outs) { return (outs + 3) / 4 * 4; }

template <class T, class OUT>
void launch_matmul(const Plan& p, const uint8_t* codes, const uint8_t* exponents, const T* x, const MatvecShape& s, OUT* y, hipStream_t st)
{
    const auto kernel = p.token_tiles == 1 ? group_matmul_kernel<T, OUT, 1> : p.token_tiles == 2 ? group_matmul_kernel<T, OUT, 2> : group_matmul_kernel<T, OUT, 4>;
    launch_kernel(kernel, dim3(p.row_blocks * p.token_blocks * p.parts), dim3(256), st, codes, exponents, x, s, y);
}

template <class T>
void launch_few(dim3 grid, dim3 block, const uint8_t* codes, const uint8_t* exponents, const T* x, const MatvecShape& s, T* y, hipStream_t st)
{
    auto kernel = s.tokens == 1 ? group_matvec_kernel<T, 1> : group_matvec_kernel<T, 2>;
    if constexpr (sizeof(T) == 2)
        if (s.tokens > 2) kernel = group_matvec_kernel<T, 4>;
    launch_kernel(kernel, grid, block, st, codes, exponents, x, s, y);
}

template <class T>
void launch_of(const Groups& w, MatvecShape s, const T* x, uint32_t dtype, T* y, void* workspace, hipStream_t st)
{
    const auto codes = static_cast<const uint8_t*>(w.codes);
    if (few_tokens(s.tokens, s.outs, s.cols, dtype)) {
        s.steps = ceil_div((uint64_t)s.groups << s.group_log2, 64 * kLaneCols);
        const uint32_t rounds = ceil_div(s.steps, kFew);
        s.team = rounds ? ceil_div(s.steps, rounds) : 1;
        // Several teams to a workgroup where 512 workgroups are left: one token in fp32, 1 and 4 teams: 16384 x 1024 8.0 and 5.7 us, 8192 x 1024 5.2 and 4.2, 2048 x 1024 3.2 and 3.8.
        const uint32_t teams = min(kFew / s.team, max(1u, ceil_div(s.outs, kFew) / 512));
        launch_few(grid_of_blocks(ceil_div(s.outs, kFew * teams)), dim3(64 * s.team * teams), codes, w.exponents, x, s, y, st);
        return;
    }
    const Plan p = plan_of(s.tokens, s.outs, s.cols, dtype);
    s.row_blocks = p.row_blocks, s.token_blocks = p.token_blocks, s.steps = p.steps, s.y_part = 0;
    if (p.parts == 1) {
        launch_matmul<T, T>(p, codes, w.exponents, x, s, y, st);
        return;
    }
    const uint64_t y_stride = s.y_stride;
    float* parts = static_cast<float*>(workspace);
    s.y_stride = pitch_of(s.outs);
    s.y_part = s.tokens * s.y_stride;
    launch_matmul<T, float>(p, codes, w.exponents, x, s, parts, st);
    launch_kernel(add_token_parts_kernel<T>, dim3(ceil_div(s.y_part / 4, 64)), dim3(kBlock), st, parts, p.parts, s.tokens, s.outs, y, y_stride);
}

}  // namespace

size_t group_matvec_workspace(size_t tokens, size_t outs, size_t cols, uint32_t dtype)
{
    if (few_tokens(tokens, outs, cols, dtype)) return 0;
    const Plan p = plan_of(tokens, outs, cols, dtype);
    return p.parts > 1 ? p.parts * tokens * pitch_of(outs) * sizeof(float) : 0;
}

void launch_group_matvec(const Groups& w, size_t outs, size_t cols, const ogq_group_params_t* p, const Values& x, size_t tokens, uint32_t dtype,
                         const Result& y, void* workspace, hipStream_t st)
{
    MatvecShape s = {};
    s.tokens = (uint32_t)tokens, s.outs = (uint32_t)outs, s.cols = (uint32_t)cols;
    s.groups = ceil_div(cols, p->group_size);
    s.group_log2 = p->group_size == 32 ? 5 : p->group_size == 64 ? 6 : 7;
    s.x_stride = x.stride, s.y_stride = y.stride;
    if (dtype == OGQ_FP32) launch_of(w, s, static_cast<const float*>(x.data), dtype, static_cast<float*>(y.data), workspace, st);
    else if (dtype == OGQ_BF16) launch_of(w, s, static_cast<const __bf16*>(x.data), dtype, static_cast<__bf16*>(y.data), workspace, st);
    else launch_of(w, s, static_cast<const _Float16*>(x.data), dtype, static_cast<_Float16*>(y.data), workspace, st);
}

}  // namespace ogq
