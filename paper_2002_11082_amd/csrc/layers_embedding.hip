// libogq_layers: rows of a table by tokens, and the table's gradient.
//
// The gradient's rows are sums over equal tokens.  The tokens are sorted with their positions first, so that a sum has its rows one behind the other, in their order, whatever the
// order in which workgroups come: keys of 64 bits, the token above the position, no two of them alike.  Bound by memory: the table's gradient is written once, most of it zeros.
#include "layers_common.h"

namespace ogq {

namespace {

constexpr uint32_t kRun = 1024;   // keys that a workgroup sorts
constexpr uint32_t kWays = 32;    // sorted runs that a launch makes one of
constexpr uint32_t kGroup = 64;   // rows of a token, where it has at least two such groups, that are summed on their own; the last group has up to twice as many, less one
constexpr uint32_t kNone = 0xFFFFFFFFu;

// Token n, or kNone where it names no row.
__device__ __forceinline__ uint32_t token_of(const void* tokens, bool wide, uint64_t n, uint32_t vocab)
{
    const int64_t t = wide ? static_cast<const int64_t*>(tokens)[n] : (int64_t)static_cast<const int32_t*>(tokens)[n];
    return t >= 0 && t < (int64_t)vocab ? (uint32_t)t : kNone;
}

// 2^log2 threads to a row, which take its pieces in turn.  Bound by memory.
template <class T>
__global__ __launch_bounds__(kBlock) void embedding_kernel(const void* tokens, bool wide, uint32_t number, const T* table, uint64_t table_stride, uint32_t vocab, uint32_t cols,
                                                         uint32_t threads_log2, float scale, T* y, uint64_t y_stride)
{
    constexpr int N = kPiece<T>, kAhead = 2;
    const uint64_t row = ((uint64_t)block_number() << (8 - threads_log2)) + (threadIdx.x >> threads_log2);
    if (row >= number) return;
    const uint32_t threads = 1u << threads_log2, thread = threadIdx.x & (threads - 1), token = token_of(tokens, wide, row, vocab);
    const T* from = table + (uint64_t)(token == kNone ? 0 : token) * table_stride;
    T* to = y + row * y_stride;
    for (uint32_t first = thread * N; first < cols; first += kAhead * threads * N) {
        float v[kAhead][N] = {};
        if (token != kNone) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) load_piece<false>(from + first + k * threads * N, valid_of<T>(first + k * threads * N, cols), v[k]);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (token != kNone) {  // (a scale of any sign leaves the zeros of no token positive)
#pragma unroll
                for (int i = 0; i < N; ++i) v[k][i] *= scale;
            }
            store_piece<false>(to + first + k * threads * N, valid_of<T>(first + k * threads * N, cols), v[k]);
        }
    }
}

// How many of the `length` keys of a sorted run are less than `key`; `length` is below 2^log2.
__device__ __forceinline__ uint32_t count_below(const uint64_t* run, uint32_t length, uint32_t log2, uint64_t key)
{
    uint32_t below = 0;
    for (int bit = (int)log2 - 1; bit >= 0; --bit) {
        const uint32_t probe = below + (1u << bit);
        if (probe <= length && run[probe - 1] < key) below = probe;
    }
    return below;
}

// 1024 keys to a workgroup: every wavefront places its 64 by counting, then a key's place among all is its own place and what the other fifteen have below it.
__global__ __launch_bounds__(kRun) void sort_runs_kernel(const void* tokens, bool wide, uint32_t number, uint32_t vocab, uint64_t* keys)
{
    __shared__ uint64_t sorted[kRun];
    const uint32_t position = blockIdx.x * kRun + threadIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // (behind the last token: keys above all others)
    const uint32_t token = position < number ? token_of(tokens, wide, position, vocab) : kNone;
    uint64_t key = (uint64_t)token << 32 | position;
    uint32_t place = 0;
#pragma unroll 8
    for (int n = 0; n < 64; ++n) {
        const uint64_t other = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(token, n) << 32 | (uint32_t)__builtin_amdgcn_readlane(position, n);
        place += other < key ? 1 : 0;
    }
    sorted[wave * 64 + place] = key;
    __syncthreads();
    key = sorted[threadIdx.x];
    place = lane;
#pragma unroll
    for (uint32_t w = 0; w < kRun / 64; ++w)
        if (w != wave) place += count_below(sorted + w * 64, 64, 7, key);
    keys[blockIdx.x * kRun + place] = key;
}

// Runs of `run` sorted keys into runs of kWays times as many: a key's place is its own and what the other runs have below it.  `total` is a multiple of kRun.
__global__ __launch_bounds__(kBlock) void merge_runs_kernel(const uint64_t* from, uint64_t* to, uint32_t total, uint32_t run, uint32_t run_log2)
{
    const uint32_t at = blockIdx.x * kBlock + threadIdx.x;  // (all of a workgroup's are of one run)
    const uint32_t mine = (blockIdx.x * kBlock) >> run_log2, base = mine / kWays * kWays;
    const uint64_t key = from[at];
    uint32_t place = at - (mine << run_log2);
    // eight searches at a time, whose loads are under way together
    for (uint32_t r = base; r < base + kWays; r += 8) {
        if ((uint64_t)r << run_log2 >= total) break;
        uint32_t below[8] = {}, length[8];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) {
            const uint64_t begin = (uint64_t)(r + k) << run_log2;
            length[k] = r + k == mine || begin >= total ? 0 : (uint32_t)min((uint64_t)run, total - begin);
        }
        for (int bit = (int)run_log2; bit >= 0; --bit) {
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) {
                const uint32_t probe = below[k] + (1u << bit);
                const bool inside = probe <= length[k];
                // (a key that is there in any case)
                const uint64_t other = from[inside ? ((uint64_t)(r + k) << run_log2) + probe - 1 : at];
                if (inside && other < key) below[k] = probe;
            }
        }
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) place += below[k];
    }
    to[((uint64_t)base << run_log2) + place] = key;
}

// starts[v]: the first key of token v or one above it, for v = 0 ... vocab.
__global__ __launch_bounds__(kBlock) void starts_kernel(const uint64_t* keys, uint32_t number, uint32_t vocab, uint32_t* starts)
{
    const uint64_t v = (uint64_t)blockIdx.x * kBlock + threadIdx.x;
    if (v > vocab) return;
    starts[v] = count_below(keys, number, 32 - __builtin_clz(number), v << 32);
}

// The columns of a lane: a piece of a row, which lies as PieceAt says where the row has as many values.
template <class T>
struct Piece {
    PieceAt<T> at;
    int valid;
    bool whole;
    __device__ __forceinline__ Piece(uint32_t col, uint32_t cols) : at(col, max(cols, (uint32_t)kPiece<T>)), valid(valid_of<T>(col, cols)), whole(cols >= kPiece<T>) {}
    __device__ __forceinline__ bool there() const { return valid > 0; }
    __device__ __forceinline__ void add(const T* row, float (&sum)[kPiece<T>]) const
    {
        float v[kPiece<T>];
        values_of<T>(whole ? load_whole(row + at.col) : load_raw(row, valid), v);
#pragma unroll
        for (int i = 0; i < kPiece<T>; ++i) sum[i] += v[i];
    }
};

// The rows of keys first ... last, added one after the other.  All of the wavefront's lanes call it.
template <class T>
__device__ __forceinline__ void add_rows(const uint64_t* keys, uint32_t first, uint32_t last, const T* dy, uint64_t dy_stride, const Piece<T>& piece, float (&sum)[kPiece<T>])
{
    const uint32_t lane = threadIdx.x & 63;
    for (uint32_t at = first; at < last; at += 64) {
        const uint32_t here = min(64u, last - at), mine = (uint32_t)keys[at + min(lane, here - 1)];
        uint32_t n = 0;
        for (; n + 8 <= here; n += 8) {
            float v[8][kPiece<T>];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
#pragma unroll
                for (int i = 0; i < kPiece<T>; ++i) v[k][i] = 0.0f;
                piece.add(dy + (uint64_t)__builtin_amdgcn_readlane(mine, n + k) * dy_stride, v[k]);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int i = 0; i < kPiece<T>; ++i) sum[i] += v[k][i];
        }
        for (; n < here; ++n) piece.add(dy + (uint64_t)__builtin_amdgcn_readlane(mine, n) * dy_stride, sum);
    }
}

struct Table {
    uint32_t number, vocab, cols, blocks, pitch;  // blocks: of 64 pieces, along a row
    uint64_t dy_stride;
    float scale;
};

// The groups of tokens that have two or more of them.  A token's groups begin kGroup keys apart, so that of kGroup keys at most one begins a group, and a wavefront that looks at these
// keys sums it: sums[n] is the group that begins among keys n * kGroup ...
template <class T>
__global__ __launch_bounds__(kBlock) void add_groups_kernel(const uint64_t* keys, const uint32_t* starts, const T* dy, Table s, float* sums)
{
    const uint64_t unit = (uint64_t)block_number() * 4 + (threadIdx.x >> 6);
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t slot = unit / s.blocks;
    if (slot * kGroup >= s.number) return;
    const uint32_t at = (uint32_t)(slot * kGroup) + lane;
    bool begins = false;
    uint32_t last = 0;
    if (at < s.number) {
        const uint32_t token = (uint32_t)(keys[at] >> 32);
        if (token != kNone) {
            const uint32_t first = starts[token], end = starts[token + 1], group = (at - first) / kGroup, groups = (end - first) / kGroup;
            begins = groups >= 2 && (at - first) % kGroup == 0 && group < groups;
            last = group + 1 == groups ? end : at + kGroup;
        }
    }
    const uint64_t which = __builtin_amdgcn_ballot_w64(begins);
    if (which == 0) return;
    const int leader = __builtin_ctzll(which);
    const Piece<T> piece((uint32_t)(unit % s.blocks * 64 + lane) * kPiece<T>, s.cols);
    float sum[kPiece<T>] = {};
    add_rows(keys, __builtin_amdgcn_readlane(at, leader), __builtin_amdgcn_readlane(last, leader), dy, s.dy_stride, piece, sum);
    if (!piece.there()) return;
    float* out = sums + slot * s.pitch + (piece.whole ? piece.at.col : 0);
    memcpy(out, sum, sizeof sum);
}

// A row of the table's gradient, 64 pieces of it, to a wavefront: zeros, the sum of its rows, or the sum of its groups.
template <class T, bool ACCUMULATE>
__global__ __launch_bounds__(kBlock) void table_gradient_kernel(const uint64_t* keys, const uint32_t* starts, const T* dy, Table s, const float* sums, float* dtable,
                                                              uint64_t dtable_stride)
{
    constexpr int N = kPiece<T>;
    const uint64_t unit = (uint64_t)block_number() * 4 + (threadIdx.x >> 6), token = unit / s.blocks;
    if (token >= s.vocab) return;
    const uint32_t first = __builtin_amdgcn_readfirstlane(starts[token]), last = __builtin_amdgcn_readfirstlane(starts[token + 1]);
    if (ACCUMULATE && first == last) return;
    const Piece<T> piece((uint32_t)(unit % s.blocks * 64 + (threadIdx.x & 63)) * N, s.cols);
    float sum[N] = {};
    const uint32_t groups = (last - first) / kGroup;
    if (groups >= 2) {
        const float* from = sums + (uint64_t)(first / kGroup) * s.pitch + (piece.whole ? piece.at.col : 0);
#pragma unroll 4
        for (uint32_t n = 0; n < groups; ++n) {
            float v[N];
            memcpy(v, from + (uint64_t)n * s.pitch, sizeof v);
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] += v[i];
        }
    } else if (first != last) {
        add_rows(keys, first, last, dy, s.dy_stride, piece, sum);
    }
    if (!piece.there()) return;
    float* out = dtable + token * dtable_stride + (piece.whole ? piece.at.col : 0);
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] *= s.scale;
    if (piece.whole && piece.at.again == 0) {
        if (ACCUMULATE) {
            float old[N];
            memcpy(old, out, sizeof old);
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] += old[i];
        }
        memcpy(out, sum, sizeof sum);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (piece.whole ? piece.at.counts(i) : i < piece.valid) out[i] = ACCUMULATE ? out[i] + sum[i] : sum[i];
}

// The gradient of no tokens.
__global__ __launch_bounds__(kBlock) void zero_table_kernel(float* dtable, uint64_t stride, uint32_t rows, uint32_t cols)
{
    const uint64_t unit = (uint64_t)block_number(), blocks = (cols + kBlock * 4 - 1) / (kBlock * 4), row = unit / blocks;
    if (row >= rows) return;
    const uint32_t col = (uint32_t)(unit % blocks * kBlock + threadIdx.x) * 4;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
        if (col + i < cols) dtable[row * stride + col + i] = 0.0f;
}

// What lies where in the workspace.
struct Space {
    size_t keys, starts, sums, bytes;  // bytes of one of two buffers of keys, of starts, of the groups' sums, of all
};

size_t whole16(size_t n) { return (n + 15) / 16 * 16; }
size_t pitch_of(size_t cols) { return (cols + 7) / 8 * 8; }

Space space_of(size_t number, size_t vocab, size_t cols)
{
    Space s;
    s.keys = ceil_div(number, kRun) * kRun * sizeof(uint64_t);
    s.starts = whole16((vocab + 1) * sizeof(uint32_t));
    s.sums = number >= 2 * kGroup ? ceil_div(number, kGroup) * pitch_of(cols) * sizeof(float) : 0;
    s.bytes = 2 * s.keys + s.starts + s.sums;
    return s;
}

}  // namespace

void launch_embedding_forward(const Integers& tokens, size_t number, const Values& table, size_t vocab, size_t cols, uint32_t dtype, float scale, const Result& y,
                              hipStream_t st)
{
    with_type(dtype, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const uint64_t pieces = ceil_div(cols, kPiece<T>);
        uint32_t log2 = 0;
        while (log2 < 8 && ((uint64_t)2 << log2) <= pieces) ++log2;
        launch_kernel(embedding_kernel<T>, grid_of_blocks(ceil_div(number, kBlock >> log2)), dim3(kBlock), st, tokens.data, tokens.type == OGQ_INT64, (uint32_t)number,
                      static_cast<const T*>(table.data), table.stride, (uint32_t)vocab, (uint32_t)cols, log2, scale, static_cast<T*>(y.data), y.stride);
    });
}

size_t embedding_gradient_workspace(size_t number, size_t vocab, size_t cols) { return space_of(number, vocab, cols).bytes; }

void launch_embedding_gradient(const Integers& tokens, size_t number, const Values& dy, size_t vocab, size_t cols, uint32_t dtype, float scale, bool accumulate,
                               const Result& dtable, void* workspace, hipStream_t st)
{
    float* out = static_cast<float*>(dtable.data);
    if (number == 0) {
        launch_kernel(zero_table_kernel, grid_of_blocks(vocab * ceil_div(cols, kBlock * 4)), dim3(kBlock), st, out, dtable.stride, (uint32_t)vocab, (uint32_t)cols);
        return;
    }
    const Space space = space_of(number, vocab, cols);
    char* at = static_cast<char*>(workspace);
    uint64_t *keys = reinterpret_cast<uint64_t*>(at), *other = reinterpret_cast<uint64_t*>(at + space.keys);
    uint32_t* starts = reinterpret_cast<uint32_t*>(at + 2 * space.keys);
    float* sums = reinterpret_cast<float*>(at + 2 * space.keys + space.starts);
    const uint32_t runs = (uint32_t)ceil_div(number, kRun), total = runs * kRun;
    launch_kernel(sort_runs_kernel, dim3(runs), dim3(kRun), st, tokens.data, tokens.type == OGQ_INT64, (uint32_t)number, (uint32_t)vocab, keys);
    uint32_t log2 = 10;
    for (uint64_t run = kRun; run < total; run *= kWays, log2 += 5) {
        launch_kernel(merge_runs_kernel, dim3(total / kBlock), dim3(kBlock), st, static_cast<const uint64_t*>(keys), other, total, (uint32_t)run, log2);
        std::swap(keys, other);
    }
    launch_kernel(starts_kernel, dim3((uint32_t)ceil_div(vocab + 1, kBlock)), dim3(kBlock), st, static_cast<const uint64_t*>(keys), (uint32_t)number, (uint32_t)vocab, starts);
    with_type(dtype, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const uint32_t blocks = (uint32_t)ceil_div(cols, 64 * kPiece<T>);
        const Table s{(uint32_t)number, (uint32_t)vocab, (uint32_t)cols, blocks, (uint32_t)pitch_of(cols), dy.stride, scale};
        const auto from = static_cast<const T*>(dy.data);
        if (space.sums != 0)
            launch_kernel(add_groups_kernel<T>, grid_of_blocks(ceil_div(ceil_div(number, kGroup) * blocks, 4)), dim3(kBlock), st, static_cast<const uint64_t*>(keys),
                          static_cast<const uint32_t*>(starts), from, s, sums);
        launch_kernel(accumulate ? table_gradient_kernel<T, true> : table_gradient_kernel<T, false>, grid_of_blocks(ceil_div((uint64_t)vocab * blocks, 4)), dim3(kBlock), st,
                      static_cast<const uint64_t*>(keys), static_cast<const uint32_t*>(starts), from, s, static_cast<const float*>(sums), out, dtable.stride);
    });
}

}  // namespace ogq
