// libogq_layers: rows of a table by tokens, and the table's gradient.
//
// The gradient's rows are sums over equal tokens.  The tokens are sorted with their positions first, so that a sum has its rows one behind the other, in their order, whatever the
// order in which workgroups come: keys of 64 bits, the token above the position, no two of them alike.  A wavefront then adds the rows of a window of neighbouring keys, so that a frequent token
// is as much work as many rare ones.  Bound by memory: the table's gradient is written once, most of it zeros, behind which the sorting hides; rows that tokens name twice.  16384 tokens of
// 32768 x 4096 bf16: the rows 40 us, sorting and zeros 33 + 46 (537 MB, 6.8 TB/s), the windows' sums 70 to 80, those of several windows 13.
#include "layers_common.h"

namespace ogq {

namespace {

constexpr uint32_t kRun = 1024;   // keys that a workgroup sorts
constexpr uint32_t kWays = 32;    // sorted runs that a launch makes one of
constexpr uint32_t kLeast = 8, kMost = 32;  // neighbouring keys whose rows a wavefront adds, a window: a power of two
constexpr uint32_t kNone = 0xFFFFFFFFu;

// Token n, or kNone where it names no row.
__device__ __forceinline__ uint32_t token_of(const void* tokens, bool wide, uint64_t n, uint32_t vocab)
{
    const int64_t t = wide ? static_cast<const int64_t*>(tokens)[n] : (int64_t)static_cast<const int32_t*>(tokens)[n];
    return t >= 0 && t < (int64_t)vocab ? (uint32_t)t : kNone;
}

// 2^log2 threads to a row, which take its pieces in turn.  Bound by memory: 16384 rows of 4096 bf16 40 us, 134 MB written at 3.4 TB/s while 84 MB of rows are gathered.
template <class T>
__global__ __launch_bounds__(kBlock) void embedding_kernel(const void* tokens, bool wide, uint32_t number, const T* table, uint64_t table_stride, uint32_t vocab, uint32_t cols,
                                                         uint32_t threads_log2, float scale, T* y, uint64_t y_stride)
{
    constexpr int N = kPiece<T>, kAhead = 2;
    const uint64_t row = ((uint64_t)this_block() << (8 - threads_log2)) + (threadIdx.x >> threads_log2);
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

// Zeros for the table's gradient: rows of `length` values in units of kUnit, `units` of them to a row (one row where the table has no gaps), or `together` short rows to a unit (0: rows are not short).
// 4096 tokens in a table of 200000 x 16 with gaps, all launches: 26 us, a row to a unit 446; without gaps 25.
constexpr uint32_t kUnit = 16384;
struct Fill {
    float* to;
    uint64_t rows, length, stride, units, first, last;  // units first ... last of all rows' are this launch's
    uint32_t together;
};

// Four zeros at `at` of a row of which `left` values are left.
__device__ __forceinline__ void fill_piece(float* to, uint32_t at, uint64_t left)
{
    const f32x4 zero = {};
    if (at + 4 <= left) {
        memcpy(to + at, &zero, sizeof zero);
    } else {
        for (uint32_t i = at; i < at + 4; ++i)
            if (i < left) to[i] = 0.0f;
    }
}

__device__ __forceinline__ void fill_unit(const Fill& f, uint64_t unit)
{
    if (f.together != 0) {
        const uint32_t pieces = (uint32_t)(f.length + 3) / 4;
#pragma unroll
        for (uint32_t n = 0; n < kUnit / 4 / kRun; ++n) {
            const uint32_t at = n * kRun + threadIdx.x, in = at / pieces, begin = (at - in * pieces) * 4;
            const uint64_t row = unit * f.together + in;
            if (in < f.together && row < f.rows) fill_piece(f.to + row * f.stride, begin, f.length);
        }
        return;
    }
    const uint64_t row = f.units == 1 ? unit : unit / f.units, begin = (unit - row * f.units) * kUnit;
    float* to = f.to + row * f.stride + begin;
    const uint64_t left = f.length - begin;
#pragma unroll
    for (uint32_t n = 0; n < kUnit / 4 / kRun; ++n) fill_piece(to, (n * kRun + threadIdx.x) * 4, left);
}

// The first `runs` workgroups sort 1024 keys each: every wavefront places its 64 by counting, then neighbouring runs become one, four times over: a key's place is its own and what the other run
// has below it.  The other workgroups fill.
__global__ __launch_bounds__(kRun) void sort_runs_kernel(const void* tokens, bool wide, uint32_t number, uint32_t vocab, uint32_t runs, uint64_t* keys, Fill fill)
{
    __shared__ uint64_t sorted[2][kRun];
    if (this_block() >= runs) {
        const uint64_t unit = fill.first + (this_block() - runs);
        if (unit < fill.last) fill_unit(fill, unit);
        return;
    }
    const uint32_t position = this_block() * kRun + threadIdx.x, lane = threadIdx.x & 63;
    // (behind the last token: keys above all others)
    const uint32_t token = position < number ? token_of(tokens, wide, position, vocab) : kNone;
    uint32_t place = threadIdx.x - lane;
#pragma unroll 8
    for (uint32_t n = 0; n < 64; ++n) {  // (a lane's position is above those of the lanes before it)
        const uint32_t other = __builtin_amdgcn_readlane(token, n);
        place += other < token || (other == token && n < lane) ? 1 : 0;
    }
    uint32_t side = 0;
    sorted[0][place] = (uint64_t)token << 32 | position;
    uint64_t key;
    for (uint32_t length = 64;; length *= 2) {
        __syncthreads();
        key = sorted[side][threadIdx.x];
        if (length == kRun) break;
        const uint64_t* other = &sorted[side][(threadIdx.x ^ length) & ~(length - 1)];
        uint32_t below = 0;
        for (uint32_t bit = length; bit != 0; bit /= 2) {
            const uint32_t probe = below + bit;
            if (probe <= length && other[probe - 1] < key) below = probe;
        }
        side ^= 1;
        sorted[side][(threadIdx.x & ~(2 * length - 1)) + (threadIdx.x & (length - 1)) + below] = key;
    }
    keys[position] = key;
}

// Runs of `run` sorted keys into runs of kWays times as many: a key's place is its own and what the other runs have below it.  Eight lanes to a key, each of which searches four runs, side by
// side: first among 128 samples of each run, which are in LDS, then in memory: in runs of 1024 three loads that wait for one another, in place of ten.  `total` is a multiple of kRun.  The workgroups behind those that the keys need fill.
constexpr uint32_t kKeys = kRun / 8;  // of a workgroup
__global__ __launch_bounds__(kRun) void merge_runs_kernel(const uint64_t* from, uint64_t* to, uint32_t total, uint32_t run, uint32_t run_log2, Fill fill)
{
    constexpr uint32_t kSide = kWays / 8, kSamplesLog2 = 7, kSamples = 1u << kSamplesLog2;
    __shared__ uint64_t samples[kWays * kSamples];
    if (this_block() >= total / kKeys) {
        const uint64_t unit = fill.first + (this_block() - total / kKeys);
        if (unit < fill.last) fill_unit(fill, unit);
        return;
    }
    const uint32_t at = this_block() * kKeys + threadIdx.x / 8, mine = (this_block() * kKeys) >> run_log2, base = mine / kWays * kWays;  // (all of a workgroup's keys are of one run)
    const uint32_t apart_log2 = run_log2 - kSamplesLog2, first = threadIdx.x % 8 * kSide;
    const uint64_t start = (uint64_t)base << run_log2, key = from[at];
#pragma unroll
    for (uint32_t k = 0; k < kWays * kSamples / kRun; ++k) {  // sample n is the last of its keys: behind the last key of all, one above them
        const uint64_t n = k * kRun + threadIdx.x, which = start + ((n + 1) << apart_log2) - 1;
        samples[n] = which < total ? from[which] : ~0ull;
    }
    __syncthreads();
    uint32_t below[kSide] = {};
    // how many of a run's samples are below the key: as many times their distance keys are
#pragma unroll
    for (int bit = kSamplesLog2; bit >= 0; --bit)
#pragma unroll
        for (uint32_t k = 0; k < kSide; ++k) {
            const uint32_t probe = below[k] + (1u << bit);
            if (probe <= kSamples && samples[(first + k) * kSamples + min(probe, kSamples) - 1] < key) below[k] = probe;
        }
#pragma unroll
    for (uint32_t k = 0; k < kSide; ++k) below[k] <<= apart_log2;
    for (int bit = (int)apart_log2 - 1; bit >= 0; --bit)
#pragma unroll
        for (uint32_t k = 0; k < kSide; ++k) {
            const uint32_t probe = below[k] + (1u << bit);
            const uint64_t which = start + ((uint64_t)(first + k) << run_log2) + probe - 1;
            const bool inside = probe <= run && which < total;
            const uint64_t other = from[inside ? which : at];  // (a key that is there in any case)
            if (inside && other < key) below[k] = probe;
        }
    uint32_t place = 0;
#pragma unroll
    for (uint32_t k = 0; k < kSide; ++k) place += base + first + k != mine ? below[k] : 0;
    place += dpp_u32<kDppXor1>(place);
    place += dpp_u32<kDppXor2>(place);
    place += dpp_u32<kDppHalfMirror>(place);
    if (first == 0) to[start + (at - (mine << run_log2)) + place] = key;
}

// The columns of a lane: a piece of a row, which lies as PieceAt says where the row has as many values.
template <class T>
struct Piece {
    PieceAt<T> at;
    int valid;
    bool whole;
    __device__ __forceinline__ Piece(uint32_t col, uint32_t cols) : at(col, max(cols, (uint32_t)kPiece<T>)), valid(valid_of<T>(col, cols)), whole(cols >= kPiece<T>) {}
    __device__ __forceinline__ bool there() const { return valid > 0; }
    __device__ __forceinline__ uint4 load(const T* row) const { return whole ? load_whole(row + at.col) : load_raw(row, valid); }
    __device__ __forceinline__ uint32_t col() const { return whole ? at.col : 0; }
    // A row of the table's gradient, of which a lane has these values.  Added to what is there, the ones that the last piece has twice count once.
    template <bool ACCUMULATE>
    __device__ __forceinline__ void store(float* row, float scale, const float (&sum)[kPiece<T>]) const
    {
        constexpr int N = kPiece<T>;
        if (!there()) return;
        float v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = sum[i] * scale;
        float* out = row + col();
        if (whole && (!ACCUMULATE || at.again == 0)) {
            if constexpr (ACCUMULATE) {
                float old[N];
                memcpy(old, out, sizeof old);
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] += old[i];
            }
            memcpy(out, v, sizeof v);
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (whole ? at.counts(i) : i < valid) out[i] = ACCUMULATE ? out[i] + v[i] : v[i];
    }
};

struct Table {
    uint32_t number, cols, blocks, pitch, window;  // blocks: of 64 pieces, along a row; window: keys of one (or rows of the table)
    uint64_t dy_stride, dtable_stride;
    float scale;
};

// The token of a key, kNone for what is not there.
__device__ __forceinline__ uint32_t token_at(const uint64_t* keys, uint32_t number, uint64_t at) { return at < number ? (uint32_t)(keys[at] >> 32) : kNone; }

// A window of neighbouring keys to a wavefront: the rows of each token among them are added one after the other.  A token whose keys all lie here is finished; of the others (the first one may have begun
// before, the last one may go on) the sums wait for the next kernel, sums[2 n] of one that had begun before window n, sums[2 n + 1] of one that begins there.
template <class T, bool ACCUMULATE>
__global__ __launch_bounds__(kBlock) void add_windows_kernel(const uint64_t* keys, const T* dy, Table s, float* sums, float* dtable)
{
    constexpr int N = kPiece<T>, kAhead = 8;
    const uint64_t unit = (uint64_t)this_block() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), window = unit / s.blocks;
    if (window * s.window >= s.number) return;
    const uint32_t lane = threadIdx.x & 63, first = (uint32_t)window * s.window;
    const uint64_t key = lane < s.window && first + lane < s.number ? keys[first + lane] : ~0ull;
    const uint32_t token = (uint32_t)(key >> 32), position = (uint32_t)key;
    const uint32_t before = window == 0 ? kNone : token_at(keys, s.number, first - 1), behind = token_at(keys, s.number, (uint64_t)first + s.window);
    const uint32_t here = __builtin_popcountll(__builtin_amdgcn_ballot_w64(token != kNone));  // (keys of no token are the last ones)
    if (here == 0) return;
    const uint32_t left = __shfl_up(token, 1);
    const uint64_t begins = __builtin_amdgcn_ballot_w64(lane == 0 || token != left);
    const Piece<T> piece((uint32_t)(unit % s.blocks * 64 + lane) * N, s.cols);
    uint4 next[kAhead];
    const auto fetch = [&](uint32_t n) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) next[k] = piece.load(dy + (uint64_t)__builtin_amdgcn_readlane(position, min(n + k, here - 1)) * s.dy_stride);
    };
    float sum[N];
    fetch(0);
    for (uint32_t n = 0; n < here; n += kAhead) {
        uint4 now[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) now[k] = next[k];
        fetch(n + kAhead);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const uint32_t at = n + k;
            if (at >= here) break;
            const bool begin = begins >> at & 1, end = at + 1 == here || (begins >> (at + 1) & 1);
            float v[N];
            values_of<T>(now[k], v);
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] = begin ? v[i] : sum[i] + v[i];
            if (!end) continue;
            const uint32_t mine = __builtin_amdgcn_readlane(token, at);
            // (whether its first key here is the window's first, and of a token that the key before names)
            const bool begun = mine == before && mine == (uint32_t)__builtin_amdgcn_readfirstlane(token), goes_on = at + 1 == s.window && mine == behind;
            if (!begun && !goes_on) {
                piece.template store<ACCUMULATE>(dtable + (uint64_t)mine * s.dtable_stride, s.scale, sum);
            } else if (piece.there()) {
                memcpy(sums + (2 * window + (begun ? 0 : 1)) * s.pitch + piece.col(), sum, sizeof sum);
            }
        }
    }
}

// The tokens whose keys lie in several windows: the workgroup of the window in which a token's last key lies adds the sums of its windows, a quarter of them in each wavefront, one after the
// other.
template <class T, bool ACCUMULATE>
__global__ __launch_bounds__(kBlock) void join_windows_kernel(const uint64_t* keys, Table s, const float* sums, float* dtable)
{
    constexpr int N = kPiece<T>;
    const uint64_t window = this_block() / s.blocks + 1, first = window * s.window;
    if (first >= s.number) return;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t token = token_at(keys, s.number, first);
    if (token == kNone || token != token_at(keys, s.number, first - 1) || token == token_at(keys, s.number, first + s.window)) return;
    // the windows before this one into which the token had gone on: the nearest that the key before does not name is where it begins
    uint64_t begin = window;
    for (;;) {
        const uint64_t at = begin - 1 - lane;  // (one below 0 is none)
        const bool on = begin >= 1 + (uint64_t)lane && at != 0 && token_at(keys, s.number, at * s.window - 1) == token;
        const uint64_t all = __builtin_amdgcn_ballot_w64(on);
        if (~all == 0) {
            begin -= 64;
            continue;
        }
        begin -= 1 + __builtin_ctzll(~all);
        break;
    }
    const Piece<T> piece((this_block() % s.blocks * 64 + lane) * N, s.cols);
    const uint64_t number = window - begin + 1, each = (number + 3) / 4, last = min(number, (wave + 1) * each);
    float sum[N] = {};
    if (piece.there()) {
#pragma unroll 8
        for (uint64_t n = wave * each; n < last; ++n) {
            float v[N];
            memcpy(v, sums + (2 * (begin + n) + (n == 0 ? 1 : 0)) * s.pitch + piece.col(), sizeof v);
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] += v[i];
        }
    }
    __shared__ float shared[3][N][64];
    if (wave != 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) shared[wave - 1][i][lane] = sum[i];
    }
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] += shared[w][i][lane];
    piece.template store<ACCUMULATE>(dtable + (uint64_t)token * s.dtable_stride, s.scale, sum);
}

// Up to kFew tokens in one launch: a workgroup has s.window rows of the table's gradient, 64 pieces of each; all of its wavefronts look at all of the tokens, four to a lane, and each adds the rows of
// its own 64 of them, in their order, 8 under way together.  Rows that only one wavefront's tokens name are stored by it, those of several are added in LDS, in the wavefronts' order; others are zeros.  Bound by latency: 256 tokens in
// a table of 1000 x 512 bf16 4.3 us (sorted 15.9); 256 x 4096 of one token 16 us.
constexpr uint32_t kFew = 256;
template <class T, bool ACCUMULATE>
__global__ __launch_bounds__(kBlock) void few_tokens_gradient_kernel(const void* tokens, bool wide, uint32_t vocab, const T* dy, Table s, float* dtable)
{
    constexpr int N = kPiece<T>, kAhead = 8, kWaves = kFew / 64;
    __shared__ float shared[2][kWaves][N][64];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint64_t first = (uint64_t)(this_block() / s.blocks) * s.window;
    if (first >= vocab) return;
    const uint32_t rows = (uint32_t)min((uint64_t)s.window, vocab - first);
    const Piece<T> piece((this_block() % s.blocks * 64 + lane) * N, s.cols);
    uint32_t row[kWaves];  // of this workgroup's that a token names, kNone for others
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
        const uint32_t at = k * 64 + lane, token = at < s.number ? token_of(tokens, wide, at, vocab) : kNone;
        row[k] = token != kNone && token >= first && token - (uint32_t)first < rows ? token - (uint32_t)first : kNone;
    }
    float* out = dtable + first * s.dtable_stride;
    uint32_t side = 0;
    for (uint32_t r = 0; r < rows; ++r, out += s.dtable_stride) {
        uint32_t having = 0;  // the wavefronts whose tokens name this row
        uint64_t which = 0;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            const uint64_t all = __builtin_amdgcn_ballot_w64(row[k] == r);
            having |= all != 0 ? 1u << k : 0u;
            which = k == wave ? all : which;
        }
        float sum[N] = {};
        if (having == 0) {
            if (!ACCUMULATE && r % kWaves == wave) piece.template store<false>(out, 0.0f, sum);
            continue;
        }
        while (which != 0) {
            const uint32_t count = __builtin_popcountll(which);
            uint4 v[kAhead];
#pragma unroll
            for (uint32_t n = 0; n < kAhead; ++n) {  // (behind the last one it is loaded again, and not used)
                v[n] = piece.load(dy + (uint64_t)(wave * 64 + __builtin_ctzll(which)) * s.dy_stride);
                if (n + 1 < count) which &= which - 1;
            }
            if (count <= kAhead) which = 0;
#pragma unroll
            for (uint32_t n = 0; n < kAhead; ++n) {
                float a[N];
                values_of<T>(v[n], a);
                if (n < count) {
#pragma unroll
                    for (int i = 0; i < N; ++i) sum[i] += a[i];
                }
            }
        }
        if ((having & (having - 1)) == 0) {
            if (having >> wave & 1) piece.template store<ACCUMULATE>(out, s.scale, sum);
            continue;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) shared[side][wave][i][lane] = sum[i];
        __syncthreads();
        if (wave == r % kWaves) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                sum[i] = shared[side][0][i][lane];
#pragma unroll
                for (int k = 1; k < kWaves; ++k) sum[i] += shared[side][k][i][lane];
            }
            piece.template store<ACCUMULATE>(out, s.scale, sum);
        }
        side ^= 1;  // (a side is written again behind the next barrier, which its reader reaches when it has read)
    }
}

// The gradient of no tokens.
__global__ __launch_bounds__(kRun) void fill_kernel(Fill fill)
{
    if (this_block() < fill.last) fill_unit(fill, this_block());
}

// What lies where in the workspace.
struct Space {
    size_t keys, sums, bytes;  // bytes of one of two buffers of keys, of the windows' sums, of all
    uint32_t window;
};

size_t pitch_of(size_t cols) { return (cols + 7) / 8 * 8; }

Space space_of(size_t number, size_t cols)
{
    Space s{};
    if (number <= kFew) return s;
    s.keys = ceil_div(number, kRun) * kRun * sizeof(uint64_t);
    // Keys of a window: few where there are few wavefronts, since a wavefront has eight rows under way at a time; many otherwise, since each window may leave two sums that are written and read
    // once more.  bf16, all launches, windows of 8, 16, 32, 64 keys: 300 tokens x 512 16.4, 19.2, 24.6, 36.4 us; 4096 x 1024 34.5, 38.4, 46.9, 64.9; 32768 x 1024 67.4, 59.7, 58.8, 68.7;
    // 16384 x 4096 192.5, 185.8, 180.8, 193.0.
    s.window = kLeast;
    while (s.window < kMost && number * cols / s.window > (size_t)2048 * 512) s.window *= 2;
    s.sums = number > s.window ? 2 * ceil_div(number, s.window) * pitch_of(cols) * sizeof(float) : 0;
    s.bytes = (number > kRun ? 2 : 1) * s.keys + s.sums;
    return s;
}

Fill fill_of(const Result& dtable, size_t vocab, size_t cols)
{
    const bool gaps = dtable.stride != cols && vocab > 1;
    Fill f{static_cast<float*>(dtable.data), gaps ? vocab : 1, gaps ? cols : vocab * cols, dtable.stride, 0, 0, 0, 0};
    f.units = ceil_div(f.length, kUnit);
    f.last = f.units * f.rows;
    if (gaps && cols <= kUnit / 2) {
        f.together = (uint32_t)(kUnit / 4 / ceil_div(cols, 4));
        f.last = ceil_div(vocab, f.together);
    }
    return f;
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
        launch_kernel(embedding_kernel<T>, grid_of(ceil_div(number, kBlock >> log2)), dim3(kBlock), st, tokens.data, tokens.type == OGQ_INT64, (uint32_t)number,
                      static_cast<const T*>(table.data), table.stride, (uint32_t)vocab, (uint32_t)cols, log2, scale, static_cast<T*>(y.data), y.stride);
    });
}

size_t embedding_gradient_workspace(size_t number, size_t, size_t cols) { return space_of(number, cols).bytes; }

void launch_embedding_gradient(const Integers& tokens, size_t number, const Values& dy, size_t vocab, size_t cols, uint32_t dtype, float scale, bool accumulate,
                               const Result& dtable, void* workspace, hipStream_t st)
{
    float* out = static_cast<float*>(dtable.data);
    const Fill fill = fill_of(dtable, vocab, cols);
    if (number == 0) {
        launch_kernel(fill_kernel, grid_of(fill.last), dim3(kRun), st, fill);
        return;
    }
    if (number <= kFew) {
        with_type(dtype, [&](auto* t) {
            using T = std::remove_pointer_t<decltype(t)>;
            const uint32_t blocks = (uint32_t)ceil_div(cols, 64 * kPiece<T>);
            // Rows of a workgroup: many only where there are many, since a wavefront takes the rows of its tokens one behind the other.  256 tokens, bf16, 1, 4, 16, 32 rows: 1000 x 512 4.3, 5.3, 9.5,
            // 13.2 us (sorted 15.9); 32768 x 1024 69.0, 32.0, 26.3, 32.6 (25.6).
            const uint64_t all = (uint64_t)vocab * blocks;
            const uint32_t rows = all >= 16384 ? 16 : all >= 4096 ? 4 : 1;
            const Table s{(uint32_t)number, (uint32_t)cols, blocks, 0, rows, dy.stride, dtable.stride, scale};
            launch_kernel(accumulate ? few_tokens_gradient_kernel<T, true> : few_tokens_gradient_kernel<T, false>, grid_of(ceil_div(vocab, rows) * blocks), dim3(kBlock),
                          st, tokens.data, tokens.type == OGQ_INT64, (uint32_t)vocab, static_cast<const T*>(dy.data), s, out);
        });
        return;
    }
    const Space space = space_of(number, cols);
    uint64_t *keys = static_cast<uint64_t*>(workspace), *other = keys + space.keys / sizeof(uint64_t);
    const uint32_t runs = (uint32_t)ceil_div(number, kRun), total = runs * kRun;
    float* sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + space.bytes - space.sums);
    // the launches that sort fill the table as well, each an equal part
    uint32_t launches = 1;
    for (uint64_t run = kRun; run < total; run *= kWays) ++launches;
    const auto part = [&](uint32_t n) {
        Fill f = fill;
        f.first = fill.last * n / launches, f.last = fill.last * (n + 1) / launches;
        if (accumulate) f.last = f.first;
        return f;
    };
    Fill now = part(0);
    launch_kernel(sort_runs_kernel, grid_of(runs + now.last - now.first), dim3(kRun), st, tokens.data, tokens.type == OGQ_INT64, (uint32_t)number, (uint32_t)vocab, runs, keys,
                  now);
    uint32_t log2 = 10, n = 1;
    for (uint64_t run = kRun; run < total; run *= kWays, log2 += 5) {
        now = part(n++);
        launch_kernel(merge_runs_kernel, grid_of(total / kKeys + now.last - now.first), dim3(kRun), st, static_cast<const uint64_t*>(keys), other, total, (uint32_t)run, log2,
                      now);
        std::swap(keys, other);
    }
    with_type(dtype, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const uint32_t blocks = (uint32_t)ceil_div(cols, 64 * kPiece<T>);
        const Table s{(uint32_t)number, (uint32_t)cols, blocks, (uint32_t)pitch_of(cols), space.window, dy.stride, dtable.stride, scale};
        const uint64_t windows = ceil_div(number, space.window);
        launch_kernel(accumulate ? add_windows_kernel<T, true> : add_windows_kernel<T, false>, grid_of(ceil_div(windows * blocks, 4)), dim3(kBlock), st, static_cast<const uint64_t*>(keys),
                      static_cast<const T*>(dy.data), s, sums, out);
        if (windows > 1)
            launch_kernel(accumulate ? join_windows_kernel<T, true> : join_windows_kernel<T, false>, grid_of((windows - 1) * blocks), dim3(kBlock), st, static_cast<const uint64_t*>(keys), s,
                          static_cast<const float*>(sums), out);
    });
}

}  // namespace ogq
