// Embedding: rows of a weight looked up by token and scaled, and the weight's
// gradient, the sum over the rows of each token.
//
//   y[i] = scale weight[t_i],   dweight[v] = scale sum over i with t_i = v of dy[i]
//
// Both are bound by memory (8,192 rows of 4096 in bfloat16 17 us, 7.8 TB/s with
// the commonest words' rows in the caches).  The gradient is formed without
// atomics on values, so that it is the same on every run, and in one of two
// forms: few rows in one launch, where every row looks for its like; more
// sorted by (token, row), the sorted order cut into equal units, of which a wave
// each adds up the runs of equal tokens, and runs that cross units joined from
// their units' shares.  Cut by units and not by tokens, the work is even however
// often a token occurs (in text the commonest word is a twentieth of all).  All
// of dweight is written, and the zeros beside what else there is to do: they are
// most of the time.

#include <cmath>
#include <new>

#include "gd.h"
#include "gd_host.hpp"
#include "gd_rows.hpp"

namespace gd {

constexpr uint32_t kEmbedMaxDim = 1u << 20, kEmbedMaxRows = 1u << 24;
constexpr uint32_t kNoToken = 0xFFFFFFFFu;  // padding: sorted behind every token
constexpr uint32_t kPadding = 0x7FFFFFFFu;  // what stands for it where tokens are compared: above them all, below 2^32 - 1
constexpr uint32_t kSortChunk = 4096, kSortThreads = 1024;
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

// Sorted rows a unit holds: as many, up to 32, as leave three waves a compute unit, each with a slice of 64 vectors of a
// unit's columns.  Few short rows make many small units for the sake of parallel work (14,003 rows of 237 in float16 with
// units of 16 and 32: 40 and 46 us), many or long ones larger, of which fewer partial sums are written (16,384 of 1024 in
// bfloat16: 54 and 51; with 64 8,192 of 4096 take 120 us in place of 118, and 200,000 of 256 301 in place of 310).
constexpr uint64_t kUnitWaves = 768;
constexpr uint32_t slice_count(uint32_t dim, int type) {
    const uint32_t columns = kWave * 16 / (type == GD_F32 ? 4 : 2);
    return (dim + columns - 1) / columns;
}
constexpr uint32_t unit_rows(uint64_t rows, uint32_t slices) {
    uint32_t unit = 32;
    while (unit > 8 && (rows + unit - 1) / unit * slices < kUnitWaves) unit /= 2;
    return unit;
}
// No number of rows up to this one makes more units: where units are below 32, twice their rows made fewer than kUnitWaves waves.
constexpr uint64_t most_units(uint64_t rows, uint32_t slices) {
    return std::max<uint64_t>(std::min<uint64_t>((rows + 7) / 8, 2 * kUnitWaves / slices), (rows + 31) / 32);
}

// The token of row i: kNoToken for ids outside the vocabulary.
__device__ __forceinline__ uint32_t token_at(const void* tokens, bool wide, uint64_t i, uint32_t vocab) {
    const int64_t t = wide ? ((const int64_t*)tokens)[i] : (int64_t)((const int32_t*)tokens)[i];
    return t >= 0 && t < (int64_t)vocab ? (uint32_t)t : kNoToken;
}

// The tokens of rows i, i + step and so on, past the last row that one again.  All loads before the first use.
template <int N>
__device__ __forceinline__ void tokens_at(const void* tokens, bool wide, uint64_t i, uint64_t step, uint64_t rows, uint32_t vocab,
                                          uint32_t (&out)[N]) {
    int64_t t[N];
    if (wide) {
#pragma unroll
        for (int k = 0; k < N; ++k) t[k] = ((const int64_t*)tokens)[min(i + k * step, rows - 1)];
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) t[k] = ((const int32_t*)tokens)[min(i + k * step, rows - 1)];
    }
#pragma unroll
    for (int k = 0; k < N; ++k) out[k] = t[k] >= 0 && t[k] < (int64_t)vocab ? (uint32_t)t[k] : kNoToken;
}

// y[i] = scale weight[t_i]: LANES lanes a row, VECS 16-byte vectors a lane at a time.
template <typename T, int LANES, int VECS>
__global__ __launch_bounds__(kBlock) void k_embed(gd_embed_io io, uint32_t vocab, uint32_t dim, bool wide) {
    constexpr int E = 16 / sizeof(T), kRows = kBlock / LANES;
    const uint32_t lane = threadIdx.x % LANES;
    for (uint64_t row = (uint64_t)blockIdx.x * kRows + threadIdx.x / LANES; row < io.rows; row += (uint64_t)gridDim.x * kRows) {
        const uint32_t t = token_at(io.tokens, wide, row, vocab);
        const T* from = (const T*)io.weight + (t == kNoToken ? 0 : (uint64_t)t * io.weight_stride);
        T* to = (T*)io.y + row * io.y_stride;
        for (uint32_t e = lane * E; e < dim; e += LANES * E * VECS) {
            Pack<T, E> v[VECS];
#pragma unroll
            for (int i = 0; i < VECS; ++i) {
                const uint32_t at = min(e + i * LANES * E, dim);
                v[i] = load_some<E>(from + at, t == kNoToken ? 0 : (int)(dim - at));
            }
#pragma unroll
            for (int i = 0; i < VECS; ++i) {
                const uint32_t at = min(e + i * LANES * E, dim);
                if (t != kNoToken)
#pragma unroll
                    for (int j = 0; j < E; ++j) v[i].v[j] = (T)((float)v[i].v[j] * io.scale);
                store_stream<E>(to + at, v[i], (int)(dim - at));
            }
        }
    }
}

// out = or += scale s, columns from c on, n of which exist.
template <int N>
__device__ __forceinline__ void put_gradient(float* out, const float (&s)[N], float scale, int n, bool accumulate) {
    Pack<float, N> v;
    if (accumulate) v = load_some<N>(out, n);
#pragma unroll
    for (int j = 0; j < N; ++j) v.v[j] = accumulate ? v.v[j] + scale * s[j] : scale * s[j];
    store_some<N>(out, v, n);
}

// The columns of a row from c on that a lane takes, a 16-byte vector of dy.  Where the row ends inside it, the vector is
// the one that ends with the row, and what it shares with the lane before is left out.  So every load is made, by every
// lane: loads behind conditions wait for one another (14,003 rows of 237 in float16 took
// 26 us so, now 18).
template <typename T, bool SHORT>  // SHORT: dim is below a vector, and read element by element
struct Columns {
    static constexpr int E = 16 / sizeof(T);
    uint32_t at, dim, skip;  // skip: elements of the vector that are not the lane's
    __device__ __forceinline__ Columns(uint32_t c, uint32_t dim) : dim(dim) {
        at = SHORT ? 0 : min(c, dim - E);
        skip = min(c - at, (uint32_t)E);
    }
    __device__ __forceinline__ u4 load(const T* row) const {
        Pack<T, E> r;
        if constexpr (SHORT) {
#pragma unroll
            for (int j = 0; j < E; ++j) r.v[j] = row[min((uint32_t)j, dim - 1)];
        } else {
            r = load_pack<E>(row + at);
        }
        u4 w;  // as words: elements would be taken apart behind the load, and waited for
        __builtin_memcpy(&w, &r, sizeof w);
        return w;
    }
    static __device__ __forceinline__ void add(float (&sum)[E], const u4& w) {
        Pack<T, E> r;
        __builtin_memcpy(&r, &w, sizeof w);
#pragma unroll
        for (int j = 0; j < E; ++j) sum[j] += (float)r.v[j];
    }
    __device__ __forceinline__ void put(float* row, const float (&s)[E], float scale, bool accumulate) const {
        if (!SHORT && skip == 0) {
            put_gradient<E>(row + at, s, scale, E, accumulate);
            return;
        }
#pragma unroll
        for (int j = 0; j < E; ++j)
            if ((uint32_t)j >= skip && (!SHORT || (uint32_t)j < dim)) {
                float* const to = row + at + j;
                *to = accumulate ? *to + scale * s[j] : scale * s[j];
            }
    }
};

// ---- Few rows: all of it in one launch ----
//
// A block takes a row and looks through all tokens for its own: the first row
// of a token finds all rows of it, in order, and writes their sum, the others
// end.  Of a token with many rows the first few rows' blocks take a share of the
// columns each, so that the commonest word is no block's work alone (4,096 rows
// of 512 in bfloat16, one word: 25 us, by one block 66).  Blocks between those
// write zeros, over rows of dweight that no token names.  Looking costs rows^2
// reads of tokens, from the caches, and stays beside the zeros up to kFewRows:
// 3,000 rows of 500 in binary32 for 85,000 words take 31 us, sorted (below) 38;
// 4,000 of 1024 in bfloat16 for 1,000 words 15 and 22, 4,096 of 8192 26 and 41.
// Longer rows, whose slices a block would take in turn, are sorted (64 rows of
// 65,536: 49 us, sorted 15).
constexpr uint32_t kFewSlices = 16;
constexpr uint32_t kFewRows = 4096, kFewThreads = 512, kFewWaves = kFewThreads / kWave, kFewAtOnce = 8;
constexpr uint32_t kFewTogether = 32;  // rows of a token that a wave adds up alone: 1,000 rows of 1024 8.4 us, with 16 12.2
constexpr uint32_t kRunLanes = 16, kRunAtOnce = 4, kRunShare = 16;  // where a token has more: lanes a row, rows at a time and a block
constexpr uint32_t kFillFloats = 16384;  // of zeros that a block writes, about
constexpr uint32_t kFewBlocks = 1u << 22;

template <typename T, bool SHORT>
__global__ __launch_bounds__(kFewThreads) void k_embed_few(gd_embed_grad io, uint32_t vocab, uint32_t dim, bool wide,
                                                           uint32_t fills, uint32_t per_fill) {
    typedef Columns<T, SHORT> Cols;
    constexpr int E = Cols::E;
    constexpr uint32_t kSlice = kWave * E, kRunSlice = kRunLanes * E, kRunGroups = kFewThreads / kRunLanes;
    __shared__ uint64_t mask[kFewRows / kWave];
    __shared__ union {
        uint16_t list[kFewRows];                    // of a token's rows
        uint32_t named[(kFillFloats + 31) / 32];    // a bit for each row that a block of zeros looks after
    } lds;
    __shared__ float shares[kRunGroups][kRunSlice];
    const uint32_t rows = (uint32_t)io.rows, wave = wave_index(), lane = lane_id();
    // rows' blocks are spread evenly among those of zeros: the ones wait, the others write
    const uint64_t all = (uint64_t)rows + fills, at = blockIdx.x;
    const uint32_t i = (uint32_t)(at * rows / all);
    if ((at + 1) * rows / all == i) {
        auto& named = lds.named;
        const uint32_t first = (uint32_t)(at - i) * per_fill, n = min(per_fill, vocab - first);
        for (uint32_t w = threadIdx.x; w < (n + 31) / 32; w += kFewThreads) named[w] = 0;
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < rows; j += kFewThreads) {
            const uint32_t t = token_at(io.tokens, wide, j, vocab) - first;
            if (t < n) atomicOr(&named[t / 32], 1u << t % 32);
        }
        __syncthreads();
        const uint32_t per_row = (dim + 3) / 4;
        const uint64_t vectors = (uint64_t)n * per_row;
        for (uint64_t v = threadIdx.x; v < vectors; v += kFewThreads) {
            const uint32_t row = n == 1 ? 0 : (uint32_t)v / per_row;
            const uint32_t e = (uint32_t)(v - (uint64_t)row * per_row) * 4;
            if (!(named[row / 32] >> row % 32 & 1))
                store_stream<4>(io.dweight + (uint64_t)(first + row) * io.dweight_stride + e, Pack<float, 4>{}, (int)(dim - e));
        }
        return;
    }
    const uint32_t token = token_at(io.tokens, wide, i, vocab);
    if (token == kNoToken) return;
    auto& list = lds.list;
    uint32_t others[kFewRows / kFewThreads];
    tokens_at(io.tokens, wide, threadIdx.x, kFewThreads, rows, vocab, others);
#pragma unroll
    for (uint32_t k = 0; k < kFewRows / kFewThreads; ++k) {
        const uint64_t m = ballot(others[k] == token && k * kFewThreads + threadIdx.x < rows);
        if (lane == 0) mask[k * kFewWaves + wave] = m;
    }
    __syncthreads();
    uint64_t mine = mask[lane];
    static_assert(kFewRows == kWave * kWave);
    const uint64_t before = lane < i / kWave ? mine : lane == i / kWave ? mine & ((1ull << i % kWave) - 1) : 0;
    // the token's first row's block writes the sum, of many rows its first rows' blocks a share of the columns each: the
    // more the more rows, and no block more than four (4,096 rows of 8192: 26 us, by rows alone 51)
    const uint32_t scan = wave_incl_scan((uint32_t)popc64(before) << 16 | (uint32_t)popc64(mine)), ends = lane_value(scan, kWave - 1);
    const uint32_t place = ends >> 16, incl = scan & 0xFFFF, count = ends & 0xFFFF;
    const uint32_t shares_of_row = (dim + kRunSlice - 1) / kRunSlice;
    const uint32_t blocks = count <= kFewTogether ? 1 : min(max(count / kRunShare, (shares_of_row + 3) / 4), min(count, shares_of_row));
    if (place >= blocks) return;
    if (wave == 0)
        for (uint32_t to = incl - popc64(mine); mine; mine &= mine - 1, ++to)
            list[to] = (uint16_t)(lane * kWave + (uint32_t)__ffsll((unsigned long long)mine) - 1);
    __syncthreads();
    float* out = io.dweight + (uint64_t)token * io.dweight_stride;
    // adds rows first to first + N of the list
    const auto add = [&](auto at_once, uint32_t first, const Cols& cols, float (&sum)[E]) {
        constexpr uint32_t N = at_once();
        u4 d[N];
#pragma unroll
        for (uint32_t k = 0; k < N; ++k) d[k] = cols.load((const T*)io.dy + (uint64_t)list[min(first + k, count - 1)] * io.dy_stride);
#pragma unroll
        for (uint32_t k = 0; k < N; ++k)
            if (first + k < count) Cols::add(sum, d[k]);
    };
    if (count <= kFewTogether) {  // a wave takes a slice of the columns
        for (uint32_t s = wave * kSlice; s < dim; s += kFewWaves * kSlice) {
            const Cols cols(s + lane * E, dim);
            float sum[E] = {};
            for (uint32_t first = 0; first < count; first += kFewAtOnce)
                add(std::integral_constant<uint32_t, kFewAtOnce>(), first, cols, sum);
            cols.put(out, sum, io.scale, io.accumulate != 0);
        }
        return;
    }
    const uint32_t group = threadIdx.x / kRunLanes, l = threadIdx.x % kRunLanes;
    for (uint32_t s = place * kRunSlice; s < dim; s += blocks * kRunSlice) {  // groups of lanes share the rows
        const Cols cols(s + l * E, dim);
        double total[E];
#pragma unroll
        for (int j = 0; j < E; ++j) total[j] = 0.0;
        for (uint32_t first = group * kRunAtOnce; first < count; first += kRunGroups * kRunAtOnce) {
            float sum[E] = {};
            add(std::integral_constant<uint32_t, kRunAtOnce>(), first, cols, sum);
#pragma unroll
            for (int j = 0; j < E; ++j) total[j] += sum[j];
        }
#pragma unroll
        for (int j = 0; j < E; ++j) shares[group][j * kRunLanes + l] = (float)total[j];
        __syncthreads();
        if (threadIdx.x < kRunSlice) {
            double v = 0.0;
#pragma unroll
            for (uint32_t g = 0; g < kRunGroups; ++g) v += shares[g][threadIdx.x];
            const uint32_t j = threadIdx.x / kRunLanes;  // of the lane's vector
            const float sum[1] = {(float)v};
            if (j >= cols.skip && (!SHORT || j < dim)) put_gradient<1>(out + cols.at + j, sum, io.scale, 1, io.accumulate != 0);
        }
        __syncthreads();
    }
}

// ---- More rows ----

// Zeros over [rows][dim] at `stride`, shared by `blocks` blocks, a 16-byte vector a thread and turn.  There are
// as many blocks as such turns, up to kFillBlocks: 85,000 x 500 take 26 us so, 34 with 512 blocks that go round.
constexpr uint32_t kFillBlocks = 1u << 20;
__device__ __forceinline__ void fill_zeros(float* out, uint32_t rows, uint32_t dim, uint64_t stride, uint32_t block, uint32_t blocks) {
    const Pack<float, 4> zeros = {};
    const uint32_t per_row = (dim + 3) / 4, threads = blockDim.x;
    const bool one_run = stride == dim;
    const uint64_t all = one_run ? (uint64_t)rows * dim : (uint64_t)rows * per_row;
    for (uint64_t v = (uint64_t)block * threads + threadIdx.x; one_run ? v * 4 < all : v < all; v += (uint64_t)blocks * threads) {
        if (one_run) {
            store_stream<4>(out + v * 4, zeros, (int)min(all - v * 4, (uint64_t)4));
        } else {
            const uint64_t row = v / per_row;
            const uint32_t e = (uint32_t)(v - row * per_row) * 4;
            store_stream<4>(out + row * stride + e, zeros, (int)(dim - e));
        }
    }
}
uint32_t fill_blocks(uint32_t rows, uint32_t dim, uint32_t threads) {
    return (uint32_t)std::min<uint64_t>(((uint64_t)rows * ((dim + 3ull) / 4) + threads - 1) / threads, kFillBlocks);
}

// Sorts chunks of 4,096 rows by (token, row): an element's place is the number
// of those before it, counted.  A block takes 64 elements, one a lane, and its
// sixteen waves a share each of the chunk's tokens, four at a time from LDS.
// (Sorted by exchanges, 2,048 in a block, 3,000 rows took 22 us.)  Blocks from
// `sorts` on write zeros over the first `filled` rows.
constexpr uint32_t kSortWaves = kSortThreads / kWave, kChunkBlocks = kSortChunk / kWave;
__global__ __launch_bounds__(kSortThreads) void k_embed_sort(gd_embed_grad io, uint32_t vocab, uint32_t dim, bool wide,
                                                             uint32_t sorts, uint64_t* out, uint32_t filled) {
    if (blockIdx.x >= sorts) {
        fill_zeros(io.dweight, filled, dim, io.dweight_stride, blockIdx.x - sorts, gridDim.x - sorts);
        return;
    }
    __shared__ __align__(16) uint32_t lds[kSortChunk];
    __shared__ uint32_t counts[kSortWaves][kWave];
    const uint64_t first = (uint64_t)(blockIdx.x / kChunkBlocks) * kSortChunk;
    const uint32_t n = (uint32_t)min(io.rows - first, (uint64_t)kSortChunk), padded = (n + kWave - 1) / kWave * kWave;
    uint32_t tokens[kSortChunk / kSortThreads];
    tokens_at(io.tokens, wide, first + threadIdx.x, kSortThreads, io.rows, vocab, tokens);
#pragma unroll
    for (uint32_t k = 0; k < kSortChunk / kSortThreads; ++k) {
        const uint32_t i = k * kSortThreads + threadIdx.x;
        lds[i] = i < n ? min(tokens[k], kPadding) : 0xFFFFFFFFu;
    }
    __syncthreads();
    const uint32_t i0 = blockIdx.x % kChunkBlocks * kWave, i = i0 + lane_id();
    if (i0 >= n) return;
    const uint32_t mine = lds[i], share = (padded / kWave + kSortWaves - 1) / kSortWaves * kWave;
    uint32_t j = min(wave_index() * share, padded);
    const uint32_t end = min(j + share, padded);
    uint32_t before = 0;
    const auto count = [&](uint32_t stop, uint32_t bound) {  // tokens below the bound
#pragma unroll 4
        for (; j < stop; j += 4) {
            const u4 t = *(const u4*)(lds + j);
#pragma unroll
            for (int k = 0; k < 4; ++k) before += t[k] < bound;
        }
    };
    count(min(end, i0), mine + 1);  // equal ones of lower rows are before it
    for (const uint32_t stop = min(end, i0 + kWave); j < stop; ++j) before += lds[j] < mine + (j < i);
    count(end, mine);
    counts[wave_index()][lane_id()] = before;
    __syncthreads();
    if (wave_index() || i >= n) return;
    before = 0;
#pragma unroll
    for (uint32_t w = 0; w < kSortWaves; ++w) before += counts[w][lane_id()];
    out[first + before] = (uint64_t)(mine == kPadding ? kNoToken : mine) << 32 | (uint32_t)(first + i);
}

// The sorted chunks in one order: an element's place is the number of smaller
// ones, a search in each other chunk, four chunks at a time and eight places in
// each (by halves 14,003 rows took 4 us more).  Blocks from `ranks` on write zeros over `fill` rows.
constexpr uint32_t kRankThreads = 256;
__global__ __launch_bounds__(kRankThreads) void k_embed_rank(const uint64_t* chunk, uint32_t rows, uint32_t chunks, uint64_t* order,
                                                       uint32_t ranks, float* out, uint32_t fill, uint32_t dim, uint64_t stride) {
    if (blockIdx.x >= ranks) {
        fill_zeros(out, fill, dim, stride, blockIdx.x - ranks, gridDim.x - ranks);
        return;
    }
    const uint32_t i = blockIdx.x * kRankThreads + threadIdx.x;
    if (i >= rows) return;
    const uint64_t key = chunk[i];
    const uint32_t own = i / kSortChunk;
    uint32_t rank = i % kSortChunk;
    constexpr int kAtOnce = 4, kWays = 8;
    for (uint32_t c = 0; c < chunks; c += kAtOnce) {
        uint32_t at[kAtOnce] = {}, len[kAtOnce];
        const uint64_t* in[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            len[k] = c + k < chunks && c + k != own ? min(rows - (c + k) * kSortChunk, kSortChunk) : 0;
            in[k] = len[k] ? chunk + (c + k) * kSortChunk : chunk;
        }
#pragma unroll
        for (uint32_t step = kSortChunk / kWays; step; step /= kWays) {
            uint64_t other[kAtOnce][kWays];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
                for (uint32_t w = 0; w < kWays; ++w) other[k][w] = in[k][min(at[k] + (w + 1) * step, max(len[k], 1u)) - 1];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                uint32_t before = 0;
#pragma unroll
                for (uint32_t w = 0; w < kWays; ++w) before += (at[k] + (w + 1) * step <= len[k]) & (other[k][w] < key);
                at[k] += before * step;
            }
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) rank += at[k];
    }
    order[rank] = key;
}

// A wave adds up one unit of the sorted rows, a slice of 64 vectors of columns:
// a run of equal tokens that lies within the unit goes to dweight, one that
// began before it to part[2 unit], one that begins in it and goes on behind it
// to part[2 unit + 1].  A lane reads the key of one row, and the rows' loads,
// each group's while the one before is added up, take it from there.
constexpr int kSumWaves = 4, kSumAtOnce = 8;
template <typename T, bool SHORT>
__global__ __launch_bounds__(kSumWaves* kWave) void k_embed_sum(gd_embed_grad io, const uint64_t* order, uint32_t unit,
                                                                uint32_t units, uint32_t dim, float* part) {
    typedef Columns<T, SHORT> Cols;
    constexpr int E = Cols::E;
    const uint32_t u = blockIdx.x * kSumWaves + wave_index();
    if (u >= units) return;
    const uint32_t begin = u * unit, rows = (uint32_t)io.rows, all = min(unit, rows - begin);
    const uint64_t key = order[begin + min((uint32_t)lane_id(), all - 1)];
    const uint32_t key_token = (uint32_t)(key >> 32), key_row = (uint32_t)key;
    const uint32_t ahead = (uint32_t)(order[begin - (begin != 0)] >> 32), behind = (uint32_t)(order[min(begin + all, rows - 1)] >> 32);
    const uint32_t n = min((uint32_t)popc64(ballot(key_token != kNoToken)), all);  // padding is behind all others
    if (n == 0) return;
    const Cols cols(blockIdx.y * (kWave * E) + (uint32_t)lane_id() * E, dim);
    const auto load = [&](u4 (&d)[kSumAtOnce], uint32_t i) {
#pragma unroll
        for (int k = 0; k < kSumAtOnce; ++k)
            d[k] = cols.load((const T*)io.dy + (uint64_t)lane_value(key_row, (int)min(i + k, n - 1)) * io.dy_stride);
    };
    u4 next[kSumAtOnce];
    load(next, 0);
    uint32_t run = lane_value(key_token, 0);
    const bool joins = begin && ahead == run;  // the first run began before
    const bool goes_on = n == all && begin + n < rows && behind == lane_value(key_token, (int)n - 1);  // the last run goes on
    float sum[E];
#pragma unroll
    for (int j = 0; j < E; ++j) sum[j] = 0.0f;
    bool first = true;
    const auto flush = [&](bool last) {
        const bool share = first && joins, open = !share && last && goes_on;
        float* const to = share || open ? part + ((uint64_t)u * 2 + open) * dim : io.dweight + (uint64_t)run * io.dweight_stride;
        cols.put(to, sum, share || open ? 1.0f : io.scale, !(share || open) && io.accumulate != 0);
    };
    for (uint32_t i = 0; i < n; i += kSumAtOnce) {
        u4 d[kSumAtOnce];
#pragma unroll
        for (int k = 0; k < kSumAtOnce; ++k) d[k] = next[k];
        if (i + kSumAtOnce < n) load(next, i + kSumAtOnce);
#pragma unroll
        for (int k = 0; k < kSumAtOnce; ++k) {
            if (i + k >= n) break;
            const uint32_t t = lane_value(key_token, (int)(i + k));
            if (t != run) {
                flush(false);
                run = t, first = false;
#pragma unroll
                for (int j = 0; j < E; ++j) sum[j] = 0.0f;
            }
            Cols::add(sum, d[k]);
        }
    }
    flush(true);
}

// Runs that cross units: block u takes the one that begins in unit u, eight
// waves a share of its units each, joined in 64 bits.
constexpr int kRunWaves = 8;
__global__ __launch_bounds__(kRunWaves* kWave) void k_embed_join(gd_embed_grad io, const uint64_t* order, uint32_t unit,
                                                                 uint32_t units, uint32_t dim, const float* part) {
    __shared__ double lds[kRunWaves][kWave * 4];
    const uint32_t u = blockIdx.x;
    const auto token = [&](uint64_t i) { return (uint32_t)(order[i] >> 32); };
    const uint64_t begin = (uint64_t)u * unit;
    const uint32_t run = token(begin + unit - 1), behind = token(begin + unit), ahead = token(begin - (u != 0));
    if (run == kNoToken || behind != run || (u && ahead == run)) return;  // it ends with the unit, or began before it
    uint32_t last = u + 1, past = units;  // the last unit that it reaches, 64 looked at in turn
    while (past - last > 1) {
        const uint32_t step = (past - last - 1 + kWave - 1) / kWave, mid = last + (lane_id() + 1) * step;
        const uint64_t within = ballot(mid < past && token((uint64_t)min(mid, past - 1) * unit) == run);
        last += popc64(within) * step;
        past = min(past, last + step);
    }
    const uint32_t c = min(blockIdx.y * (kWave * 4) + (uint32_t)lane_id() * 4, dim);
    const int n = (int)(dim - c);
    double s[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 4
    for (uint32_t w = u + wave_index(); w <= last; w += kRunWaves) {
        const Pack<float, 4> p = load_some<4>(part + ((uint64_t)w * 2 + (w == u)) * dim + c, n);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] += p.v[j];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) lds[wave_index()][j * kWave + lane_id()] = s[j];
    __syncthreads();
    if (wave_index()) return;
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        double all = 0.0;
#pragma unroll
        for (int w = 0; w < kRunWaves; ++w) all += lds[w][j * kWave + lane_id()];
        v[j] = (float)all;
    }
    put_gradient<4>(io.dweight + (uint64_t)run * io.dweight_stride + c, v, io.scale, n, io.accumulate != 0);
}

template <typename T>
hipError_t launch_embed(const gd_embed_io& io, uint32_t vocab, uint32_t dim, bool wide, hipStream_t st) {
    constexpr uint32_t E = 16 / sizeof(T);
    const uint32_t vecs = (dim + E - 1) / E;
    const auto run = [&](auto lanes, auto each) {
        constexpr uint32_t kRows = kBlock / lanes();
        const uint32_t blocks = (uint32_t)std::min<uint64_t>((io.rows + kRows - 1) / kRows, 1u << 20);
        k_embed<T, lanes(), each()><<<dim3(blocks), dim3(kBlock), 0, st>>>(io, vocab, dim, wide);
        return hipGetLastError();
    };
    using std::integral_constant;
    if (vecs <= 8) return run(integral_constant<int, 8>(), integral_constant<int, 1>());
    if (vecs <= 16) return run(integral_constant<int, 16>(), integral_constant<int, 1>());
    if (vecs <= 64) return run(integral_constant<int, 64>(), integral_constant<int, 1>());
    if (vecs <= 128) return run(integral_constant<int, 64>(), integral_constant<int, 2>());
    return run(integral_constant<int, 64>(), integral_constant<int, 4>());
}

}  // namespace gd

struct gd_embed {
    int device = 0;
    uint32_t vocab = 0, dim = 0;
    int type = GD_F32;
    uint64_t max_rows = 0;
    uint64_t* chunk = nullptr;  // [max_rows] keys sorted by chunk
    uint64_t* order = nullptr;  // [max_rows] keys sorted
    float* part = nullptr;      // [most_units][2][dim]
    gd::DeviceMemory mem;
};

extern "C" {

gd_status gd_embed_create(gd_embed** out, uint32_t vocab, uint32_t dim, gd_dtype type, uint64_t max_rows) {
    if (!out) return GD_ERR_ARG;
    *out = nullptr;
    const int ty = gd::enum_int(&type);
    if (vocab == 0 || vocab > 0x7FFFFFFFu || dim == 0 || dim > gd::kEmbedMaxDim || max_rows > gd::kEmbedMaxRows ||
        ty < GD_F32 || ty > GD_F16)
        return GD_ERR_ARG;
    gd_embed* e = new (std::nothrow) gd_embed();
    if (!e) return GD_ERR_OOM;
    e->vocab = vocab;
    e->dim = dim;
    e->type = ty;
    e->max_rows = max_rows;
    gd_status st = GD_OK;
    try {
        if (hipGetDevice(&e->device) != hipSuccess) st = GD_ERR_HIP;
        else if (!e->mem.alloc(&e->chunk, max_rows) || !e->mem.alloc(&e->order, max_rows) ||
                 !e->mem.alloc(&e->part, gd::most_units(max_rows, gd::slice_count(dim, ty)) * 2 * dim))
            st = GD_ERR_OOM;
    } catch (const std::bad_alloc&) {
        st = GD_ERR_OOM;
    }
    if (st != GD_OK) {
        delete e;
        return st;
    }
    *out = e;
    return GD_OK;
}

void gd_embed_destroy(gd_embed* e) {
    if (!e) return;
    gd::DeviceGuard guard(e->device);
    delete e;
}

gd_status gd_embed_forward(gd_embed* e, const gd_embed_io* io, void* stream) {
    if (!e || !io || !std::isfinite(io->scale)) return GD_ERR_ARG;
    const int wide = gd::enum_int(&io->index);
    if (wide < GD_I32 || wide > GD_I64 || io->weight_stride < e->dim || !io->weight) return GD_ERR_ARG;
    if (io->rows == 0) return GD_OK;
    if (!io->tokens || !io->y || io->y_stride < e->dim) return GD_ERR_ARG;
    gd::DeviceGuard guard(e->device);
    if (!guard.ok) return GD_ERR_HIP;
    const hipError_t r = gd::with_type(e->type, [&](auto zero) {
        return gd::launch_embed<decltype(zero)>(*io, e->vocab, e->dim, wide == GD_I64, (hipStream_t)stream);
    });
    return r == hipSuccess ? GD_OK : GD_ERR_HIP;
}

gd_status gd_embed_backward(gd_embed* e, const gd_embed_grad* io, void* stream) {
    if (!e || !io || io->rows > e->max_rows || !std::isfinite(io->scale)) return GD_ERR_ARG;
    const int wide = gd::enum_int(&io->index);
    if (wide < GD_I32 || wide > GD_I64 || !io->dweight || io->dweight_stride < e->dim) return GD_ERR_ARG;
    if (io->rows && (!io->tokens || !io->dy || io->dy_stride < e->dim)) return GD_ERR_ARG;
    if (!io->rows && io->accumulate) return GD_OK;
    gd::DeviceGuard guard(e->device);
    if (!guard.ok) return GD_ERR_HIP;
    const hipStream_t st = (hipStream_t)stream;
    const uint32_t per_fill = std::max(gd::kFillFloats / e->dim, 1u);
    const uint64_t fills = io->accumulate ? 0 : ((uint64_t)e->vocab + per_fill - 1) / per_fill;
    const uint32_t slices = gd::slice_count(e->dim, e->type);
    if (io->rows <= gd::kFewRows && slices <= gd::kFewSlices && fills <= gd::kFewBlocks) {
        const hipError_t r = gd::with_type(e->type, [&](auto zero) {
            using T = decltype(zero);
            const auto kernel = e->dim * sizeof(T) < 16 ? gd::k_embed_few<T, true> : gd::k_embed_few<T, false>;
            kernel<<<dim3((uint32_t)(io->rows + fills)), dim3(gd::kFewThreads), 0, st>>>(*io, e->vocab, e->dim, wide == GD_I64,
                                                                                          (uint32_t)fills, per_fill);
            return hipGetLastError();
        });
        return r == hipSuccess ? GD_OK : GD_ERR_HIP;
    }
    const uint32_t chunks = (uint32_t)((io->rows + gd::kSortChunk - 1) / gd::kSortChunk);
    // The zeros are written beside the sort, and where its chunks are joined most of them beside that: each of the two
    // launches waits on memory for some microseconds, of which the zeros need not be waited for.
    const uint32_t first = io->accumulate ? 0 : chunks > 1 ? e->vocab / 4 : e->vocab, rest = io->accumulate ? 0 : e->vocab - first;
    const uint32_t sorts = chunks * gd::kChunkBlocks;
    gd::k_embed_sort<<<dim3(sorts + gd::fill_blocks(first, e->dim, gd::kSortThreads)), dim3(gd::kSortThreads), 0, st>>>(
        *io, e->vocab, e->dim, wide == GD_I64, sorts, chunks > 1 ? e->chunk : e->order, first);
    hipError_t r = hipGetLastError();
    if (r != hipSuccess) return GD_ERR_HIP;
    if (!io->rows) return GD_OK;
    if (chunks > 1) {
        const uint32_t ranks = (uint32_t)((io->rows + gd::kRankThreads - 1) / gd::kRankThreads);
        gd::k_embed_rank<<<dim3(ranks + gd::fill_blocks(rest, e->dim, gd::kRankThreads)), dim3(gd::kRankThreads), 0, st>>>(
            e->chunk, (uint32_t)io->rows, chunks, e->order, ranks, io->dweight + (uint64_t)first * io->dweight_stride, rest, e->dim,
            io->dweight_stride);
        if (hipGetLastError() != hipSuccess) return GD_ERR_HIP;
    }
    const uint32_t unit = gd::unit_rows(io->rows, slices);
    const uint32_t units = (uint32_t)((io->rows + unit - 1) / unit);
    r = gd::with_type(e->type, [&](auto zero) {
        using T = decltype(zero);
        const auto kernel = e->dim * sizeof(T) < 16 ? gd::k_embed_sum<T, true> : gd::k_embed_sum<T, false>;
        kernel<<<dim3((units + gd::kSumWaves - 1) / gd::kSumWaves, slices),
                 dim3(gd::kSumWaves * gd::kWave), 0, st>>>(*io, e->order, unit, units, e->dim, e->part);
        return hipGetLastError();
    });
    if (r != hipSuccess) return GD_ERR_HIP;
    if (units > 1) {
        gd::k_embed_join<<<dim3(units - 1, (e->dim + gd::kWave * 4 - 1) / (gd::kWave * 4)), dim3(gd::kRunWaves * gd::kWave),
                           0, st>>>(*io, e->order, unit, units, e->dim, e->part);
        if (hipGetLastError() != hipSuccess) return GD_ERR_HIP;
    }
    return GD_OK;
}

}  // extern "C"
