// Embedding: rows of a weight looked up by token and scaled, and the weight's
// gradient, the sum over the rows of each token.
//
//   y[i] = scale weight[t_i],   dweight[v] = scale sum over i with t_i = v of dy[i]
//
// Both are bound by memory.  The gradient is formed without atomics on values,
// so that it is the same on every run: rows are sorted by (token, row), the
// sorted order is cut into equal units, a wave adds up a unit's runs of equal
// tokens, and runs that cross units are joined from their units' shares.  Cut
// by units and not by tokens, the work is even however often a token occurs
// (in text the commonest word is a twentieth of all).  All of dweight is
// written with zeros in the launch that sorts, which hides the sort behind it.

#include <cmath>
#include <new>

#include "gd.h"
#include "gd_host.hpp"
#include "gd_rows.hpp"

namespace gd {

constexpr uint32_t kEmbedMaxDim = 1u << 20, kEmbedMaxRows = 1u << 24;
constexpr uint32_t kNoToken = 0xFFFFFFFFu;  // padding: sorted behind every token
constexpr uint32_t kSortChunk = 2048, kSortThreads = 1024;

// Sorted rows a unit holds, by the number of rows: few rows make many small units for the sake of parallel work, many
// make larger ones, of which fewer partial sums are written.
__host__ __device__ constexpr uint32_t unit_rows(uint64_t rows) { return rows <= 4096 ? 16 : rows <= 16384 ? 32 : 64; }
constexpr uint64_t unit_count(uint64_t rows) { return (rows + unit_rows(rows) - 1) / unit_rows(rows); }
// The most units that any number of rows up to this one makes.
constexpr uint64_t most_units(uint64_t rows) { return std::max<uint64_t>(std::min<uint64_t>((rows + 15) / 16, 512), (rows + 63) / 64); }
static_assert(unit_count(4096) == 256 && unit_count(16384) == 512 && unit_count(16385) == 257);

// The token of row i: kNoToken for ids outside the vocabulary.
__device__ __forceinline__ uint32_t token_at(const void* tokens, bool wide, uint64_t i, uint32_t vocab) {
    const int64_t t = wide ? ((const int64_t*)tokens)[i] : (int64_t)((const int32_t*)tokens)[i];
    return t >= 0 && t < (int64_t)vocab ? (uint32_t)t : kNoToken;
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

// Zeros over [rows][dim] at `stride`, the blocks `block` of `blocks` sharing it.
__device__ __forceinline__ void fill_zeros(float* out, uint64_t rows, uint64_t dim, uint64_t stride, uint64_t block,
                                           uint64_t blocks) {
    const Pack<float, 4> zeros = {};
    if (stride == dim) {  // one run
        const uint64_t all = rows * dim;
        for (uint64_t e = (block * kSortThreads + threadIdx.x) * 4; e < all; e += blocks * kSortThreads * 4)
            store_stream<4>(out + e, zeros, (int)min(all - e, (uint64_t)4));
        return;
    }
    for (uint64_t row = block * (kSortThreads / kWave) + wave_index(); row < rows; row += blocks * (kSortThreads / kWave))
        for (uint64_t e = lane_id() * 4; e < dim; e += kWave * 4)
            store_stream<4>(out + row * stride + e, zeros, (int)min(dim - e, (uint64_t)4));
}

// Blocks below `chunks` sort 2,048 rows each by (token, row), bitonic: element
// e 1024 + t is thread t's, so that exchanges at a distance below 64 stay
// within a wave, the farthest within a thread, and the others pass through LDS.
// The other blocks write zeros.
__global__ __launch_bounds__(kSortThreads) void k_embed_sort(gd_embed_grad io, uint32_t vocab, uint32_t dim, bool wide,
                                                             uint32_t chunks, uint64_t* out) {
    if (blockIdx.x >= chunks) {
        fill_zeros(io.dweight, vocab, dim, io.dweight_stride, blockIdx.x - chunks, gridDim.x - chunks);
        return;
    }
    __shared__ uint64_t lds[kSortChunk];
    const uint64_t first = (uint64_t)blockIdx.x * kSortChunk;
    const uint32_t n = (uint32_t)min(io.rows - first, (uint64_t)kSortChunk);
    uint64_t key[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const uint32_t i = e * kSortThreads + threadIdx.x;
        key[e] = ~0ull;
        if (i < n) key[e] = (uint64_t)token_at(io.tokens, wide, first + i, vocab) << 32 | (uint32_t)(first + i);
    }
    uint32_t all = 2;  // a power of two that holds them: what lies behind is not looked at
    while (all < n) all *= 2;
    for (uint32_t k = 2; k <= all; k *= 2)
        for (uint32_t d = k / 2; d; d /= 2) {
            if (d == kSortThreads) {  // k is the whole chunk: ascending
                const uint64_t lo = min(key[0], key[1]), hi = max(key[0], key[1]);
                key[0] = lo, key[1] = hi;
                continue;
            }
            uint64_t other[2];
            if (d >= (uint32_t)kWave) {
                __syncthreads();
                lds[threadIdx.x] = key[0], lds[kSortThreads + threadIdx.x] = key[1];
                __syncthreads();
                other[0] = lds[threadIdx.x ^ d], other[1] = lds[(kSortThreads + threadIdx.x) ^ d];
            } else {
                other[0] = __shfl_xor((unsigned long long)key[0], (int)d);
                other[1] = __shfl_xor((unsigned long long)key[1], (int)d);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t i = e * kSortThreads + threadIdx.x;
                key[e] = ((i & d) == 0) == ((i & k) == 0) ? min(key[e], other[e]) : max(key[e], other[e]);
            }
        }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const uint32_t i = e * kSortThreads + threadIdx.x;
        if (i < n) out[first + i] = key[e];
    }
}

// The sorted chunks in one order: an element's place is the number of smaller
// ones, a binary search in each other chunk, four of them at a time.
__global__ __launch_bounds__(kBlock) void k_embed_rank(const uint64_t* chunk, uint32_t rows, uint32_t chunks,
                                                       uint64_t* order) {
    const uint32_t i = blockIdx.x * kBlock + threadIdx.x;
    if (i >= rows) return;
    const uint64_t key = chunk[i];
    const uint32_t own = i / kSortChunk;
    uint32_t rank = i % kSortChunk;
    constexpr int kAtOnce = 4;
    for (uint32_t c = 0; c < chunks; c += kAtOnce) {
        uint32_t at[kAtOnce] = {}, len[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            len[k] = c + k < chunks && c + k != own ? min(rows - (c + k) * kSortChunk, kSortChunk) : 0;
#pragma unroll
        for (uint32_t step = kSortChunk; step; step /= 2)
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k)
                if (at[k] + step <= len[k] && chunk[(c + k) * kSortChunk + at[k] + step - 1] < key) at[k] += step;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) rank += at[k];
    }
    order[rank] = key;
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

// A wave adds up one unit of the sorted rows, a slice of 64 vectors of columns:
// a run of equal tokens that lies within the unit goes to dweight, one that
// began before it to part[2 unit], one that begins in it and goes on behind it
// to part[2 unit + 1].
constexpr int kSumWaves = 4, kSumAtOnce = 8;
template <typename T>
__global__ __launch_bounds__(kSumWaves* kWave) void k_embed_sum(gd_embed_grad io, const uint64_t* order, uint32_t unit,
                                                                uint32_t units, uint32_t dim, float* part) {
    constexpr int E = 16 / sizeof(T);
    const uint32_t u = blockIdx.x * kSumWaves + wave_index();
    if (u >= units) return;
    const uint32_t c = min(blockIdx.y * (kWave * E) + (uint32_t)lane_id() * E, dim);
    const int n = (int)(dim - c);
    const uint64_t begin = (uint64_t)u * unit, end = min(begin + unit, io.rows);
    const auto token = [&](uint64_t i) { return (uint32_t)(order[i] >> 32); };
    const bool joins = begin && token(begin - 1) == token(begin);        // the first run began before the unit
    const bool goes_on = end < io.rows && token(end) == token(end - 1);  // the last run goes on behind it
    float sum[E];
#pragma unroll
    for (int j = 0; j < E; ++j) sum[j] = 0.0f;
    uint32_t run = token(begin);
    bool first = true;
    const auto flush = [&](bool last) {
        if (run == kNoToken) return;
        float* shares = part + (uint64_t)u * 2 * dim + c;
        if (first && joins) {
            Pack<float, E> v;
#pragma unroll
            for (int j = 0; j < E; ++j) v.v[j] = sum[j];
            store_some<E>(shares, v, n);
        } else if (last && goes_on) {
            Pack<float, E> v;
#pragma unroll
            for (int j = 0; j < E; ++j) v.v[j] = sum[j];
            store_some<E>(shares + dim, v, n);
        } else {
            put_gradient<E>(io.dweight + (uint64_t)run * io.dweight_stride + c, sum, io.scale, n, io.accumulate != 0);
        }
    };
    for (uint64_t i = begin; i < end; i += kSumAtOnce) {
        uint32_t t[kSumAtOnce];
        Pack<T, E> d[kSumAtOnce];
#pragma unroll
        for (int k = 0; k < kSumAtOnce; ++k) {
            const uint64_t key = order[min(i + k, end - 1)];
            t[k] = (uint32_t)(key >> 32);
            d[k] = load_some<E>((const T*)io.dy + (uint64_t)(uint32_t)key * io.dy_stride + c,
                                i + k < end && t[k] != kNoToken ? n : 0);
        }
#pragma unroll
        for (int k = 0; k < kSumAtOnce; ++k) {
            if (i + k >= end) break;
            if (t[k] != run) {
                flush(false);
                run = t[k], first = false;
#pragma unroll
                for (int j = 0; j < E; ++j) sum[j] = 0.0f;
            }
#pragma unroll
            for (int j = 0; j < E; ++j) sum[j] += (float)d[k].v[j];
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
    const uint32_t run = token((uint64_t)u * unit + unit - 1);
    if (run == kNoToken || token((uint64_t)(u + 1) * unit) != run) return;       // it ends with the unit
    if (u && token((uint64_t)u * unit - 1) == run) return;                       // it began before
    uint32_t last = u + 1, past = units;                                          // the last unit that it reaches
    while (past - last > 1) {
        const uint32_t mid = last + (past - last) / 2;
        if (token((uint64_t)mid * unit) == run) last = mid;
        else past = mid;
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
                 !e->mem.alloc(&e->part, gd::most_units(max_rows) * 2 * dim))
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
    const uint32_t chunks = (uint32_t)((io->rows + gd::kSortChunk - 1) / gd::kSortChunk);
    // blocks of zeros: two a compute unit, fewer where there is less to write
    const uint64_t zeros = io->accumulate ? 0 : ((uint64_t)e->vocab * e->dim + 4 * gd::kSortThreads - 1) / (4 * gd::kSortThreads);
    const uint32_t fill = (uint32_t)std::min<uint64_t>(zeros, 512);
    gd::k_embed_sort<<<dim3(chunks + fill), dim3(gd::kSortThreads), 0, st>>>(*io, e->vocab, e->dim, wide == GD_I64, chunks,
                                                                            chunks > 1 ? e->chunk : e->order);
    hipError_t r = hipGetLastError();
    if (r != hipSuccess) return GD_ERR_HIP;
    if (!io->rows) return GD_OK;
    if (chunks > 1) {
        gd::k_embed_rank<<<dim3((uint32_t)((io->rows + gd::kBlock - 1) / gd::kBlock)), dim3(gd::kBlock), 0, st>>>(
            e->chunk, (uint32_t)io->rows, chunks, e->order);
        if (hipGetLastError() != hipSuccess) return GD_ERR_HIP;
    }
    const uint32_t unit = gd::unit_rows(io->rows), units = (uint32_t)gd::unit_count(io->rows);
    r = gd::with_type(e->type, [&](auto zero) {
        using T = decltype(zero);
        constexpr uint32_t kColumns = gd::kWave * 16 / sizeof(T);
        gd::k_embed_sum<T><<<dim3((units + gd::kSumWaves - 1) / gd::kSumWaves, (e->dim + kColumns - 1) / kColumns),
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
