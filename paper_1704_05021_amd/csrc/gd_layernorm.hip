// Layer norm of rows with the residual's addition, forward (output in the
// type or in 8 bits with a scale per row) and backward.
//
//   h = x + residual,  c = h - mean(h),  y = c / sqrt(mean(c^2) + eps) * weight + bias
//   a = dy weight, xhat = c rstd:  dx = rstd (a - mean(a) - xhat mean(a xhat)) + dsum
//   dweight = sum over rows of dy xhat,  dbias = sum over rows of dy
//
// One pass over memory: a row lies in registers between its sums and its
// output.  All sums of a row are formed at once, behind one barrier, from
// d = h - h[0] in 64 bits: mean = h[0] + mean(d), mean(c^2) = mean(d^2) -
// mean(d)^2.  The shift by an element keeps the difference of the squares
// exact where a row lies far from zero (its mean 10^4 times its spread), and
// sums in 64 bits make the result the same whatever the split of the row.

#include <cmath>
#include <new>

#include "gd.h"
#include "gd_host.hpp"
#include "gd_rows.hpp"

namespace gd {

constexpr uint32_t kLayerNormMaxDim = 32768;
constexpr uint32_t kLayerNormParts = 512;        // partial sums of the weight's and the bias's gradient, at most
constexpr uint32_t kLayerNormBackWaves = 4096;   // waves of the backward pass: four a SIMD, as many as its registers hold
constexpr uint32_t kLayerNormMaxBlocks = 1u << 20;

// What a row's factor and shift come to.
struct RowStats {
    double mean;
    float rstd;
    // h less the mean: in 64 bits and rounded once, as elementary operations give it, so that codes of 8 bits come out the
    // same; or in 32 bits by the mean's two halves, two roundings, which is far below a 16-bit result's own.
    __device__ __forceinline__ float centred(float h, float high, float low) const { return (h - high) - low; }
    __device__ __forceinline__ float centred(float h) const { return (float)((double)h - mean); }
};
__device__ __forceinline__ RowStats row_stats(double pivot, double d, double dd, double per_dim, float eps) {
    const double m = d * per_dim, var = dd * per_dim - m * m;
    // a spread below the sums' rounding may come out a hair under zero; NaN stays
    return {pivot + m, (float)rsqrt((var < 0.0 ? 0.0 : var) + (double)eps)};
}

// How a row of dim elements divides into vectors of eight.
enum RowEnds {
    kShort = 0,  // dim is below 8: read element by element
    kRagged = 1, // the last vector is the one that ends with the row; what it shares with the one before is left out
    kWhole = 2,
    kFull = 3    // and every thread has one
};

// The vector of eight elements that a thread takes of a row: where it lies, and which of its elements are the thread's.
template <int ENDS>
struct Place {
    uint32_t at, dim, mine;  // mine: a bit for each
    __device__ __forceinline__ Place(uint32_t e, uint32_t dim) : dim(dim) {
        at = ENDS == kShort ? 0 : min(e, dim - 8);
        if (ENDS == kFull)
            at = e, mine = 0xFF;
        else if (ENDS == kWhole)
            mine = e < dim ? 0xFF : 0;
        else if (ENDS == kRagged)
            mine = 0xFFu << min(e - at, 8u) & 0xFF;
        else
            mine = e ? 0 : (1u << dim) - 1;
    }
    // Every load is made, by every thread and whatever is asked for: loads behind conditions wait for one another
    // (8192 x 4096 in bfloat16 forward took 88 us so).
    template <typename T>
    __device__ __forceinline__ Pack<T, 8> load(const T* row) const {
        if constexpr (ENDS == kShort) {
            Pack<T, 8> r;
#pragma unroll
            for (int j = 0; j < 8; ++j) r.v[j] = row[min((uint32_t)j, dim - 1)];
            return r;
        }
        return load_pack<8>(row + at);
    }
    // In binary32, `rest` in place of what is not the thread's.
    template <typename T>
    __device__ __forceinline__ void get(float (&v)[8], const Pack<T, 8>& raw, float rest) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (float)raw.v[j];
        if (ENDS == kFull || mine == 0xFF) return;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = ENDS < kWhole && mine >> j & 1 ? v[j] : rest;
    }
    template <typename T>
    __device__ __forceinline__ void store(T* row, const Pack<T, 8>& r, bool on) const {
        if (!on) return;
        if (mine == 0xFF) {
            if constexpr (sizeof(r) % 16 == 0)
                store_stream<8>(row + at, r, 8);
            else
                store_pack<8>(row + at, r);
        } else if (ENDS < kWhole) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (mine >> j & 1) row[at + j] = r.v[j];
        }
    }
};

template <typename T, int WAVES, int V, int ENDS, bool INT8>
__global__ __launch_bounds__(NormShape<WAVES>::kThreads) void k_layernorm(gd_layernorm_io io, uint32_t dim, double per_dim) {
    using S = NormShape<WAVES>;
    __shared__ double lds_sum[2][S::kThreads / kWave];
    __shared__ uint32_t lds_max[S::kThreads / kWave];
    const uint32_t t = threadIdx.x % S::kRow;
    constexpr bool kOnce = INT8 || sizeof(T) == 4;  // c is rounded once, and not twice
    const bool add = io.residual != nullptr, shift = io.bias != nullptr;
    // every wave of a block takes the same number of turns (the last ones of rows past the end write nothing)
    for (uint64_t first = (uint64_t)blockIdx.x * S::kRows; first < io.rows; first += (uint64_t)gridDim.x * S::kRows) {
        const uint64_t row = first + threadIdx.x / S::kRow, from = min(row, io.rows - 1);
        const bool on = row < io.rows;
        // without a residual or a bias what is there is read in their place, and not used
        const T* x = (const T*)io.x + from * io.x_stride;
        const T* r = add ? (const T*)io.residual + from * io.residual_stride : x;
        const T* b = (const T*)(shift ? io.bias : io.weight);
        const T x0 = *x, r0 = *r;
        Pack<T, 8> xs[V], rs[V], ws[V], bs[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const Place<ENDS> p((t + i * S::kRow) * 8, dim);
            xs[i] = p.load(x);
            rs[i] = p.load(r);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const Place<ENDS> p((t + i * S::kRow) * 8, dim);
            ws[i] = p.load((const T*)io.weight);
            bs[i] = p.load(b);
        }
        // elements past the row's end are its first, which adds nothing to the sums
        const float pivot = add ? (float)x0 + (float)r0 : (float)x0;
        const double from_here = pivot;
        float h[V][8];
        double s[2] = {0.0, 0.0};  // of d and d^2
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const Place<ENDS> p((t + i * S::kRow) * 8, dim);
            float rv[8];
            p.get(h[i], xs[i], (float)x0);
            p.get(rv, rs[i], (float)r0);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                h[i][j] = add ? h[i][j] + rv[j] : h[i][j];
                const double d = (double)h[i][j] - from_here;
                s[0] += d;
                s[1] = fma(d, d, s[1]);
            }
        }
        row_sums<WAVES>(s, lds_sum);
        const RowStats st = row_stats(from_here, s[0], s[1], per_dim, io.eps);
        const float high = (float)st.mean, low = (float)(st.mean - (double)high);
        uint32_t big = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const Place<ENDS> p((t + i * S::kRow) * 8, dim);
            Pack<T, 8> sum, y;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sum.v[j] = (T)h[i][j];
                const float c = kOnce ? st.centred(h[i][j]) : st.centred(h[i][j], high, low);
                h[i][j] = c * st.rstd * (float)ws[i].v[j] + (shift ? (float)bs[i].v[j] : 0.0f);
                y.v[j] = (T)h[i][j];
                if (INT8 && p.mine >> j & 1) big = max(big, __float_as_uint(h[i][j]) & 0x7FFFFFFFu);
            }
            if (io.sum) p.store((T*)io.sum + row * io.sum_stride, sum, on);
            if (!INT8) p.store((T*)io.y + row * io.y_stride, y, on);
        }
        if constexpr (INT8) {
            const RowScale q = row_scale(row_max<WAVES>(big, lds_max));
            if (t == 0 && on) io.y_scale[row] = q.scale;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                Pack<int8_t, 8> y;
#pragma unroll
                for (int j = 0; j < 8; ++j) y.v[j] = quantise(h[i][j], q.step);
                Place<ENDS>((t + i * S::kRow) * 8, dim).store((int8_t*)io.y + row * io.y_stride, y, on);
            }
        }
        if constexpr (WAVES > 1) __syncthreads();  // before the next row's sums
    }
}

__device__ __forceinline__ uint32_t bits_of(float v) { return __float_as_uint(v); }
template <typename T>
__device__ __forceinline__ uint32_t bits_of(T v) {
    uint16_t b;
    __builtin_memcpy(&b, &v, 2);
    return b;
}
template <typename T>
__device__ __forceinline__ float value_of_bits(uint32_t b) {
    T v;
    __builtin_memcpy(&v, &b, sizeof v);
    return (float)v;
}
// Eight elements as they came from memory.  Kept as words: of elements the compiler makes eight values, which it takes apart
// right behind the load, and so waits for the next row before it works on this one.
template <typename T>
struct Words {
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    words w[sizeof(T) / 2];
    __device__ __forceinline__ Words() {}
    __device__ __forceinline__ Words(const Pack<T, 8>& p) { __builtin_memcpy(w, &p, sizeof p); }
    __device__ __forceinline__ operator Pack<T, 8>() const {
        Pack<T, 8> p;
        __builtin_memcpy(&p, w, sizeof p);
        return p;
    }
};

// A block takes several rows, and loads each while it works on the one before;
// its share of the sums over rows goes to part[blockIdx.x]: dweight's, then dbias's.
template <typename T, int WAVES, int V, int ENDS>
__global__ __launch_bounds__(NormShape<WAVES>::kThreads, 4) void k_layernorm_back(gd_layernorm_grad io, uint32_t dim,
                                                                                  double per_dim, float* part) {
    using S = NormShape<WAVES>;
    __shared__ double lds_sum[2][4][S::kThreads / kWave];
    const uint32_t t = threadIdx.x % S::kRow;
    const uint64_t turn = (uint64_t)gridDim.x * S::kRows;
    const bool add = io.dsum != nullptr;
    struct Row {
        Words<T> x[V], dy[V], dsum[V];
        uint32_t first;  // its bits
    };
    const auto place = [&](int i) { return Place<ENDS>((t + i * S::kRow) * 8, dim); };
    const auto load = [&](Row& r, uint64_t first) {
        const uint64_t row = min(first + threadIdx.x / S::kRow, io.rows - 1);
        const T *x = (const T*)io.x + row * io.x_stride, *dy = (const T*)io.dy + row * io.dy_stride;
        const T* dsum = add ? (const T*)io.dsum + row * io.dsum_stride : dy;
        r.first = bits_of(*x);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            r.x[i] = place(i).load(x);
            r.dy[i] = place(i).load(dy);
            r.dsum[i] = place(i).load(dsum);
        }
    };
    constexpr bool kAhead = V == 1;  // more elements a thread leave no registers for it
    Pack<T, 8> ws[V];
    float dw[V][8], db[V][8];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        ws[i] = place(i).load((const T*)io.weight);
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[i][j] = db[i][j] = 0.0f;
    }
    const auto w = [&](int i, int j) { return (float)ws[i].v[j]; };  // not 0 past the row's end, but dy is
    Row next;
    uint64_t first = (uint64_t)blockIdx.x * S::kRows;
    if (kAhead) load(next, first);
    for (uint32_t odd = 0; first < io.rows; first += turn, odd ^= 1) {
        const uint64_t row = first + threadIdx.x / S::kRow;
        const bool on = row < io.rows;
        if (!kAhead) load(next, first);
        const Row r = next;
        if (kAhead && first + turn < io.rows) load(next, first + turn);
        const float x0 = value_of_bits<T>(r.first);
        const double from_here = x0;
        double s[4] = {0.0, 0.0, 0.0, 0.0};  // of d, d^2, a, a d: d and a are 0 past the row's end
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float x[8], g[8];
            place(i).template get<T>(x, r.x[i], x0);
            place(i).template get<T>(g, r.dy[i], 0.0f);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const double d = (double)x[j] - from_here, a = g[j] * w(i, j);
                s[0] += d;
                s[1] = fma(d, d, s[1]);
                s[2] += a;
                s[3] = fma(a, d, s[3]);
            }
        }
        // the two turns' sums lie apart, so one barrier a row is enough
        row_sums<WAVES>(s, lds_sum[odd]);
        const RowStats st = row_stats(from_here, s[0], s[1], per_dim, io.eps);
        const float high = (float)st.mean, low = (float)(st.mean - (double)high);
        const float mean_a = (float)(s[2] * per_dim);
        const float mean_ax = (float)((s[3] - s[2] * (s[0] * per_dim)) * per_dim * st.rstd);  // mean(a xhat)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float x[8], g[8];
            place(i).template get<T>(x, r.x[i], x0);
            place(i).template get<T>(g, r.dy[i], 0.0f);
            const Pack<T, 8> more = r.dsum[i];
            Pack<T, 8> d;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float xhat = st.centred(x[j], high, low) * st.rstd;
                dw[i][j] += S::kRows == 1 || on ? g[j] * xhat : 0.0f;
                db[i][j] += S::kRows == 1 || on ? g[j] : 0.0f;
                const float v = st.rstd * (g[j] * w(i, j) - mean_a - xhat * mean_ax);
                d.v[j] = (T)(add ? v + (float)more.v[j] : v);
            }
            place(i).store((T*)io.dx + row * io.dx_stride, d, on);
        }
    }
    if (!part) return;
    if constexpr (S::kRows > 1) {  // the block's rows join before the partial is written
        __shared__ float lds_dw[S::kRows][2 * V * 8 * S::kRow];
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                lds_dw[threadIdx.x / S::kRow][(i * 8 + j) * S::kRow + t] = dw[i][j];
                lds_dw[threadIdx.x / S::kRow][((V + i) * 8 + j) * S::kRow + t] = db[i][j];
            }
        __syncthreads();
        if (threadIdx.x >= (uint32_t)S::kRow) return;
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int r = 1; r < S::kRows; ++r) {
                    dw[i][j] += lds_dw[r][(i * 8 + j) * S::kRow + t];
                    db[i][j] += lds_dw[r][((V + i) * 8 + j) * S::kRow + t];
                }
    }
    const auto put = [&](float* out, float* partial, const float (&v)[V][8]) {
        float* to = gridDim.x > 1 ? partial : out;  // few rows: the block's share is all of it
        if (!to) return;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const Place<ENDS> p = place(i);
            Pack<float, 8> d;
            if (to == out && io.accumulate) d = p.load(to);
#pragma unroll
            for (int j = 0; j < 8; ++j) d.v[j] = to == out && io.accumulate ? d.v[j] + v[i][j] : v[i][j];
            p.store(to, d, true);
        }
    };
    put(io.dweight, part + (uint64_t)blockIdx.x * 2 * dim, dw);
    put(io.dbias, part + ((uint64_t)blockIdx.x * 2 + 1) * dim, db);
}

// dweight and dbias from the blocks' shares, in 64 bits and a fixed order: 32
// columns by 32 groups of shares a block, a wave reads two 128-byte runs at a time.
constexpr int kJoinColumns = 32, kJoinGroups = 32;
__global__ __launch_bounds__(kJoinColumns* kJoinGroups) void k_layernorm_join(const float* part, uint32_t parts,
                                                                              uint32_t dim, float* dweight, float* dbias,
                                                                              bool accumulate) {
    __shared__ double lds[kJoinGroups][kJoinColumns];
    const uint32_t c = threadIdx.x % kJoinColumns, g = threadIdx.x / kJoinColumns;
    const uint32_t e = blockIdx.x * kJoinColumns + c;  // of both gradients laid end to end
    double s = 0.0;
    if (e < 2 * dim)
#pragma unroll 8
        for (uint32_t p = g; p < parts; p += kJoinGroups) s += part[(uint64_t)p * 2 * dim + e];
    lds[g][c] = s;
    __syncthreads();
    float* out = e < dim ? dweight : dbias;
    if (g != 0 || e >= 2 * dim || !out) return;
    out += e < dim ? e : e - dim;
    s = accumulate ? (double)*out : 0.0;
#pragma unroll
    for (int i = 0; i < kJoinGroups; ++i) s += lds[i][c];
    *out = (float)s;
}

template <typename T, int WAVES, int V, int ENDS>
hipError_t launch_layernorm(const gd_layernorm_io& io, uint32_t dim, hipStream_t st) {
    using S = NormShape<WAVES>;
    const uint32_t blocks = (uint32_t)std::min<uint64_t>((io.rows + S::kRows - 1) / S::kRows, kLayerNormMaxBlocks);
    if (io.y_scale)
        k_layernorm<T, WAVES, V, ENDS, true><<<dim3(blocks), dim3(S::kThreads), 0, st>>>(io, dim, 1.0 / dim);
    else
        k_layernorm<T, WAVES, V, ENDS, false><<<dim3(blocks), dim3(S::kThreads), 0, st>>>(io, dim, 1.0 / dim);
    return hipGetLastError();
}

template <typename T, int WAVES, int V, int ENDS>
hipError_t launch_layernorm_back(const gd_layernorm_grad& io, uint32_t dim, float* part, hipStream_t st) {
    using S = NormShape<WAVES>;
    const bool sums = io.dweight || io.dbias;
    const uint32_t most = std::min(kLayerNormBackWaves * kWave / S::kThreads, kLayerNormParts);
    const uint64_t turns = (io.rows + S::kRows - 1) / S::kRows;
    // few rows go to one block, which writes the gradients itself
    const bool one = turns <= 4 && turns * dim <= 1u << 14;
    const uint32_t parts = one ? (turns != 0) : (uint32_t)std::min<uint64_t>(turns, most);
    if (parts) {
        k_layernorm_back<T, WAVES, V, ENDS><<<dim3(parts), dim3(S::kThreads), 0, st>>>(io, dim, 1.0 / dim, sums ? part : nullptr);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!sums || parts == 1 || (!parts && io.accumulate)) return hipSuccess;
    k_layernorm_join<<<dim3((2 * dim + kJoinColumns - 1) / kJoinColumns), dim3(kJoinColumns * kJoinGroups), 0, st>>>(
        part, parts, dim, io.dweight, io.dbias, io.accumulate != 0);
    return hipGetLastError();
}

template <int WAVES, int V, typename F>
hipError_t with_ends(uint32_t dim, F f) {
    if (dim == WAVES * kWave * 8 * V) return f(std::integral_constant<int, kFull>());
    if constexpr (WAVES == 1)
        if (dim < 8) return f(std::integral_constant<int, kShort>());
    return dim % 8 ? f(std::integral_constant<int, kRagged>()) : f(std::integral_constant<int, kWhole>());
}

}  // namespace gd

struct gd_layernorm {
    int device = 0;
    uint32_t dim = 0;
    int type = GD_F32;
    float* part = nullptr;  // [kLayerNormParts][2][dim]
    gd::DeviceMemory mem;
};

extern "C" {

gd_status gd_layernorm_create(gd_layernorm** out, uint32_t dim, gd_dtype type) {
    if (!out) return GD_ERR_ARG;
    *out = nullptr;
    const int ty = gd::enum_int(&type);
    if (dim == 0 || dim > gd::kLayerNormMaxDim || ty < GD_F32 || ty > GD_F16) return GD_ERR_ARG;
    gd_layernorm* n = new (std::nothrow) gd_layernorm();
    if (!n) return GD_ERR_OOM;
    n->dim = dim;
    n->type = ty;
    gd_status st = GD_OK;
    try {
        if (hipGetDevice(&n->device) != hipSuccess) st = GD_ERR_HIP;
        else if (!n->mem.alloc(&n->part, (size_t)gd::kLayerNormParts * 2 * dim)) st = GD_ERR_OOM;
    } catch (const std::bad_alloc&) {
        st = GD_ERR_OOM;
    }
    if (st != GD_OK) {
        delete n;
        return st;
    }
    *out = n;
    return GD_OK;
}

void gd_layernorm_destroy(gd_layernorm* n) {
    if (!n) return;
    gd::DeviceGuard guard(n->device);
    delete n;
}

gd_status gd_layernorm_forward(gd_layernorm* n, const gd_layernorm_io* io, void* stream) {
    if (!n || !io || !(io->eps >= 0.0f) || std::isinf(io->eps)) return GD_ERR_ARG;
    if (io->rows == 0) return GD_OK;
    if (!io->x || !io->weight || !io->y || io->x_stride < n->dim || io->y_stride < n->dim ||
        (io->residual && io->residual_stride < n->dim) || (io->sum && io->sum_stride < n->dim))
        return GD_ERR_ARG;
    gd::DeviceGuard guard(n->device);
    if (!guard.ok) return GD_ERR_HIP;
    const hipError_t e = gd::with_type(n->type, [&](auto zero) {
        return gd::with_shape(n->dim, false, [&](auto waves, auto v) {
            return gd::with_ends<waves(), v()>(n->dim, [&](auto ends) {
                return gd::launch_layernorm<decltype(zero), waves(), v(), ends()>(*io, n->dim, (hipStream_t)stream);
            });
        });
    });
    return e == hipSuccess ? GD_OK : GD_ERR_HIP;
}

gd_status gd_layernorm_backward(gd_layernorm* n, const gd_layernorm_grad* io, void* stream) {
    if (!n || !io || !(io->eps >= 0.0f) || std::isinf(io->eps)) return GD_ERR_ARG;
    if (io->rows && (!io->dy || !io->x || !io->weight || !io->dx || io->dy_stride < n->dim || io->x_stride < n->dim ||
                     io->dx_stride < n->dim || (io->dsum && io->dsum_stride < n->dim)))
        return GD_ERR_ARG;
    gd::DeviceGuard guard(n->device);
    if (!guard.ok) return GD_ERR_HIP;
    const hipError_t e = gd::with_type(n->type, [&](auto zero) {
        return gd::with_shape(n->dim, true, [&](auto waves, auto v) {
            return gd::with_ends<waves(), v()>(n->dim, [&](auto ends) {
                return gd::launch_layernorm_back<decltype(zero), waves(), v(), ends()>(*io, n->dim, n->part, (hipStream_t)stream);
            });
        });
    });
    return e == hipSuccess ? GD_OK : GD_ERR_HIP;
}

}  // extern "C"
