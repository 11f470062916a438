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
};
__device__ __forceinline__ RowStats row_stats(double pivot, double d, double dd, uint32_t dim, float eps) {
    const double m = d / dim, var = dd / dim - m * m;
    // a spread below the sums' rounding may come out a hair under zero; NaN stays
    return {pivot + m, (float)rsqrt((var < 0.0 ? 0.0 : var) + (double)eps)};
}

template <typename T, int WAVES, int V, bool INT8>
__global__ __launch_bounds__(NormShape<WAVES>::kThreads) void k_layernorm(gd_layernorm_io io, uint32_t dim) {
    using S = NormShape<WAVES>;
    __shared__ double lds_d[S::kThreads / kWave], lds_dd[S::kThreads / kWave];
    __shared__ uint32_t lds_max[S::kThreads / kWave];
    const uint32_t t = threadIdx.x % S::kRow;
    Pack<T, 8> w[V], b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint32_t e = min((t + i * S::kRow) * 8, dim);
        w[i] = load_some<8>((const T*)io.weight + e, (int)(dim - e));
        b[i] = Pack<T, 8>{};
        if (io.bias) b[i] = load_some<8>((const T*)io.bias + e, (int)(dim - e));
    }
    // every wave of a block takes the same number of turns (the last ones of rows past the end do nothing)
    for (uint64_t first = (uint64_t)blockIdx.x * S::kRows; first < io.rows; first += (uint64_t)gridDim.x * S::kRows) {
        const uint64_t row = first + threadIdx.x / S::kRow;
        const bool on = row < io.rows;
        float h[V][8], pivot = on ? (float)((const T*)io.x)[row * io.x_stride] : 0.0f;
        if (io.residual && on) pivot += (float)((const T*)io.residual)[row * io.residual_stride];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t e = (t + i * S::kRow) * 8;
            const int n = on ? (int)(dim - min(e, dim)) : 0;
            const Pack<T, 8> x = load_some<8>((const T*)io.x + row * io.x_stride + e, n);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[i][j] = (float)x.v[j];
            if (io.residual) {
                const Pack<T, 8> r = load_some<8>((const T*)io.residual + row * io.residual_stride + e, n);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] += (float)r.v[j];
            }
        }
        double s = 0.0, ss = 0.0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t e = (t + i * S::kRow) * 8;
            const int n = on ? (int)(dim - min(e, dim)) : 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const double d = j < n ? (double)h[i][j] - (double)pivot : 0.0;
                s += d;
                ss = fma(d, d, ss);
            }
        }
        row_sums<WAVES>(s, ss, lds_d, lds_dd);
        const RowStats st = row_stats(pivot, s, ss, dim, io.eps);
        uint32_t big = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t e = (t + i * S::kRow) * 8;
            const int n = on ? (int)(dim - min(e, dim)) : 0;
            Pack<T, 8> sum, y;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sum.v[j] = (T)h[i][j];
                h[i][j] = (float)((double)h[i][j] - st.mean) * st.rstd * (float)w[i].v[j] + (float)b[i].v[j];
                y.v[j] = (T)h[i][j];
                if (j < n) big = max(big, __float_as_uint(h[i][j]) & 0x7FFFFFFFu);
            }
            if (io.sum) store_stream<8>((T*)io.sum + row * io.sum_stride + e, sum, n);
            if (!INT8) store_stream<8>((T*)io.y + row * io.y_stride + e, y, n);
        }
        if constexpr (INT8) {
            const RowScale q = row_scale(row_max<WAVES>(big, lds_max));
            if (t == 0 && on) io.y_scale[row] = q.scale;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint32_t e = (t + i * S::kRow) * 8;
                Pack<int8_t, 8> y;
#pragma unroll
                for (int j = 0; j < 8; ++j) y.v[j] = quantise(h[i][j], q.step);
                store_some<8>((int8_t*)io.y + row * io.y_stride + e, y, on ? (int)(dim - min(e, dim)) : 0);
            }
        }
        if constexpr (WAVES > 1) __syncthreads();  // before the next row's sums
    }
}

// A block takes several rows, and loads each while it works on the one before;
// its share of the sums over rows goes to part[blockIdx.x]: dweight's, then dbias's.
template <typename T, int WAVES, int V>
__global__ __launch_bounds__(NormShape<WAVES>::kThreads) void k_layernorm_back(gd_layernorm_grad io, uint32_t dim,
                                                                               float* part) {
    using S = NormShape<WAVES>;
    __shared__ double lds_sum[2][4][S::kThreads / kWave];
    const uint32_t t = threadIdx.x % S::kRow;
    const uint64_t turn = (uint64_t)gridDim.x * S::kRows;
    struct Row {
        Pack<T, 8> x[V], dy[V], dsum[V];
        T first;
    };
    const auto here = [&](int i) { return (t + i * S::kRow) * 8; };
    const auto load = [&](Row& r, uint64_t first) {
        const uint64_t row = first + threadIdx.x / S::kRow;
        r.first = row < io.rows ? ((const T*)io.x)[row * io.x_stride] : (T)0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t e = here(i);
            const int n = row < io.rows ? (int)(dim - min(e, dim)) : 0;
            r.x[i] = load_some<8>((const T*)io.x + row * io.x_stride + e, n);
            r.dy[i] = load_some<8>((const T*)io.dy + row * io.dy_stride + e, n);
            if (io.dsum) r.dsum[i] = load_some<8>((const T*)io.dsum + row * io.dsum_stride + e, n);
        }
    };
    constexpr bool kAhead = V == 1;  // more elements a thread leave no registers for it
    Pack<T, 8> w[V];
    float dw[V][8], db[V][8];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint32_t e = min(here(i), dim);
        w[i] = load_some<8>((const T*)io.weight + e, (int)(dim - e));
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[i][j] = db[i][j] = 0.0f;
    }
    Row next;
    uint64_t first = (uint64_t)blockIdx.x * S::kRows;
    if (kAhead) load(next, first);
    for (uint32_t odd = 0; first < io.rows; first += turn, odd ^= 1) {
        const uint64_t row = first + threadIdx.x / S::kRow;
        const bool on = row < io.rows;
        if (!kAhead) load(next, first);
        const Row r = next;
        if (kAhead && first + turn < io.rows) load(next, first + turn);
        const double pivot = (float)r.first;
        double s[4] = {0.0, 0.0, 0.0, 0.0};  // of d, d^2, a, a d
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int n = on ? (int)(dim - min(here(i), dim)) : 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const double d = j < n ? (double)(float)r.x[i].v[j] - pivot : 0.0;
                const double a = (float)r.dy[i].v[j] * (float)w[i].v[j];
                s[0] += d;
                s[1] = fma(d, d, s[1]);
                s[2] += a;
                s[3] = fma(a, d, s[3]);
            }
        }
        // the two turns' sums lie apart, so one barrier a row is enough
        row_sums<WAVES>(s, lds_sum[odd]);
        const RowStats st = row_stats(pivot, s[0], s[1], dim, io.eps);
        const float mean_a = (float)(s[2] / dim);
        const float mean_ax = (float)((s[3] - s[2] * (s[0] / dim)) / dim * st.rstd);  // mean(a xhat)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t e = here(i);
            const int n = on ? (int)(dim - min(e, dim)) : 0;
            Pack<T, 8> d;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float g = (float)r.dy[i].v[j], xhat = (float)((double)(float)r.x[i].v[j] - st.mean) * st.rstd;
                dw[i][j] += n > 0 ? g * xhat : 0.0f;
                db[i][j] += g;
                float v = st.rstd * (g * (float)w[i].v[j] - mean_a - xhat * mean_ax);
                if (io.dsum) v += (float)r.dsum[i].v[j];
                d.v[j] = (T)v;
            }
            store_stream<8>((T*)io.dx + row * io.dx_stride + e, d, n);
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
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t e = min(here(i), dim);
            const int n = (int)(dim - e);
            Pack<float, 8> d;
#pragma unroll
            for (int j = 0; j < 8; ++j) d.v[j] = v[i][j];
            if (gridDim.x > 1) {
                store_some<8>(partial + e, d, n);
            } else if (out) {  // few rows: the block's share is all of it
                if (io.accumulate) {
                    const Pack<float, 8> was = load_some<8>(out + e, n);
#pragma unroll
                    for (int j = 0; j < 8; ++j) d.v[j] += was.v[j];
                }
                store_some<8>(out + e, d, n);
            }
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

template <typename T, int WAVES, int V>
hipError_t launch_layernorm(const gd_layernorm_io& io, uint32_t dim, hipStream_t st) {
    using S = NormShape<WAVES>;
    const uint32_t blocks = (uint32_t)std::min<uint64_t>((io.rows + S::kRows - 1) / S::kRows, kLayerNormMaxBlocks);
    if (io.y_scale)
        k_layernorm<T, WAVES, V, true><<<dim3(blocks), dim3(S::kThreads), 0, st>>>(io, dim);
    else
        k_layernorm<T, WAVES, V, false><<<dim3(blocks), dim3(S::kThreads), 0, st>>>(io, dim);
    return hipGetLastError();
}

template <typename T, int WAVES, int V>
hipError_t launch_layernorm_back(const gd_layernorm_grad& io, uint32_t dim, float* part, hipStream_t st) {
    using S = NormShape<WAVES>;
    const bool sums = io.dweight || io.dbias;
    const uint32_t most = std::min(kLayerNormBackWaves * kWave / S::kThreads, kLayerNormParts);
    const uint64_t turns = (io.rows + S::kRows - 1) / S::kRows;
    // few rows go to one block, which writes the gradients itself
    const bool one = turns <= 4 && turns * dim <= 1u << 14;
    const uint32_t parts = one ? (turns != 0) : (uint32_t)std::min<uint64_t>(turns, most);
    if (parts) {
        k_layernorm_back<T, WAVES, V><<<dim3(parts), dim3(S::kThreads), 0, st>>>(io, dim, sums ? part : nullptr);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!sums || parts == 1 || (!parts && io.accumulate)) return hipSuccess;
    k_layernorm_join<<<dim3((2 * dim + kJoinColumns - 1) / kJoinColumns), dim3(kJoinColumns * kJoinGroups), 0, st>>>(
        part, parts, dim, io.dweight, io.dbias, io.accumulate != 0);
    return hipGetLastError();
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
            return gd::launch_layernorm<decltype(zero), waves(), v()>(*io, n->dim, (hipStream_t)stream);
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
            return gd::launch_layernorm_back<decltype(zero), waves(), v()>(*io, n->dim, n->part, (hipStream_t)stream);
        });
    });
    return e == hipSuccess ? GD_OK : GD_ERR_HIP;
}

}  // extern "C"
