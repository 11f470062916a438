// Root-mean-square norm of rows with the residual's addition, forward (output
// in the type or in 8 bits with a scale per row) and backward.
//
// Both directions are bound by memory: a row is read once, held in registers
// between its sums and its output, and written once, past the caches' reuse
// (8192 x 4096 in bfloat16 forward: 47 us so, 5.7 TB/s, and 50 us with
// ordinary stores).  Sums over a row are in 64 bits: the norm's factor then
// comes out the same whatever the split, at one 64-bit multiply-add per
// element, which the memory's time hides.  The backward pass, 70 us at that
// size, 3.8 TB/s, is bound by the chain of a row's loads, its two sums over
// eight waves and its output, in what waves its registers leave room for.

#include <cmath>
#include <new>

#include "gd.h"
#include "gd_host.hpp"
#include "gd_ops.hpp"

namespace gd {

constexpr uint32_t kNormMaxDim = 32768;
constexpr uint32_t kNormParts = 1024;       // partial sums of the weight's gradient, at most
constexpr uint32_t kNormBackWaves = 4096;   // waves of the backward pass: four a SIMD, as many as its registers hold
constexpr uint32_t kNormMaxBlocks = 1u << 20;  // a dispatch holds less than 2^32 threads

template <int WAVES>
struct NormShape {
    static constexpr int kThreads = WAVES * kWave < kBlock ? kBlock : WAVES * kWave;
    static constexpr int kRow = WAVES * kWave;          // threads of a row
    static constexpr int kRows = kThreads / kRow;       // rows of a block
};

template <typename T, int WAVES, int V, bool INT8>
__global__ __launch_bounds__(NormShape<WAVES>::kThreads) void k_norm(gd_norm_io io, uint32_t dim) {
    using S = NormShape<WAVES>;
    __shared__ double lds_sum[S::kThreads / kWave];
    __shared__ uint32_t lds_max[S::kThreads / kWave];
    const uint32_t t = threadIdx.x % S::kRow;
    Pack<T, 8> w[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint32_t e = (t + i * S::kRow) * 8;
        w[i] = load_some<8>((const T*)io.weight + min(e, dim), (int)(dim - min(e, dim)));
    }
    // every wave of a block takes the same number of turns (the last ones of rows past the end do nothing)
    for (uint64_t first = (uint64_t)blockIdx.x * S::kRows; first < io.rows; first += (uint64_t)gridDim.x * S::kRows) {
        const uint64_t row = first + threadIdx.x / S::kRow;
        const bool on = row < io.rows;
        float h[V][8];
        double ss = 0.0;
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
#pragma unroll
            for (int j = 0; j < 8; ++j) ss = fma((double)h[i][j], (double)h[i][j], ss);
        }
        ss = row_sum<WAVES>(ss, lds_sum);
        const float rstd = (float)rsqrt(ss / dim + (double)io.eps);
        uint32_t big = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t e = (t + i * S::kRow) * 8;
            const int n = on ? (int)(dim - min(e, dim)) : 0;
            Pack<T, 8> s, y;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s.v[j] = (T)h[i][j];
                h[i][j] = h[i][j] * rstd * (float)w[i].v[j];
                y.v[j] = (T)h[i][j];
                if (j < n) big = max(big, __float_as_uint(h[i][j]) & 0x7FFFFFFFu);
            }
            if (io.sum) store_stream<8>((T*)io.sum + row * io.sum_stride + e, s, n);
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

// dx = rstd (a - xhat mean(a xhat)) + dsum with a = dy weight, xhat = x rstd;
// the block's share of sum_rows dy xhat goes to part[blockIdx.x].  A block
// takes several rows, and loads each while it works on the one before.
template <typename T, int WAVES, int V>
__global__ __launch_bounds__(NormShape<WAVES>::kThreads) void k_norm_back(gd_norm_grad io, uint32_t dim, float* part) {
    using S = NormShape<WAVES>;
    __shared__ double lds_sum[2][2][S::kThreads / kWave];
    const uint32_t t = threadIdx.x % S::kRow;
    const uint64_t turn = (uint64_t)gridDim.x * S::kRows;
    struct Row {
        Pack<T, 8> x[V], dy[V], dsum[V];
    };
    const auto here = [&](int i) { return (t + i * S::kRow) * 8; };
    const auto load = [&](Row& r, uint64_t first) {
        const uint64_t row = first + threadIdx.x / S::kRow;
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
    float dw[V][8];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint32_t e = here(i);
        w[i] = load_some<8>((const T*)io.weight + min(e, dim), (int)(dim - min(e, dim)));
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[i][j] = 0.0f;
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
        double ss = 0.0, ax = 0.0;
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float xv = (float)r.x[i].v[j];
                ss = fma((double)xv, (double)xv, ss);
                ax = fma((double)((float)r.dy[i].v[j] * (float)w[i].v[j]), (double)xv, ax);
            }
        // the two turns' sums lie apart, so one barrier a row is enough
        row_sums<WAVES>(ss, ax, lds_sum[odd][0], lds_sum[odd][1]);
        const float rstd = (float)rsqrt(ss / dim + (double)io.eps);
        const float mean = (float)(ax / dim * rstd);  // mean(a xhat)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t e = here(i);
            const int n = on ? (int)(dim - min(e, dim)) : 0;
            Pack<T, 8> d;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float g = (float)r.dy[i].v[j], xhat = (float)r.x[i].v[j] * rstd;
                dw[i][j] += n > 0 ? g * xhat : 0.0f;
                float v = rstd * (g * (float)w[i].v[j] - xhat * mean);
                if (io.dsum) v += (float)r.dsum[i].v[j];
                d.v[j] = (T)v;
            }
            store_stream<8>((T*)io.dx + row * io.dx_stride + e, d, n);
        }
    }
    if (!part) return;
    if constexpr (S::kRows > 1) {  // the block's rows join before the partial is written
        __shared__ float lds_dw[S::kRows][V * 8 * S::kRow];
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) lds_dw[threadIdx.x / S::kRow][(i * 8 + j) * S::kRow + t] = dw[i][j];
        __syncthreads();
        if (threadIdx.x >= (uint32_t)S::kRow) return;
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int r = 1; r < S::kRows; ++r) dw[i][j] += lds_dw[r][(i * 8 + j) * S::kRow + t];
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint32_t e = (t + i * S::kRow) * 8;
        Pack<float, 8> d;
#pragma unroll
        for (int j = 0; j < 8; ++j) d.v[j] = dw[i][j];
        const int n = (int)(dim - min(e, dim));
        if (gridDim.x == 1) {  // few rows: the block's share is all of it
            if (io.accumulate) {
                const Pack<float, 8> was = load_some<8>(io.dweight + min(e, dim), n);
#pragma unroll
                for (int j = 0; j < 8; ++j) d.v[j] += was.v[j];
            }
            store_some<8>(io.dweight + min(e, dim), d, n);
        } else {
            store_some<8>(part + (uint64_t)blockIdx.x * dim + min(e, dim), d, n);
        }
    }
}

// 32 columns by 32 groups of partials a block: a wave reads two 128-byte runs at a time.
constexpr int kSumColumns = 32, kSumGroups = 32;
__global__ __launch_bounds__(kSumColumns* kSumGroups) void k_sum_parts(const float* part, uint32_t parts,
                                                                       uint64_t columns, float* out, bool accumulate) {
    __shared__ double lds[kSumGroups][kSumColumns];
    const uint32_t c = threadIdx.x % kSumColumns, g = threadIdx.x / kSumColumns;
    for (uint64_t first = (uint64_t)blockIdx.x * kSumColumns; first < columns;
         first += (uint64_t)gridDim.x * kSumColumns) {
        double s = 0.0;
        if (first + c < columns)
#pragma unroll 8
            for (uint32_t p = g; p < parts; p += kSumGroups) s += part[p * columns + first + c];
        lds[g][c] = s;
        __syncthreads();
        if (g == 0 && first + c < columns) {
            s = accumulate ? (double)out[first + c] : 0.0;
#pragma unroll
            for (int i = 0; i < kSumGroups; ++i) s += lds[i][c];
            out[first + c] = (float)s;
        }
        __syncthreads();
    }
}

hipError_t launch_sum_parts(const float* part, uint32_t parts, uint64_t columns, float* out, bool accumulate,
                            hipStream_t st) {
    const uint64_t blocks = std::min<uint64_t>((columns + kSumColumns - 1) / kSumColumns, 1u << 20);
    k_sum_parts<<<dim3((uint32_t)blocks), dim3(kSumColumns * kSumGroups), 0, st>>>(part, parts, columns, out, accumulate);
    return hipGetLastError();
}

template <typename T, int WAVES, int V>
hipError_t launch_norm(const gd_norm_io& io, uint32_t dim, hipStream_t st) {
    using S = NormShape<WAVES>;
    const uint32_t blocks = (uint32_t)std::min<uint64_t>((io.rows + S::kRows - 1) / S::kRows, kNormMaxBlocks);
    if (io.y_scale)
        k_norm<T, WAVES, V, true><<<dim3(blocks), dim3(S::kThreads), 0, st>>>(io, dim);
    else
        k_norm<T, WAVES, V, false><<<dim3(blocks), dim3(S::kThreads), 0, st>>>(io, dim);
    return hipGetLastError();
}

template <typename T, int WAVES, int V>
hipError_t launch_norm_back(const gd_norm_grad& io, uint32_t dim, float* part, hipStream_t st) {
    using S = NormShape<WAVES>;
    const uint32_t most = std::min(kNormBackWaves * kWave / S::kThreads, kNormParts);
    const uint64_t turns = (io.rows + S::kRows - 1) / S::kRows;
    // few rows go to one block, which writes the weight's gradient itself: 8 x 500 take 8.2 us, with the second launch
    // 11.2; 4 x 8192 would take 12.1, with it 11.5
    const bool one = turns <= 4 && turns * dim <= 1u << 14;
    const uint32_t parts = one ? (turns != 0) : (uint32_t)std::min<uint64_t>(turns, most);
    if (parts) {
        k_norm_back<T, WAVES, V><<<dim3(parts), dim3(S::kThreads), 0, st>>>(io, dim, io.dweight ? part : nullptr);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!io.dweight || parts == 1 || (!parts && io.accumulate)) return hipSuccess;
    return launch_sum_parts(part, parts, dim, io.dweight, io.accumulate != 0, st);
}

// Rows in 8 bits: the form of k_norm without the norm.
template <typename T, int WAVES, int V>
__global__ __launch_bounds__(NormShape<WAVES>::kThreads) void k_quantise(const T* x, uint64_t rows, uint32_t columns,
                                                                         uint64_t x_stride, int8_t* q,
                                                                         uint64_t q_stride, float* scale) {
    using S = NormShape<WAVES>;
    __shared__ uint32_t lds_max[S::kThreads / kWave];
    const uint32_t t = threadIdx.x % S::kRow;
    for (uint64_t first = (uint64_t)blockIdx.x * S::kRows; first < rows; first += (uint64_t)gridDim.x * S::kRows) {
        const uint64_t row = first + threadIdx.x / S::kRow;
        Pack<T, 8> v[V];
        uint32_t big = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t e = (t + i * S::kRow) * 8;
            v[i] = load_some<8>(x + row * x_stride + e, row < rows ? (int)(columns - min(e, columns)) : 0);
        }
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) big = max(big, __float_as_uint((float)v[i].v[j]) & 0x7FFFFFFFu);
        // a row longer than the registers hold is read again below
        for (uint32_t e = (t + V * S::kRow) * 8; row < rows && e < columns; e += S::kRow * 8) {
            const Pack<T, 8> m = load_some<8>(x + row * x_stride + e, (int)(columns - e));
#pragma unroll
            for (int j = 0; j < 8; ++j) big = max(big, __float_as_uint((float)m.v[j]) & 0x7FFFFFFFu);
        }
        const RowScale s = row_scale(row_max<WAVES>(big, lds_max));
        if (t == 0 && row < rows) scale[row] = s.scale;
        for (uint32_t i = 0; row < rows && (t + i * S::kRow) * 8 < columns; ++i) {
            const uint32_t e = (t + i * S::kRow) * 8;
            Pack<T, 8> m;
            if (i >= (uint32_t)V) m = load_some<8>(x + row * x_stride + e, (int)(columns - e));
#pragma unroll
            for (int c = 0; c < V; ++c)
                if (i == (uint32_t)c) m = v[c];
            Pack<int8_t, 8> y;
#pragma unroll
            for (int j = 0; j < 8; ++j) y.v[j] = quantise((float)m.v[j], s.step);
            store_some<8>(q + row * q_stride + e, y, (int)(columns - e));
        }
        if constexpr (WAVES > 1) __syncthreads();  // before the next row's maximum
    }
}

template <typename T, int WAVES, int V>
hipError_t launch_quantise(const void* x, uint64_t rows, uint32_t columns, uint64_t x_stride, int8_t* q,
                           uint64_t q_stride, float* scale, hipStream_t st) {
    using S = NormShape<WAVES>;
    const uint32_t blocks = (uint32_t)std::min<uint64_t>((rows + S::kRows - 1) / S::kRows, kNormMaxBlocks);
    k_quantise<T, WAVES, V><<<dim3(blocks), dim3(S::kThreads), 0, st>>>((const T*)x, rows, columns, x_stride, q, q_stride, scale);
    return hipGetLastError();
}

// Calls f with the waves of a row and the 8-element vectors of a thread as
// constants.  One vector a thread does best (8192 x 4096 in bfloat16 forward:
// 50 us with eight waves a row, 63 with four, 91 with one; 8192 x 1024: 13 us
// with two, 16 with one), up to blocks of 512 threads, whose barriers cost
// less than those of 1,024 (4096 x 8192: 57 and 60 us; backward, where a
// thread holds more, 97 and 77).
template <typename F>
hipError_t with_shape(uint32_t dim, bool back, F f) {
    if (dim <= 512) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
    if (dim <= 1024) return f(std::integral_constant<int, 2>(), std::integral_constant<int, 1>());
    if (dim <= 2048) return f(std::integral_constant<int, 4>(), std::integral_constant<int, 1>());
    if (dim <= 4096) return f(std::integral_constant<int, 8>(), std::integral_constant<int, 1>());
    if (dim <= 8192 && !back) return f(std::integral_constant<int, 8>(), std::integral_constant<int, 2>());
    if (dim <= 8192) return f(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
    if (dim <= 16384) return f(std::integral_constant<int, 16>(), std::integral_constant<int, 2>());
    return f(std::integral_constant<int, 16>(), std::integral_constant<int, 4>());
}

// Calls f with a zero of the element type.
template <typename F>
hipError_t with_type(int type, F f) {
    return type == GD_F32 ? f(0.0f) : type == GD_BF16 ? f((bf16)0.0f) : f((f16)0.0f);
}

}  // namespace gd

struct gd_norm {
    int device = 0;
    uint32_t dim = 0;
    int type = GD_F32;
    float* part = nullptr;  // [kNormParts * dim]
    gd::DeviceMemory mem;
};

extern "C" {

gd_status gd_norm_create(gd_norm** out, uint32_t dim, gd_dtype type) {
    if (!out) return GD_ERR_ARG;
    *out = nullptr;
    const int ty = gd::enum_int(&type);
    if (dim == 0 || dim > gd::kNormMaxDim || ty < GD_F32 || ty > GD_F16) return GD_ERR_ARG;
    gd_norm* n = new (std::nothrow) gd_norm();
    if (!n) return GD_ERR_OOM;
    n->dim = dim;
    n->type = ty;
    gd_status st = GD_OK;
    try {
        if (hipGetDevice(&n->device) != hipSuccess) st = GD_ERR_HIP;
        else if (!n->mem.alloc(&n->part, (size_t)gd::kNormParts * dim)) st = GD_ERR_OOM;
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

void gd_norm_destroy(gd_norm* n) {
    if (!n) return;
    gd::DeviceGuard guard(n->device);
    delete n;
}

gd_status gd_norm_forward(gd_norm* n, const gd_norm_io* io, void* stream) {
    if (!n || !io || !(io->eps >= 0.0f) || std::isinf(io->eps)) return GD_ERR_ARG;
    if (io->rows == 0) return GD_OK;
    if (!io->x || !io->weight || !io->y || io->x_stride < n->dim || io->y_stride < n->dim ||
        (io->residual && io->residual_stride < n->dim) || (io->sum && io->sum_stride < n->dim))
        return GD_ERR_ARG;
    gd::DeviceGuard guard(n->device);
    if (!guard.ok) return GD_ERR_HIP;
    const hipError_t e = gd::with_type(n->type, [&](auto zero) {
        return gd::with_shape(n->dim, false, [&](auto waves, auto v) {
            return gd::launch_norm<decltype(zero), waves(), v()>(*io, n->dim, (hipStream_t)stream);
        });
    });
    return e == hipSuccess ? GD_OK : GD_ERR_HIP;
}

gd_status gd_norm_backward(gd_norm* n, const gd_norm_grad* io, void* stream) {
    if (!n || !io || !(io->eps >= 0.0f) || std::isinf(io->eps)) return GD_ERR_ARG;
    if (io->rows && (!io->dy || !io->x || !io->weight || !io->dx || io->dy_stride < n->dim || io->x_stride < n->dim ||
                     io->dx_stride < n->dim || (io->dsum && io->dsum_stride < n->dim)))
        return GD_ERR_ARG;
    gd::DeviceGuard guard(n->device);
    if (!guard.ok) return GD_ERR_HIP;
    const hipError_t e = gd::with_type(n->type, [&](auto zero) {
        return gd::with_shape(n->dim, true, [&](auto waves, auto v) {
            return gd::launch_norm_back<decltype(zero), waves(), v()>(*io, n->dim, n->part, (hipStream_t)stream);
        });
    });
    return e == hipSuccess ? GD_OK : GD_ERR_HIP;
}

gd_status gd_quantise_rows(const void* x, gd_dtype type, uint64_t rows, uint64_t columns, uint64_t x_stride, int8_t* q,
                           uint64_t q_stride, float* scale, void* stream) {
    const int ty = gd::enum_int(&type);
    if (ty < GD_F32 || ty > GD_F16 || columns == 0 || columns > 0x7FFFFFFFull) return GD_ERR_ARG;
    if (rows == 0) return GD_OK;
    if (!x || !q || !scale || x_stride < columns || q_stride < columns) return GD_ERR_ARG;
    const hipError_t e = gd::with_type(ty, [&](auto zero) {
        return gd::with_shape((uint32_t)columns, false, [&](auto waves, auto v) {
            return gd::launch_quantise<decltype(zero), waves(), v()>(x, rows, (uint32_t)columns, x_stride, q, q_stride,
                                                                     scale, (hipStream_t)stream);
        });
    });
    return e == hipSuccess ? GD_OK : GD_ERR_HIP;
}

}  // extern "C"
