// Linear layers: argument checks, the gradient at the activation's input, and
// the sequence of products of the forward and backward calls.

#include <cmath>
#include <new>

#include "gd_gemm.hpp"
#include "gd_host.hpp"

namespace gd {

// dz = dy act'(pre), rounded, and its sums over the block's rows.  A wave takes
// 512 columns of a row at a time, a lane 8; the block's waves take rows in
// turn.  Bound by memory: 6 bytes an element in 16 bits.
constexpr int kSlopeColumns = kWave * 8;
// The sums of few rows, one block's of sixteen waves, go out at once.
template <typename T, int WAVES>
__global__ __launch_bounds__(WAVES* kWave) void k_slope(gd_linear_grad io, uint32_t columns, int act, float* part) {
    __shared__ float lds[WAVES][kSlopeColumns];
    const uint32_t c = blockIdx.x * kSlopeColumns + lane_id() * 8;
    const int n = (int)(columns - min(c, columns));
    float sum[8] = {};
    for (uint64_t row = (uint64_t)blockIdx.y * WAVES + wave_index(); row < io.rows; row += (uint64_t)gridDim.y * WAVES) {
        Pack<T, 8> d = load_some<8>((const T*)io.dy + row * io.dy_stride + c, n);
        if (act != GD_ACT_NONE) {
            const Pack<T, 8> z = load_some<8>((const T*)io.pre + row * io.pre_stride + c, n);
            float at[8], v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) at[j] = (float)z.v[j], v[j] = (float)d.v[j];
            act_slope<sizeof(T) == 4>(act, at, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) d.v[j] = (T)v[j];
            store_some<8>((T*)io.dz + row * io.dz_stride + c, d, n);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += (float)d.v[j];
    }
    if (!io.dbias) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) lds[wave_index()][lane_id() * 8 + j] = sum[j];
    __syncthreads();
    for (uint32_t j = threadIdx.x; j < (uint32_t)kSlopeColumns; j += WAVES * kWave) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) s += lds[w][j];
        const uint32_t col = blockIdx.x * kSlopeColumns + j;
        if (col >= columns) continue;
        if (gridDim.y == 1)
            io.dbias[col] = io.accumulate ? io.dbias[col] + s : s;
        else
            part[(uint64_t)blockIdx.y * columns + col] = s;
    }
}

hipError_t launch_slope(const gd_linear_grad& io, int type, uint32_t columns, int act, float* part, hipStream_t st) {
    // one block down the rows up to 64 of them: a second launch costs more than the four turns of its waves
    const uint32_t groups = io.rows <= 64 ? (io.rows != 0) : (uint32_t)std::min<uint64_t>((io.rows + 15) / 16, kBiasParts);
    if (groups) {
        const dim3 grid((columns + kSlopeColumns - 1) / kSlopeColumns, groups);
        const auto run = [&](auto zero) {
            using T = decltype(zero);
            if (groups == 1)
                k_slope<T, 16><<<grid, dim3(16 * kWave), 0, st>>>(io, columns, act, part);
            else
                k_slope<T, 4><<<grid, dim3(4 * kWave), 0, st>>>(io, columns, act, part);
        };
        if (type == GD_F32)
            run(0.0f);
        else if (type == GD_BF16)
            run((bf16)0.0f);
        else
            run((f16)0.0f);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!io.dbias || groups == 1 || (!groups && io.accumulate)) return hipSuccess;
    return launch_sum_parts(part, groups, columns, io.dbias, io.accumulate != 0, st);
}

template <typename T>
hipError_t forward(const GemmArgs& a, const GemmRoom& room, bool int8, hipStream_t st) {
    return int8 ? launch_gemm<int8_t, T, kAlong>(a, room, st) : launch_gemm<T, T, kAlong>(a, room, st);
}

}  // namespace gd

struct gd_linear {
    int device = 0;
    uint32_t in = 0, out = 0;
    int type = GD_F32, act = GD_ACT_NONE;
    uint64_t max_rows = 0;
    float* room = nullptr;  // [kLinearRoom]
    float* part = nullptr;  // [kBiasParts * out]
    char* pad = nullptr;    // padded copies of operands, where in or out is no whole number of 16-byte chunks
    uint64_t pad_bytes = 0;
    gd::DeviceMemory mem;
};

extern "C" {

gd_status gd_linear_create(gd_linear** out, uint32_t in, uint32_t out_features, gd_dtype type, gd_act act,
                           uint64_t max_rows) {
    if (!out) return GD_ERR_ARG;
    *out = nullptr;
    const int ty = gd::enum_int(&type), ac = gd::enum_int(&act);
    if (in == 0 || out_features == 0 || in > gd::kLinearMaxDim || out_features > gd::kLinearMaxDim ||
        max_rows > 0x7FFFFFFFull || ty < GD_F32 || ty > GD_F16 || ac < GD_ACT_NONE || ac > GD_ACT_SILU)
        return GD_ERR_ARG;
    gd_linear* l = new (std::nothrow) gd_linear();
    if (!l) return GD_ERR_OOM;
    l->in = in;
    l->out = out_features;
    l->type = ty;
    l->act = ac;
    l->max_rows = max_rows;
    if (ty != GD_F32 && (in % 8 || out_features % 8)) {
        // the two operands of the forward call, of the input's gradient or of the weight's
        const uint64_t k = (in + 7ull) / 8 * 16, n = (out_features + 7ull) / 8 * 16, w = out_features * k;
        l->pad_bytes = std::min(std::max({max_rows * k + w, max_rows * n + w, max_rows * (k + n)}), gd::kLinearPad);
    }
    gd_status st = GD_OK;
    try {
        if (hipGetDevice(&l->device) != hipSuccess) st = GD_ERR_HIP;
        else if (!l->mem.alloc(&l->room, gd::kLinearRoom) ||
                 !l->mem.alloc(&l->part, (size_t)gd::kBiasParts * out_features) ||
                 (l->pad_bytes && !l->mem.alloc(&l->pad, l->pad_bytes)))
            st = GD_ERR_OOM;
    } catch (const std::bad_alloc&) {
        st = GD_ERR_OOM;
    }
    if (st != GD_OK) {
        delete l;
        return st;
    }
    *out = l;
    return GD_OK;
}

void gd_linear_destroy(gd_linear* l) {
    if (!l) return;
    gd::DeviceGuard guard(l->device);
    delete l;
}

gd_status gd_linear_forward(gd_linear* l, const gd_linear_io* io, void* stream) {
    // no rows have no scales, and an empty buffer may have no address
    if (!l || !io || io->rows > l->max_rows || (io->rows && (io->x_scale == nullptr) != (io->weight_scale == nullptr)))
        return GD_ERR_ARG;
    const auto bad = [](uint64_t stride, uint64_t least) { return stride < least || stride > gd::kLinearMaxDim; };
    if (bad(io->weight_stride, l->in) || (io->rows && (bad(io->x_stride, l->in) || bad(io->y_stride, l->out))) ||
        (io->residual && bad(io->residual_stride, l->out)) || (io->pre && bad(io->pre_stride, l->out)))
        return GD_ERR_ARG;
    const bool int8 = io->x_scale != nullptr;
    if ((int8 && l->in > gd::kLinearMaxInt8) || !gd::product_fits(l->out, io->rows)) return GD_ERR_LAYOUT;
    if (io->rows == 0) return GD_OK;
    if (!io->x || !io->weight || !io->y) return GD_ERR_ARG;
    gd::DeviceGuard guard(l->device);
    if (!guard.ok) return GD_ERR_HIP;
    gd::GemmArgs a{};
    a.p = io->weight;
    a.q = io->x;
    a.p_stride = io->weight_stride;
    a.q_stride = io->x_stride;
    a.I = l->out;
    a.J = (uint32_t)io->rows;
    a.K = l->in;
    a.part = l->room;
    a.fin.out = io->y;
    a.fin.out_stride = io->y_stride;
    a.fin.bias = io->bias;
    a.fin.residual = io->residual;
    a.fin.residual_stride = io->residual_stride;
    a.fin.pre = io->pre;
    a.fin.pre_stride = io->pre_stride;
    a.fin.p_scale = io->weight_scale;
    a.fin.q_scale = io->x_scale;
    a.fin.act = l->act;
    const hipStream_t st = (hipStream_t)stream;
    const gd::GemmRoom room{gd::kLinearRoom, l->pad, l->pad_bytes};
    const hipError_t e = l->type == GD_F32    ? gd::forward<float>(a, room, int8, st)
                         : l->type == GD_BF16 ? gd::forward<gd::bf16>(a, room, int8, st)
                                              : gd::forward<gd::f16>(a, room, int8, st);
    return e == hipSuccess ? GD_OK : GD_ERR_HIP;
}

gd_status gd_linear_backward(gd_linear* l, const gd_linear_grad* io, void* stream) {
    if (!l || !io || io->rows > l->max_rows) return GD_ERR_ARG;
    const auto bad = [](uint64_t stride, uint64_t least) { return stride < least || stride > gd::kLinearMaxDim; };
    const bool act = l->act != GD_ACT_NONE, rows = io->rows != 0;
    if ((rows && (!io->dy || bad(io->dy_stride, l->out))) ||
        (rows && act && (!io->pre || !io->dz || bad(io->pre_stride, l->out) || bad(io->dz_stride, l->out))) ||
        (rows && io->dx && (!io->weight || bad(io->weight_stride, l->in) || bad(io->dx_stride, l->in))) ||
        (io->dweight && (bad(io->dweight_stride, l->in) || (rows && (!io->x || bad(io->x_stride, l->in))))))
        return GD_ERR_ARG;
    if ((io->dx && !gd::product_fits(l->in, io->rows)) || (io->dweight && !gd::product_fits(l->in, l->out)))
        return GD_ERR_LAYOUT;
    gd::DeviceGuard guard(l->device);
    if (!guard.ok) return GD_ERR_HIP;
    const hipStream_t st = (hipStream_t)stream;
    if (act || io->dbias)
        if (gd::launch_slope(*io, l->type, l->out, l->act, l->part, st) != hipSuccess) return GD_ERR_HIP;
    const void* dz = act ? io->dz : io->dy;
    const uint64_t dz_stride = act ? io->dz_stride : io->dy_stride;
    gd::GemmArgs dx{}, dw{};
    dx.p = io->weight;
    dx.q = dz;
    dx.p_stride = io->weight_stride;
    dx.q_stride = dz_stride;
    dx.I = l->in;
    dx.J = (uint32_t)io->rows;
    dx.K = l->out;
    dx.part = l->room;
    dx.fin.out = io->dx;
    dx.fin.out_stride = io->dx_stride;
    dw.p = io->x;
    dw.q = dz;
    dw.p_stride = io->x_stride;
    dw.q_stride = dz_stride;
    dw.I = l->in;
    dw.J = l->out;
    dw.K = (uint32_t)io->rows;
    dw.part = l->room;
    dw.fin.out = io->dweight;
    dw.fin.out_stride = io->dweight_stride;
    if (io->accumulate) {
        dw.fin.residual = io->dweight;
        dw.fin.residual_stride = io->dweight_stride;
    }
    const gd::GemmArgs *want_dx = rows && io->dx ? &dx : nullptr,
                       *want_dw = io->dweight && (rows || !io->accumulate) ? &dw : nullptr;
    const gd::GemmRoom room{gd::kLinearRoom, l->pad, l->pad_bytes};
    const hipError_t e = l->type == GD_F32    ? gd::launch_backward<float>(want_dx, want_dw, room, st)
                         : l->type == GD_BF16 ? gd::launch_backward<gd::bf16>(want_dx, want_dw, room, st)
                                              : gd::launch_backward<gd::f16>(want_dx, want_dw, room, st);
    return e == hipSuccess ? GD_OK : GD_ERR_HIP;
}

}  // extern "C"
