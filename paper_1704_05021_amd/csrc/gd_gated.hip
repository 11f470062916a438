// Gated layers: y = act(x Wg^T + bg) * (x Wu^T + bu), the first half of a gated
// feed-forward block, and its backward.
//
// The weight holds Wg's rows and then Wu's.  Forward is one product with both:
// each tile takes the two rows of its results, so that the activation and the
// product of the two sums are its epilogue, and neither sum goes to memory
// unless it is kept for the backward (gd_gemm.hpp, PAIR).  Backward,
//   dzg = dy u act'(g),  dzu = dy act(g)
// are written side by side, as one matrix of twice the width: what is left are
// the two products of a linear layer of that width.

#include <cmath>
#include <new>

#include "gd_gemm.hpp"
#include "gd_host.hpp"

namespace gd {

// dz, rounded, and its sums over the block's rows.  A wave takes 512 results of
// a row at a time, a lane 8; the block's waves take rows in turn.  Bound by
// memory: 10 bytes a result in 16 bits.  The library's exponential and erf in
// 16 bits too, unlike a product's epilogue: the weight's gradient is in 32 bits,
// and every dz that rounds the other way than the formula's shows in it (SiLU
// of 4096 x 8192 by the hardware's exponential: 1.4e-5 of dz, with these 1e-6).
// g of the gate and u times the gradient in, act(g) and that times act'(g) out: what both take of g is formed once.
template <int N>
__device__ __forceinline__ void gate_slopes(int act, const float (&g)[N], float (&a)[N], float (&dg)[N]) {
    if (act == GD_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float e = 1.0f + expf(-g[j]), q = 1.0f / e;
            a[j] = g[j] / e;
            dg[j] *= q * (1.0f + g[j] * (1.0f - q));
        }
        return;
    }
    if (act == GD_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float e;
            const float cdf = normal<true>(g[j], e);
            a[j] = g[j] * cdf;
            dg[j] *= cdf + g[j] * (e * 0.39894228040143268f);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) a[j] = g[j];
    act_slope<true>(act, g, dg);
    activate<true>(act, a);
}

constexpr int kGatedColumns = kWave * 8;
template <typename T, int WAVES, bool WHOLE>  // WHOLE: rows are whole vectors, and every load is made
__global__ __launch_bounds__(WAVES* kWave) void k_gated_slope(gd_gated_grad io, uint32_t out, int act, float* part) {
    __shared__ float lds[WAVES][kGatedColumns];
    const uint32_t c0 = blockIdx.x * kGatedColumns + (uint32_t)lane_id() * 8;
    const uint32_t c = min(c0, WHOLE ? out - 8 : out);
    const int n = (int)(out - c);
    const auto load = [&](const void* p, uint64_t at) {
        if constexpr (WHOLE) return load_pack<8>((const T*)p + at);
        return load_some<8>((const T*)p + at, n);
    };
    float sum_g[8] = {}, sum_u[8] = {};
    for (uint64_t row = (uint64_t)blockIdx.y * WAVES + wave_index(); row < io.rows; row += (uint64_t)gridDim.y * WAVES) {
        const Pack<T, 8> dy = load(io.dy, row * io.dy_stride + c), gate = load(io.pre, row * io.pre_stride + c),
                         up = load(io.pre, row * io.pre_stride + out + c);
        float g[8], a[8], dg[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = (float)gate.v[j], dg[j] = (float)dy.v[j] * (float)up.v[j];
        gate_slopes(act, g, a, dg);
        Pack<T, 8> zg, zu;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            zg.v[j] = (T)dg[j];
            // a unit that ReLU turns off passes nothing, a gradient that is not finite neither; NaN is not turned off
            zu.v[j] = (T)(act == GD_ACT_RELU && g[j] <= 0.0f ? 0.0f : (float)dy.v[j] * a[j]);
            sum_g[j] += (float)zg.v[j];
            sum_u[j] += (float)zu.v[j];
        }
        if (WHOLE && c0 >= out) continue;
        T* dz = (T*)io.dz + row * io.dz_stride + c;
        store_some<8>(dz, zg, WHOLE ? 8 : n);
        store_some<8>(dz + out, zu, WHOLE ? 8 : n);
    }
    if (!io.dbias) return;
    const auto join = [&](const float (&sum)[8], uint32_t first) {
#pragma unroll
        for (int j = 0; j < 8; ++j) lds[wave_index()][lane_id() * 8 + j] = sum[j];
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < (uint32_t)kGatedColumns; j += WAVES * kWave) {
            float s = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) s += lds[w][j];
            const uint32_t col = blockIdx.x * kGatedColumns + j;
            if (col >= out) continue;
            if (gridDim.y == 1)
                io.dbias[first + col] = io.accumulate ? io.dbias[first + col] + s : s;
            else
                part[(uint64_t)blockIdx.y * 2 * out + first + col] = s;
        }
        __syncthreads();
    };
    join(sum_g, 0);
    join(sum_u, out);
}

hipError_t launch_gated_slope(const gd_gated_grad& io, int type, uint32_t out, int act, float* part, hipStream_t st) {
    // one block down the rows up to 64 of them: a second launch costs more than the four turns of its waves
    const uint32_t groups = io.rows <= 64 ? (io.rows != 0) : (uint32_t)std::min<uint64_t>((io.rows + 15) / 16, kBiasParts);
    if (groups) {
        const dim3 grid((out + kGatedColumns - 1) / kGatedColumns, groups);
        const auto run = [&](auto zero) {
            using T = decltype(zero);
            const auto with_waves = [&](auto waves) {
                if (out % 8)
                    k_gated_slope<T, waves(), false><<<grid, dim3(waves() * kWave), 0, st>>>(io, out, act, part);
                else
                    k_gated_slope<T, waves(), true><<<grid, dim3(waves() * kWave), 0, st>>>(io, out, act, part);
            };
            if (groups == 1)
                with_waves(std::integral_constant<int, 16>());
            else
                with_waves(std::integral_constant<int, 4>());
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
    return launch_sum_parts(part, groups, 2ull * out, io.dbias, io.accumulate != 0, st);
}

template <typename T>
hipError_t gated_forward(const GemmArgs& a, const GemmRoom& room, bool int8, hipStream_t st) {
    return int8 ? launch_gated<int8_t, T>(a, room, st) : launch_gated<T, T>(a, room, st);
}

}  // namespace gd

struct gd_gated {
    int device = 0;
    uint32_t in = 0, out = 0;
    int type = GD_F32, act = GD_ACT_NONE;
    uint64_t max_rows = 0;
    float* room = nullptr;  // [kLinearRoom]
    float* part = nullptr;  // [kBiasParts][2 out]
    char* pad = nullptr;    // padded copies of operands, where in or out is no whole number of 16-byte chunks
    uint64_t pad_bytes = 0;
    gd::DeviceMemory mem;
};

extern "C" {

gd_status gd_gated_create(gd_gated** out, uint32_t in, uint32_t out_features, gd_dtype type, gd_act act, uint64_t max_rows) {
    if (!out) return GD_ERR_ARG;
    *out = nullptr;
    const int ty = gd::enum_int(&type), ac = gd::enum_int(&act);
    if (in == 0 || out_features == 0 || in > gd::kLinearMaxDim || out_features > gd::kLinearMaxDim / 2 ||
        max_rows > 0x7FFFFFFFull || ty < GD_F32 || ty > GD_F16 || ac < GD_ACT_NONE || ac > GD_ACT_SILU)
        return GD_ERR_ARG;
    gd_gated* l = new (std::nothrow) gd_gated();
    if (!l) return GD_ERR_OOM;
    l->in = in;
    l->out = out_features;
    l->type = ty;
    l->act = ac;
    l->max_rows = max_rows;
    if (ty != GD_F32 && (in % 8 || 2ull * out_features % 8)) {
        // the two operands of the forward call, of the input's gradient or of the weight's
        const uint64_t k = (in + 7ull) / 8 * 16, n = (2ull * out_features + 7) / 8 * 16, w = 2 * out_features * k;
        l->pad_bytes = std::min(std::max({max_rows * k + w, max_rows * n + w, max_rows * (k + n)}), gd::kLinearPad);
    }
    gd_status st = GD_OK;
    try {
        if (hipGetDevice(&l->device) != hipSuccess) st = GD_ERR_HIP;
        else if (!l->mem.alloc(&l->room, gd::kLinearRoom) ||
                 !l->mem.alloc(&l->part, (size_t)gd::kBiasParts * 2 * out_features) ||
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

void gd_gated_destroy(gd_gated* l) {
    if (!l) return;
    gd::DeviceGuard guard(l->device);
    delete l;
}

gd_status gd_gated_forward(gd_gated* l, const gd_gated_io* io, void* stream) {
    // no rows have no scales, and an empty buffer may have no address
    if (!l || !io || io->rows > l->max_rows || (io->rows && (io->x_scale == nullptr) != (io->weight_scale == nullptr)))
        return GD_ERR_ARG;
    const auto bad = [](uint64_t stride, uint64_t least) { return stride < least || stride > gd::kLinearMaxDim; };
    if (bad(io->weight_stride, l->in) || (io->rows && (bad(io->x_stride, l->in) || bad(io->y_stride, l->out))) ||
        (io->pre && bad(io->pre_stride, 2ull * l->out)))
        return GD_ERR_ARG;
    const bool int8 = io->x_scale != nullptr;
    if ((int8 && l->in > gd::kLinearMaxInt8) || !gd::product_fits(2ull * l->out, io->rows)) return GD_ERR_LAYOUT;
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
    a.fin.pre = io->pre;
    a.fin.pre_stride = io->pre_stride;
    a.fin.p_scale = io->weight_scale;
    a.fin.q_scale = io->x_scale;
    a.fin.act = l->act;
    const hipStream_t st = (hipStream_t)stream;
    const gd::GemmRoom room{gd::kLinearRoom, l->pad, l->pad_bytes};
    const hipError_t e = l->type == GD_F32    ? gd::gated_forward<float>(a, room, int8, st)
                         : l->type == GD_BF16 ? gd::gated_forward<gd::bf16>(a, room, int8, st)
                                              : gd::gated_forward<gd::f16>(a, room, int8, st);
    return e == hipSuccess ? GD_OK : GD_ERR_HIP;
}

gd_status gd_gated_backward(gd_gated* l, const gd_gated_grad* io, void* stream) {
    if (!l || !io || io->rows > l->max_rows) return GD_ERR_ARG;
    const auto bad = [](uint64_t stride, uint64_t least) { return stride < least || stride > gd::kLinearMaxDim; };
    const bool rows = io->rows != 0;
    const uint64_t wide = 2ull * l->out;
    if ((rows && (!io->dy || !io->pre || !io->dz || bad(io->dy_stride, l->out) || bad(io->pre_stride, wide) ||
                  bad(io->dz_stride, wide))) ||
        (rows && io->dx && (!io->weight || bad(io->weight_stride, l->in) || bad(io->dx_stride, l->in))) ||
        (io->dweight && (bad(io->dweight_stride, l->in) || (rows && (!io->x || bad(io->x_stride, l->in))))))
        return GD_ERR_ARG;
    if ((io->dx && !gd::product_fits(l->in, io->rows)) || (io->dweight && !gd::product_fits(l->in, wide)))
        return GD_ERR_LAYOUT;
    gd::DeviceGuard guard(l->device);
    if (!guard.ok) return GD_ERR_HIP;
    const hipStream_t st = (hipStream_t)stream;
    if (gd::launch_gated_slope(*io, l->type, l->out, l->act, l->part, st) != hipSuccess) return GD_ERR_HIP;
    gd::GemmArgs dx{}, dw{};
    dx.p = io->weight;
    dx.q = io->dz;
    dx.p_stride = io->weight_stride;
    dx.q_stride = io->dz_stride;
    dx.I = l->in;
    dx.J = (uint32_t)io->rows;
    dx.K = (uint32_t)wide;
    dx.part = l->room;
    dx.fin.out = io->dx;
    dx.fin.out_stride = io->dx_stride;
    dw.p = io->x;
    dw.q = io->dz;
    dw.p_stride = io->x_stride;
    dw.q_stride = io->dz_stride;
    dw.I = l->in;
    dw.J = (uint32_t)wide;
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
