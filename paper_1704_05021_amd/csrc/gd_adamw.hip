// AdamW step over all tensors of a layout, with the moments in 32 or 8 bits.
//
// Bound by memory: 28 bytes an element with 32-bit moments (parameter and
// moments read and written, gradient read), 16 with 8-bit ones.  A block takes
// a chunk of 1,024 elements of one tensor, a wave the 256 that share the
// units of the 8-bit moments, a lane four of them: every array is read and
// written once, 16 bytes a lane (4 for codes), and the blocks' maxima stay in
// registers.  Chunks start anew with each tensor, so that no tensor's moments
// depend on its neighbours; a tensor that starts off a 16-byte boundary is
// read at its own alignment.
//
// Operations are those of the definition one by one (no contraction), so a
// step gives the bits that separate binary32 operations give.

#include <cmath>
#include <new>

#include "gd.h"
#include "gd_host.hpp"
#include "gd_ops.hpp"

namespace gd {

constexpr uint32_t kStateBlock = 256;   // elements that share the units of their codes
constexpr uint32_t kAdamChunk = 1024;   // elements of a block of threads
constexpr uint32_t kAdamMaxBlocks = 1u << 22;  // a dispatch holds less than 2^32 threads
constexpr uint32_t kNormBlocks = 1024;  // partial sums of the gradient's squares
constexpr uint64_t kAdamMaxElements = 1ull << 40;

struct AdamChunk {
    uint64_t start_len;  // first element | (elements - 1) << 54
    uint32_t tensor;
    uint32_t block;      // its first block of codes
};
static_assert(kAdamChunk == kBlock * 4 && kStateBlock == kWave * 4, "a lane takes four elements");

struct AdamArgs {
    gd_adamw_io io;
    const AdamChunk* chunks;
    const float* decay;
    const float* scale;  // [2] gradient scale, not 0 when the step is skipped; null: grad_scale
    uint32_t num_chunks;
    float grad_scale, beta1, one_beta1, beta2, one_beta2, step_size, root_scale, eps, lr_decay;
};

// Nearest whole number to the root of y, at most `top` (ties up): the
// hardware's root is off by an ulp at most, so its rounding by one at most, and
// the two squares, exact in binary32, settle it.
__device__ __forceinline__ float root_code(float y, float top) {
    const float r = rintf(__builtin_amdgcn_sqrtf(y));
    const float up = r + 0.5f, down = fmaxf(r - 0.5f, 0.0f);
    return fminf(r + (y >= up * up ? 1.0f : 0.0f) - (y < down * down ? 1.0f : 0.0f), top);
}

// Unit of a block of codes from its largest value's bits.
__device__ __forceinline__ float code_unit(uint32_t max_bits, float top) {
    const float big = __uint_as_float(max_bits);
    return (big < 0x1p-100f ? 0x1p-100f : big) / (top * top);  // a NaN stays
}

__device__ __forceinline__ uint32_t wave_max_bits(const float* x) {
    uint32_t b = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) b = max(b, __float_as_uint(x[j]) & 0x7FFFFFFFu);
    return lane_value(wave_incl_max(b), kWave - 1);
}

template <typename G, typename C, bool CODES>
__global__ __launch_bounds__(kBlock) void k_adamw(AdamArgs a) {
    float gs = a.grad_scale;
    if (a.scale) {
        if (a.scale[1] != 0.0f) return;
        gs = a.scale[0];
    }
    for (uint32_t ch = blockIdx.x; ch < a.num_chunks; ch += gridDim.x) {
        const AdamChunk c = a.chunks[ch];
        const uint64_t at = (c.start_len & ((1ull << 54) - 1)) + threadIdx.x * 4;
        const int n = (int)(c.start_len >> 54) + 1 - (int)threadIdx.x * 4;
        const uint32_t block = c.block + wave_index();
        if ((int)(c.start_len >> 54) < (int)(wave_index() * kStateBlock)) continue;  // no element in this wave
        const Pack<float, 4> p = load_some<4>(a.io.params + at, n);
        const Pack<G, 4> g = load_some<4>((const G*)a.io.grad + at, n);
        float m[4], v[4], root[4];
        if constexpr (CODES) {
            const Pack<int8_t, 4> mc = load_some<4>((const int8_t*)a.io.m + at, n);
            const Pack<uint8_t, 4> vc = load_some<4>((const uint8_t*)a.io.v + at, n);
            const float mu = a.io.m_unit[block], vu = a.io.v_unit[block];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float q = (float)mc.v[j], r = (float)vc.v[j];
                m[j] = mu * (q * fabsf(q));
                v[j] = vu * (r * r);
                v[j] *= v[j];
            }
        } else {
            const Pack<float, 4> ml = load_some<4>((const float*)a.io.m + at, n);
            const Pack<float, 4> vl = load_some<4>((const float*)a.io.v + at, n);
#pragma unroll
            for (int j = 0; j < 4; ++j) m[j] = ml.v[j], v[j] = vl.v[j];
        }
        const float keep = 1.0f - a.lr_decay * a.decay[c.tensor];
        Pack<float, 4> np;
        Pack<C, 4> copy;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float gv = (float)g.v[j] * gs;
            m[j] = m[j] * a.beta1 + gv * a.one_beta1;
            v[j] = v[j] * a.beta2 + gv * gv * a.one_beta2;
            root[j] = sqrtf(v[j]);
            np.v[j] = p.v[j] * keep - m[j] / (root[j] * a.root_scale + a.eps) * a.step_size;
            copy.v[j] = (C)np.v[j];
        }
        store_some<4>(a.io.params + at, np, n);
        if (a.io.copy) store_some<4>((C*)a.io.copy + at, copy, n);
        if constexpr (CODES) {
            if (n < 4)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j >= n) m[j] = root[j] = 0.0f;
            const float mu = code_unit(wave_max_bits(m), 127.0f), vu = code_unit(wave_max_bits(root), 255.0f);
            const float mi = 1.0f / mu, vi = 1.0f / vu;
            Pack<int8_t, 4> mc;
            Pack<uint8_t, 4> vc;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float q = root_code(fabsf(m[j]) * mi, 127.0f);
                mc.v[j] = (int8_t)(m[j] < 0.0f ? -q : q);
                const float r = root_code(root[j] * vi, 255.0f);
                vc.v[j] = (uint8_t)(root[j] > 0.0f ? fmaxf(r, 1.0f) : r);
            }
            store_some<4>((int8_t*)a.io.m + at, mc, n);
            store_some<4>((uint8_t*)a.io.v + at, vc, n);
            if (lane_id() == 0) {
                a.io.m_unit[block] = mu;
                a.io.v_unit[block] = vu;
            }
        } else {
            Pack<float, 4> ml, vl;
#pragma unroll
            for (int j = 0; j < 4; ++j) ml.v[j] = m[j], vl.v[j] = v[j];
            store_some<4>((float*)a.io.m + at, ml, n);
            store_some<4>((float*)a.io.v + at, vl, n);
        }
    }
}

// part[block] = its share of the gradient's sum of squares, in 64 bits.
template <typename G>
__global__ __launch_bounds__(kBlock) void k_square_sum(const G* grad, uint64_t n, double* part) {
    __shared__ double lds[kWavesPerBlock];
    double s = 0.0;
    const uint64_t step = (uint64_t)gridDim.x * kBlock * 4;
#pragma unroll 4
    for (uint64_t at = ((uint64_t)blockIdx.x * kBlock + threadIdx.x) * 4; at < n; at += step) {
        const Pack<G, 4> g = load_some<4>(grad + at, (int)min(n - at, (uint64_t)4));
#pragma unroll
        for (int j = 0; j < 4; ++j) s = fma((double)(float)g.v[j], (double)(float)g.v[j], s);
    }
    s = row_sum<kWavesPerBlock>(s, lds);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// scale[0] = the gradient's scale under the norm's bound, scale[1] = 1 when the norm is not finite.
__global__ __launch_bounds__(kBlock) void k_clip(const double* part, uint32_t parts, double grad_scale, double max_norm,
                                                 float* scale, float* norm) {
    __shared__ double lds[kWavesPerBlock];
    double s = 0.0;
    for (uint32_t i = threadIdx.x; i < parts; i += kBlock) s += part[i];
    s = row_sum<kWavesPerBlock>(s, lds);
    if (threadIdx.x != 0) return;
    const double x = fabs(grad_scale) * sqrt(s);
    scale[0] = (float)(x > max_norm ? grad_scale * (max_norm / x) : grad_scale);
    scale[1] = x <= 1.7976931348623157e308 ? 0.0f : 1.0f;
    if (norm) *norm = (float)x;
}

__global__ __launch_bounds__(kBlock) void k_decode(const AdamChunk* chunks, uint32_t num_chunks, const int8_t* mc,
                                                   const uint8_t* vc, const float* m_unit, const float* v_unit,
                                                   float* m_out, float* v_out) {
    for (uint32_t ch = blockIdx.x; ch < num_chunks; ch += gridDim.x) {
        const AdamChunk c = chunks[ch];
        const uint64_t at = (c.start_len & ((1ull << 54) - 1)) + threadIdx.x * 4;
        const int n = (int)(c.start_len >> 54) + 1 - (int)threadIdx.x * 4;
        if ((int)(c.start_len >> 54) < (int)(wave_index() * kStateBlock)) continue;
        const float mu = m_unit[c.block + wave_index()], vu = v_unit[c.block + wave_index()];
        const Pack<int8_t, 4> q = load_some<4>(mc + at, n);
        const Pack<uint8_t, 4> r = load_some<4>(vc + at, n);
        Pack<float, 4> m, v;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float x = (float)q.v[j], y = (float)r.v[j];
            m.v[j] = mu * (x * fabsf(x));
            v.v[j] = vu * (y * y);
            v.v[j] *= v.v[j];
        }
        store_some<4>(m_out + at, m, n);
        store_some<4>(v_out + at, v, n);
    }
}

template <typename G, typename C>
hipError_t launch_adamw(const AdamArgs& a, bool codes, hipStream_t st) {
    const dim3 grid(std::min(a.num_chunks, kAdamMaxBlocks));
    if (codes)
        k_adamw<G, C, true><<<grid, dim3(kBlock), 0, st>>>(a);
    else
        k_adamw<G, C, false><<<grid, dim3(kBlock), 0, st>>>(a);
    return hipGetLastError();
}

template <typename G>
hipError_t launch_square_sum(const void* grad, uint64_t n, double* part, uint32_t blocks, hipStream_t st) {
    if (blocks) k_square_sum<G><<<dim3(blocks), dim3(kBlock), 0, st>>>((const G*)grad, n, part);
    return hipGetLastError();
}

}  // namespace gd

struct gd_adamw {
    int device = 0;
    uint64_t N = 0, blocks = 0;
    uint32_t num_chunks = 0;
    bool codes = false;
    gd::AdamChunk* chunks = nullptr;  // [num_chunks]
    float* decay = nullptr;           // [T]
    double* part = nullptr;           // [kNormBlocks]
    float* scale = nullptr;           // [2]
    gd::DeviceMemory mem;
};

extern "C" {

gd_status gd_adamw_create(gd_adamw** out, const uint64_t* off, uint32_t T, gd_state state, const float* decay) {
    if (!out) return GD_ERR_ARG;
    *out = nullptr;
    const int kind = gd::enum_int(&state);
    if (!off || T == 0 || kind < GD_STATE_F32 || kind > GD_STATE_8BIT) return GD_ERR_ARG;
    if (off[0] != 0 || off[T] > gd::kAdamMaxElements) return GD_ERR_LAYOUT;
    for (uint32_t t = 0; t < T; ++t)
        if (off[t + 1] < off[t]) return GD_ERR_LAYOUT;
    if (decay)
        for (uint32_t t = 0; t < T; ++t)
            if (!(decay[t] >= 0.0f) || std::isinf(decay[t])) return GD_ERR_ARG;
    gd_adamw* o = nullptr;
    try {
        o = new gd_adamw();
        o->N = off[T];
        o->codes = kind == GD_STATE_8BIT;
        std::vector<gd::AdamChunk> chunks;
        for (uint32_t t = 0; t < T; ++t)
            for (uint64_t a = off[t]; a < off[t + 1]; a += gd::kAdamChunk) {
                const uint64_t len = std::min<uint64_t>(gd::kAdamChunk, off[t + 1] - a);
                chunks.push_back({a | (len - 1) << 54, t, (uint32_t)o->blocks});
                o->blocks += (len + gd::kStateBlock - 1) / gd::kStateBlock;
            }
        if (chunks.size() > 0xFFFFFFFFull - gd::kAdamMaxBlocks || o->blocks > 0xFFFFFFFFull) {
            delete o;
            return GD_ERR_LAYOUT;
        }
        o->num_chunks = (uint32_t)chunks.size();
        std::vector<float> d(T, 1.0f);
        if (decay) d.assign(decay, decay + T);
        gd_status st = GD_OK;
        if (hipGetDevice(&o->device) != hipSuccess) st = GD_ERR_HIP;
        else if (!o->mem.upload(&o->chunks, chunks) || !o->mem.upload(&o->decay, d) ||
                 !o->mem.alloc(&o->part, gd::kNormBlocks) || !o->mem.alloc(&o->scale, 2))
            st = GD_ERR_OOM;
        if (st != GD_OK) {
            delete o;
            return st;
        }
    } catch (const std::exception&) {
        delete o;
        return GD_ERR_OOM;
    }
    *out = o;
    return GD_OK;
}

void gd_adamw_destroy(gd_adamw* o) {
    if (!o) return;
    gd::DeviceGuard guard(o->device);
    delete o;
}

uint64_t gd_adamw_blocks(const gd_adamw* o) { return o ? o->blocks : 0; }

gd_status gd_adamw_step(gd_adamw* o, const gd_adamw_io* io, void* stream) {
    if (!o || !io) return GD_ERR_ARG;
    const int gt = gd::enum_int(&io->grad_type), ct = gd::enum_int(&io->copy_type);
    const auto fine = [](double x) { return x >= 0.0 && !std::isinf(x); };
    if (gt < GD_F32 || gt > GD_F16 || (io->copy && ct != GD_BF16 && ct != GD_F16) || io->step == 0 || !fine(io->lr) ||
        !fine(io->weight_decay) || !(io->beta1 >= 0.0 && io->beta1 < 1.0) || !(io->beta2 >= 0.0 && io->beta2 < 1.0) ||
        !(io->eps >= 0x1p-126) || std::isinf(io->eps) || !(io->max_norm >= 0.0) || !std::isfinite(io->grad_scale))
        return GD_ERR_ARG;
    if (o->N && (!io->params || !io->grad || !io->m || !io->v || (o->codes && (!io->m_unit || !io->v_unit))))
        return GD_ERR_ARG;
    gd::DeviceGuard guard(o->device);
    if (!guard.ok) return GD_ERR_HIP;
    const hipStream_t st = (hipStream_t)stream;
    gd::AdamArgs a{};
    a.io = *io;
    a.chunks = o->chunks;
    a.decay = o->decay;
    a.num_chunks = o->num_chunks;
    a.grad_scale = (float)io->grad_scale;
    a.beta1 = (float)io->beta1;
    a.one_beta1 = (float)(1.0 - io->beta1);
    a.beta2 = (float)io->beta2;
    a.one_beta2 = (float)(1.0 - io->beta2);
    a.step_size = (float)(io->lr / (1.0 - std::pow(io->beta1, (double)io->step)));
    a.root_scale = (float)(1.0 / std::sqrt(1.0 - std::pow(io->beta2, (double)io->step)));
    a.eps = (float)io->eps;
    a.lr_decay = (float)(io->lr * io->weight_decay);
    hipError_t e = hipSuccess;
    if (io->max_norm > 0.0) {
        const uint32_t blocks = (uint32_t)std::min<uint64_t>((o->N + gd::kAdamChunk - 1) / gd::kAdamChunk, gd::kNormBlocks);
        e = gt == GD_F32    ? gd::launch_square_sum<float>(io->grad, o->N, o->part, blocks, st)
            : gt == GD_BF16 ? gd::launch_square_sum<gd::bf16>(io->grad, o->N, o->part, blocks, st)
                            : gd::launch_square_sum<gd::f16>(io->grad, o->N, o->part, blocks, st);
        if (e != hipSuccess) return GD_ERR_HIP;
        gd::k_clip<<<dim3(1), dim3(gd::kBlock), 0, st>>>(o->part, blocks, io->grad_scale, io->max_norm, o->scale, io->norm);
        if (hipGetLastError() != hipSuccess) return GD_ERR_HIP;
        a.scale = o->scale;
    }
    if (!o->num_chunks) return GD_OK;
    const bool half = io->copy && ct == GD_F16;
    if (gt == GD_F32)
        e = half ? gd::launch_adamw<float, gd::f16>(a, o->codes, st) : gd::launch_adamw<float, gd::bf16>(a, o->codes, st);
    else if (gt == GD_BF16)
        e = half ? gd::launch_adamw<gd::bf16, gd::f16>(a, o->codes, st)
                 : gd::launch_adamw<gd::bf16, gd::bf16>(a, o->codes, st);
    else
        e = half ? gd::launch_adamw<gd::f16, gd::f16>(a, o->codes, st)
                 : gd::launch_adamw<gd::f16, gd::bf16>(a, o->codes, st);
    return e == hipSuccess ? GD_OK : GD_ERR_HIP;
}

gd_status gd_adamw_decode(gd_adamw* o, const void* m, const void* v, const float* m_unit, const float* v_unit,
                          float* m_out, float* v_out, void* stream) {
    if (!o || !o->codes) return GD_ERR_ARG;
    if (!o->num_chunks) return GD_OK;
    if (!m || !v || !m_unit || !v_unit || !m_out || !v_out) return GD_ERR_ARG;
    gd::DeviceGuard guard(o->device);
    if (!guard.ok) return GD_ERR_HIP;
    gd::k_decode<<<dim3(std::min(o->num_chunks, gd::kAdamMaxBlocks)), dim3(gd::kBlock), 0, (hipStream_t)stream>>>(
        o->chunks, o->num_chunks, (const int8_t*)m, (const uint8_t*)v, m_unit, v_unit, m_out, v_out);
    return hipGetLastError() == hipSuccess ? GD_OK : GD_ERR_HIP;
}

}  // extern "C"
