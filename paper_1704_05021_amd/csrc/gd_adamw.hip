// AdamW step over all tensors of a layout, with the moments in 32 or 8 bits.
//
// Bound by memory: 28 bytes an element with 32-bit moments (parameter and
// moments read and written, gradient read), 16 with 8-bit ones.  A wave takes
// the 256 elements that share the units of the 8-bit moments, a lane four of
// them: every array is read and written once, 16 bytes a lane (4 for codes),
// and the blocks' maxima stay in registers.  A block of threads takes a chunk
// of one tensor, two to four times 1,024 elements, and starts all its loads
// before the first is used: a chunk's place comes from a table, one round trip
// to memory before them.  Chunks start anew with each tensor, so that no
// tensor's moments depend on its neighbours; a tensor that starts off a
// 16-byte boundary is read at its own alignment.
//
// The moments are formed by the definition's operations one by one (no
// contraction), so that their codes do not depend on this code's shape; the
// parameter's update takes the hardware's reciprocal (one ulp).
//
// Measured over 137M elements, on several cards: 696 to 723 us with 32-bit
// moments (5.3 to 5.5 TB/s, the rate of a large copy or above it), 366 to 413
// with 8-bit ones (5.3 to 6.0 TB/s; one run a block of threads took 474),
// decoding 215 to 268 us (5.1 to 6.4 TB/s); the norm adds 105 to 111 us (5.0
// TB/s).

#include <cmath>
#include <new>

#include "gd.h"
#include "gd_host.hpp"
#include "gd_ops.hpp"

namespace gd {

constexpr uint32_t kStateBlock = 256;   // elements that share the units of their codes
constexpr uint32_t kAdamRun = 1024;      // elements that a block of threads takes side by side
constexpr int kRuns = 2, kRunsCodes = 4; // runs of a chunk, with 32- and 8-bit moments
constexpr uint32_t kAdamMaxBlocks = 1u << 22;  // a dispatch holds less than 2^32 threads
constexpr uint32_t kNormBlocks = 1024;   // partial sums of the gradient's squares
constexpr uint64_t kAdamMaxElements = 1ull << 40, kAdamBlockNumbers = 1ull << 32;

constexpr int kLenShift = 52;            // 12 bits of a chunk's length above its first element

struct AdamChunk {
    uint64_t start_len;  // first element | (elements - 1) << kLenShift
    uint32_t tensor;
    uint32_t block;      // its first block of codes
};
static_assert(kAdamRun == kBlock * 4 && kStateBlock == kWave * 4, "a lane takes four elements");

struct AdamArgs {
    gd_adamw_io io;
    const AdamChunk* chunks;
    const float* decay;
    const float* scale;  // [2] gradient scale, not 0 when the step is skipped; null: grad_scale
    uint32_t num_chunks;
    float grad_scale, beta1, one_beta1, beta2, one_beta2, step_size, root_scale, eps, lr_decay;
};

// The root of x >= 0, rounded to nearest: the hardware's is off by an ulp at
// most, and the sign of x - r (r +- ulp) tells which neighbour is nearest.
// Zero, infinity and NaN give themselves; below 2^-96 the last bit may be off.
__device__ __forceinline__ float root_of(float x) {
    const float r = __builtin_amdgcn_sqrtf(x);
    const float down = __int_as_float(__float_as_int(r) - 1), up = __int_as_float(__float_as_int(r) + 1);
    const float below = fmaf(-down, r, x), above = fmaf(-up, r, x);
    const float s = below <= 0.0f ? down : r;
    return above > 0.0f ? up : s;
}

// Nearest whole number to the root of y >= 0, at most `top` (ties up).  The
// root is taken a little too large, so that its rounding is right or one too
// high, and the square of the border below, exact in binary32, settles it.
__device__ __forceinline__ float root_code(float y, float top) {
    const float r = floorf(fmaf(__builtin_amdgcn_sqrtf(y), 1.0f + 0x1p-22f, 0.5f));
    const float border = r - 0.5f;
    return fminf(y < border * fabsf(border) ? r - 1.0f : r, top);
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

// What four codes of each moment stand for.
__device__ __forceinline__ void decode4(uint32_t mc, uint32_t vc, float mu, float vu, Pack<float, 4>& m, Pack<float, 4>& v) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float q = (float)(int8_t)(mc >> 8 * j), r = (float)(vc >> 8 * j & 0xFFu);
        m.v[j] = mu * (q * fabsf(q));
        v.v[j] = vu * (r * r);
        v.v[j] *= v.v[j];
    }
}

// A wave's 256 elements: what it loads, and what becomes of it.  WHOLE: all 256 are there.
template <typename G, typename C, bool CODES>
struct AdamRun {
    Pack<float, 4> p, m, v;
    Pack<G, 4> g;
    uint32_t mc, vc;  // four codes each
    float mu, vu;

    template <bool WHOLE>
    __device__ __forceinline__ void load(const AdamArgs& a, uint64_t at, int n, uint32_t block) {
        if (WHOLE) n = 4;
        p = load_some<4>(a.io.params + at, n);
        g = load_some<4>((const G*)a.io.grad + at, n);
        if constexpr (CODES) {
            const Pack<uint8_t, 4> mp = load_some<4>((const uint8_t*)a.io.m + at, n);
            const Pack<uint8_t, 4> vp = load_some<4>((const uint8_t*)a.io.v + at, n);
            __builtin_memcpy(&mc, &mp, 4);
            __builtin_memcpy(&vc, &vp, 4);
            mu = a.io.m_unit[block];
            vu = a.io.v_unit[block];
        } else {
            m = load_some<4>((const float*)a.io.m + at, n);
            v = load_some<4>((const float*)a.io.v + at, n);
        }
    }
    template <bool WHOLE>
    __device__ __forceinline__ void step(const AdamArgs& a, uint64_t at, int n, uint32_t block, float gs, float keep) {
        if (WHOLE) n = 4;
        float root[4];
        Pack<C, 4> copy;
        if constexpr (CODES) decode4(mc, vc, mu, vu, m, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float gv = (float)g.v[j] * gs;
            m.v[j] = m.v[j] * a.beta1 + gv * a.one_beta1;
            v.v[j] = v.v[j] * a.beta2 + gv * gv * a.one_beta2;
            root[j] = root_of(v.v[j]);
            p.v[j] = p.v[j] * keep -
                     m.v[j] * __builtin_amdgcn_rcpf(root[j] * a.root_scale + a.eps) * a.step_size;
            copy.v[j] = (C)p.v[j];
        }
        store_some<4>(a.io.params + at, p, n);
        if (a.io.copy) store_some<4>((C*)a.io.copy + at, copy, n);
        if constexpr (CODES) {
            if (!WHOLE)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j >= n) m.v[j] = root[j] = 0.0f;
            mu = code_unit(wave_max_bits(m.v), 127.0f);
            vu = code_unit(wave_max_bits(root), 255.0f);
            const float mi = 1.0f / mu, vi = 1.0f / vu;
            mc = vc = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                // a signed code goes out as itself plus 128, with its highest bit turned
                const float q = root_code(fabsf(m.v[j]) * mi, 127.0f), r = root_code(root[j] * vi, 255.0f);
                mc = __builtin_amdgcn_cvt_pk_u8_f32(128.0f + copysignf(q, m.v[j]), j, mc);
                vc = __builtin_amdgcn_cvt_pk_u8_f32(root[j] > 0.0f ? fmaxf(r, 1.0f) : r, j, vc);
            }
            mc ^= 0x80808080u;
            Pack<uint8_t, 4> mp, vp;
            __builtin_memcpy(&mp, &mc, 4);
            __builtin_memcpy(&vp, &vc, 4);
            store_some<4>((uint8_t*)a.io.m + at, mp, n);
            store_some<4>((uint8_t*)a.io.v + at, vp, n);
            if (lane_id() == 0) {
                a.io.m_unit[block] = mu;
                a.io.v_unit[block] = vu;
            }
        } else {
            store_some<4>((float*)a.io.m + at, m, n);
            store_some<4>((float*)a.io.v + at, v, n);
        }
    }
};

template <typename G, typename C, bool CODES>
__global__ __launch_bounds__(kBlock) void k_adamw(AdamArgs a) {
    constexpr int RUNS = CODES ? kRunsCodes : kRuns;
    float gs = a.grad_scale;
    if (a.scale) {
        if (a.scale[1] != 0.0f) return;
        gs = a.scale[0];
    }
    for (uint32_t ch = blockIdx.x; ch < a.num_chunks; ch += gridDim.x) {
        const AdamChunk c = a.chunks[ch];
        const uint32_t len = (uint32_t)(c.start_len >> kLenShift) + 1, wave = wave_index();
        const uint64_t at = (c.start_len & ((1ull << kLenShift) - 1)) + threadIdx.x * 4;
        const float keep = 1.0f - a.lr_decay * a.decay[c.tensor];
        AdamRun<G, C, CODES> run[RUNS];
        if (len == RUNS * kAdamRun) {
#pragma unroll
            for (int u = 0; u < RUNS; ++u) run[u].template load<true>(a, at + u * kAdamRun, 4, c.block + u * 4 + wave);
#pragma unroll
            for (int u = 0; u < RUNS; ++u)
                run[u].template step<true>(a, at + u * kAdamRun, 4, c.block + u * 4 + wave, gs, keep);
        } else {
            for (uint32_t u = 0; u * kAdamRun + wave * kStateBlock < len; ++u) {
                const int n = (int)len - (int)(u * kAdamRun + threadIdx.x * 4);
                run[0].template load<false>(a, at + u * kAdamRun, n, c.block + u * 4 + wave);
                run[0].template step<false>(a, at + u * kAdamRun, n, c.block + u * 4 + wave, gs, keep);
            }
        }
    }
}

// part[block] = its share of the gradient's sum of squares, in 64 bits.
template <typename G>
__global__ __launch_bounds__(kBlock) void k_square_sum(const G* grad, uint64_t n, double* part) {
    __shared__ double lds[kWavesPerBlock];
    constexpr int kAhead = 8;
    double s = 0.0;
    const uint64_t step = (uint64_t)gridDim.x * kBlock * 4;
    uint64_t at = ((uint64_t)blockIdx.x * kBlock + threadIdx.x) * 4;
    const auto add = [&](const Pack<G, 4>& g) {
#pragma unroll
        for (int j = 0; j < 4; ++j) s = fma((double)(float)g.v[j], (double)(float)g.v[j], s);
    };
    for (; at < n; at += kAhead * step) {
        Pack<G, 4> g[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (at + u * step + 4 <= n) g[u] = load_pack<4>(grad + at + u * step);
            else g[u] = {};
#pragma unroll
        for (int u = 0; u < kAhead; ++u) add(g[u]);
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) add(load_some<4>(grad + n / 4 * 4, (int)(n % 4)));
    s = row_sum<kWavesPerBlock>(s, lds);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// scale[0] = the gradient's scale under the norm's bound, scale[1] = 1 when
// the norm is not finite: the one in 32 bits, which is what the caller gets to
// see, so finite gradients whose norm is past that range skip the step too.  (Its own launch, 4 us: the last block of the sums
// would have to wait for every other's write to reach memory, which with a
// release by each of 1,024 blocks took 40 us.)
__global__ __launch_bounds__(kBlock) void k_clip(const double* part, uint32_t parts, double grad_scale, double max_norm,
                                                 float* scale, float* norm) {
    __shared__ double lds[kWavesPerBlock];
    double s = 0.0;
    for (uint32_t i = threadIdx.x; i < parts; i += kBlock) s += part[i];
    s = row_sum<kWavesPerBlock>(s, lds);
    if (threadIdx.x != 0) return;
    const double x = fabs(grad_scale) * sqrt(s);
    const float seen = (float)x;
    scale[0] = (float)(x > max_norm ? grad_scale * (max_norm / x) : grad_scale);
    scale[1] = seen <= 3.4028234663852886e38f ? 0.0f : 1.0f;
    if (norm) *norm = seen;
}

__global__ __launch_bounds__(kBlock) void k_decode(const AdamChunk* chunks, uint32_t num_chunks, const uint8_t* m,
                                                   const uint8_t* v, const float* m_unit, const float* v_unit,
                                                   float* m_out, float* v_out) {
    for (uint32_t ch = blockIdx.x; ch < num_chunks; ch += gridDim.x) {
        const AdamChunk c = chunks[ch];
        const uint32_t len = (uint32_t)(c.start_len >> kLenShift) + 1, wave = wave_index();
        const uint64_t at = (c.start_len & ((1ull << kLenShift) - 1)) + threadIdx.x * 4;
        Pack<float, 4> mo, vo;
        if (len == kRunsCodes * kAdamRun) {
            uint32_t mc[kRunsCodes], vc[kRunsCodes];
            float mu[kRunsCodes], vu[kRunsCodes];
#pragma unroll
            for (int u = 0; u < kRunsCodes; ++u) {
                __builtin_memcpy(&mc[u], m + at + u * kAdamRun, 4);
                __builtin_memcpy(&vc[u], v + at + u * kAdamRun, 4);
                mu[u] = m_unit[c.block + u * 4 + wave];
                vu[u] = v_unit[c.block + u * 4 + wave];
            }
#pragma unroll
            for (int u = 0; u < kRunsCodes; ++u) {
                decode4(mc[u], vc[u], mu[u], vu[u], mo, vo);
                store_stream<4>(m_out + at + u * kAdamRun, mo, 4);
                store_stream<4>(v_out + at + u * kAdamRun, vo, 4);
            }
        } else {
            for (uint32_t u = 0; u * kAdamRun + wave * kStateBlock < len; ++u) {
                const uint32_t block = c.block + u * 4 + wave;
                const int n = (int)len - (int)(u * kAdamRun + threadIdx.x * 4);
                const Pack<uint8_t, 4> mp = load_some<4>(m + at + u * kAdamRun, n), vp = load_some<4>(v + at + u * kAdamRun, n);
                uint32_t mc, vc;
                __builtin_memcpy(&mc, &mp, 4);
                __builtin_memcpy(&vc, &vp, 4);
                decode4(mc, vc, m_unit[block], v_unit[block], mo, vo);
                store_some<4>(m_out + at + u * kAdamRun, mo, n);
                store_some<4>(v_out + at + u * kAdamRun, vo, n);
            }
        }
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
hipError_t launch_clip(const gd_adamw_io& io, uint64_t n, double* part, float* scale, hipStream_t st) {
    const uint32_t blocks = (uint32_t)std::min<uint64_t>((n + kAdamRun - 1) / kAdamRun, kNormBlocks);
    if (blocks) k_square_sum<G><<<dim3(blocks), dim3(kBlock), 0, st>>>((const G*)io.grad, n, part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    k_clip<<<dim3(1), dim3(kBlock), 0, st>>>(part, blocks, io.grad_scale, io.max_norm, scale, io.norm);
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
    // counted before the table is made: one too long to be held is refused at once
    const uint64_t chunk = gd::kAdamRun * (uint64_t)(kind == GD_STATE_8BIT ? gd::kRunsCodes : gd::kRuns);
    uint64_t num_chunks = 0, blocks = 0;
    for (uint32_t t = 0; t < T; ++t) {
        const uint64_t len = off[t + 1] - off[t];
        num_chunks += (len + chunk - 1) / chunk;
        blocks += (len + gd::kStateBlock - 1) / gd::kStateBlock;
    }
    if (num_chunks > 0xFFFFFFFFull - gd::kAdamMaxBlocks || blocks > gd::kAdamBlockNumbers) return GD_ERR_LAYOUT;
    gd_adamw* o = nullptr;
    try {
        o = new gd_adamw();
        o->N = off[T];
        o->codes = kind == GD_STATE_8BIT;
        std::vector<gd::AdamChunk> chunks;
        chunks.reserve(num_chunks);
        for (uint32_t t = 0; t < T; ++t)
            for (uint64_t a = off[t]; a < off[t + 1]; a += chunk) {
                const uint64_t len = std::min<uint64_t>(chunk, off[t + 1] - a);
                chunks.push_back({a | (len - 1) << gd::kLenShift, t, (uint32_t)o->blocks});
                o->blocks += (len + gd::kStateBlock - 1) / gd::kStateBlock;
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
        e = gt == GD_F32    ? gd::launch_clip<float>(*io, o->N, o->part, o->scale, st)
            : gt == GD_BF16 ? gd::launch_clip<gd::bf16>(*io, o->N, o->part, o->scale, st)
                            : gd::launch_clip<gd::f16>(*io, o->N, o->part, o->scale, st);
        if (e != hipSuccess) return GD_ERR_HIP;
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
        o->chunks, o->num_chunks, (const uint8_t*)m, (const uint8_t*)v, m_unit, v_unit, m_out, v_out);
    return hipGetLastError() == hipSuccess ? GD_OK : GD_ERR_HIP;
}

}  // extern "C"
