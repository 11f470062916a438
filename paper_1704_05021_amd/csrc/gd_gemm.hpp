// The matrix products of the linear layers: out[j][i] = sum_k P(i, k) Q(j, k),
// with bias, activation and residual in the epilogue.
//
// Each operand lies either along k (row i or j holds consecutive k) or across
// it (row k holds consecutive i or j): forward, P is the weight and Q the
// input, both along k; for the input's gradient the weight lies across; for
// the weight's gradient both operands do.  P's rows are the result's
// contiguous direction, so that a lane's four consecutive accumulators are
// neighbours in memory.
//
// A tile of BI x BJ results takes one block, in steps of 128 bytes of k that
// pass through LDS: rows of eight 16-byte chunks, the chunk's place
// exclusive-ored with bits of the row, so that neither the stores nor the
// matrix fragments' reads of 16 rows pile onto a bank.  A matrix instruction's
// lanes each take 16 bytes along k from one row; which k they are does not
// matter as long as both operands agree.  Two forms bring a step there:
//
// gemm_staged, for any operands: while step s is multiplied from one half of
// LDS, step s + 1 goes from registers to the other half, and step s + 3 is
// loaded into those registers (two steps are under way in them).  Operands
// that lie across k are transposed in registers (16-bit elements: one byte
// permutation per two elements; 32-bit ones: none).
//
// gemm_fetch, for 16- and 8-bit operands of whole 16-byte chunks: memory
// instructions place a step in LDS, in no register (below).
//
// PAIR, for gated layers: P holds 2 I rows, I that gate and then the I that are
// gated, and result i is act(gate i) times gated i.  A tile takes both rows of
// its results, 16 that gate and the 16 that they gate in turn: so the two sums
// of a result are in the same lane's registers, two fragments apart, both
// waves' shares of the operand come from one half each, and the products are
// those of one product with 2 I rows.
#pragma once

#include <type_traits>

#include "gd.h"
#include "gd_ops.hpp"

namespace gd {

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef bf16 bf8 __attribute__((ext_vector_type(8)));
typedef f16 h8 __attribute__((ext_vector_type(8)));

template <typename A, typename B>
__device__ __forceinline__ A bits_as(const B& b) {
    static_assert(sizeof(A) == sizeof(B));
    A a;
    __builtin_memcpy(&a, &b, sizeof a);
    return a;
}

// 16 x 16 results from 16-byte fragments: lane l holds row l % 16 and chunk
// l / 16 of a fragment's four; result r of a lane is P row 4 (l / 16) + r,
// Q row l % 16.  (Results of 32 x 32 would need half as many instructions for
// the same reads of LDS, but move more accumulator registers: the product of
// 8192 x 4096 x 4096 took 220 us with them, 205 with these.)
template <typename E>
struct Mma;
template <>
struct Mma<bf16> {
    typedef f4 Sum;
    static __device__ __forceinline__ Sum multiply(u4 a, u4 b, Sum c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(bits_as<bf8>(a), bits_as<bf8>(b), c, 0, 0, 0);
    }
};
template <>
struct Mma<f16> {
    typedef f4 Sum;
    static __device__ __forceinline__ Sum multiply(u4 a, u4 b, Sum c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(bits_as<h8>(a), bits_as<h8>(b), c, 0, 0, 0);
    }
};
template <>
struct Mma<float> {
    typedef f4 Sum;
    static __device__ __forceinline__ Sum multiply(u4 a, u4 b, Sum c) {
        const f4 x = bits_as<f4>(a), y = bits_as<f4>(b);
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
        return c;
    }
};
template <>
struct Mma<int8_t> {
    typedef i4 Sum;
    static __device__ __forceinline__ Sum multiply(u4 a, u4 b, Sum c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(bits_as<i4>(a), bits_as<i4>(b), c, 0, 0, 0);
    }
};

// What becomes of a sum.
struct Finish {
    void* out;              // [J][I] of O
    uint64_t out_stride;
    const void* bias;       // [I] of O, or null
    const void* residual;   // [J][I] of O, or null; out itself where results are added to what is there
    uint64_t residual_stride;
    void* pre;              // [J][I] of O, or null
    uint64_t pre_stride;
    const float* p_scale;   // [I] and [J]: 8-bit operands
    const float* q_scale;
    int act;
    int stream;             // results are more than the caches keep for a reader: stored past them
};

struct GemmArgs {
    const void* p;
    const void* q;
    uint64_t p_stride, q_stride;
    uint32_t I, J, K;
    uint32_t tiles_i, tiles_j;
    uint32_t steps;         // k steps of one split
    float* part;            // [splits][J][I] sums in place of results (int bits for 8-bit operands), or null
    Finish fin;
};

// Activations.  For results of 16 bits the hardware's exponential and
// reciprocal serve, and erf by Abramowitz and Stegun's 7.1.26 (absolute error
// below 1.5e-7): a tile's epilogue is not hidden behind products, and erff
// and expf took 45 us of it over 8192 x 4096 results, these 13.  The slopes
// of that many take 46 us so, with erff and expf 65.

// Phi(z), the normal distribution's, and e = exp(-z^2 / 2).
template <bool EXACT>
__device__ __forceinline__ float normal(float z, float& e) {
    if (EXACT) {
        e = expf(-0.5f * (z * z));
        return 0.5f * (1.0f + erff(z * 0.70710678118654752f));
    }
    const float x = fabsf(z) * 0.70710678118654752f, t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.0f));
    float p = fmaf(1.061405429f, t, -1.453152027f);
    p = fmaf(p, t, 1.421413741f);
    p = fmaf(p, t, -0.284496736f);
    p = fmaf(p, t, 0.254829592f);
    e = __builtin_amdgcn_exp2f(x * x * -1.44269504088896341f);
    const float half = 0.5f * p * t * e;  // (1 - erf x) / 2
    return z < 0.0f ? half : 1.0f - half;
}
// 1 / (1 + exp(-z))
template <bool EXACT>
__device__ __forceinline__ float sigmoid(float z) {
    if (EXACT) return 1.0f / (1.0f + expf(-z));
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504088896341f));
}
// All of s at once, so that a choice of act is one branch: with one an element
// ReLU took 2.3 us over 3739 x 672 results, so 0.6, and SiLU 4.1, so 0.9.
template <bool EXACT, int N>
__device__ __forceinline__ void activate(int act, float (&s)[N]) {
    if (act == GD_ACT_RELU) {
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] = s[c] < 0.0f ? 0.0f : s[c];
    } else if (act == GD_ACT_GELU) {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            float e;
            s[c] *= normal<EXACT>(s[c], e);
        }
    } else if (act == GD_ACT_SILU) {
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] = EXACT ? s[c] / (1.0f + expf(-s[c])) : s[c] * sigmoid<false>(s[c]);
    }
}

// s act'(z) in place of s.  A choice of act is one branch for all of them: one
// an element took longer than the memory.  ReLU chooses and does not multiply:
// a unit that is off passes nothing, a gradient that is not finite neither.
template <bool EXACT, int N>
__device__ __forceinline__ void act_slope(int act, const float (&z)[N], float (&s)[N]) {
    if (act == GD_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < N; ++j) s[j] = z[j] > 0.0f ? s[j] : 0.0f;
    } else if (act == GD_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float e;
            const float cdf = normal<EXACT>(z[j], e);
            s[j] *= cdf + z[j] * (e * 0.39894228040143268f);
        }
    } else if (act == GD_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float q = sigmoid<EXACT>(z[j]);
            s[j] *= q * (1.0f + z[j] * (1.0f - q));
        }
    }
}

template <int N, typename O>
__device__ __forceinline__ void store_result(O* p, const Pack<O, N>& r, int n, bool stream) {
    if constexpr (N * sizeof(O) % 16 == 0) {
        if (stream) return store_stream<N>(p, r, n);
    }
    store_some<N>(p, r, n);
}

// What results of columns i to i + N - 1, n of which exist, share; a thread
// loads it once (8192 x 4096 x 4096 of 8 bits with bias, SiLU and residual:
// 131 us; loaded for every row of results, 147).
template <typename O, int N>
struct Columns {
    Pack<float, N> scale;
    Pack<O, N> bias;
    __device__ __forceinline__ Columns(const Finish& f, uint32_t i, int n) {
        if (f.p_scale) scale = load_some<N>(f.p_scale + i, n);
        if (f.bias) bias = load_some<N>((const O*)f.bias + i, n);
    }
};

// Results (j, i) to (j, i + N - 1), n of which exist, from their sums.
template <typename O, int N>
__device__ __forceinline__ void finish(const Finish& f, const Columns<O, N>& cols, uint64_t j, uint32_t i, float (&s)[N], int n) {
    Pack<O, N> more;  // on its way from here on
    if (f.residual) more = load_some<N>((const O*)f.residual + j * f.residual_stride + i, n);
    if (f.p_scale) {
        const float qs = f.q_scale[j];
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] *= qs * cols.scale.v[c];
    }
    if (f.bias)
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] += (float)cols.bias.v[c];
    if (f.pre) {
        Pack<O, N> z;
#pragma unroll
        for (int c = 0; c < N; ++c) z.v[c] = (O)s[c];
        store_result((O*)f.pre + j * f.pre_stride + i, z, n, f.stream);
    }
    activate<sizeof(O) == 4>(f.act, s);
    if (f.residual)
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] += (float)more.v[c];
    Pack<O, N> y;
#pragma unroll
    for (int c = 0; c < N; ++c) y.v[c] = (O)s[c];
    store_result((O*)f.out + j * f.out_stride + i, y, n, f.stream);
}

// The same for gated results i to i + N - 1 of `all`, from the sums of their two rows.
template <typename O, int N>
struct PairColumns {
    Columns<O, N> gate, gated;
    __device__ __forceinline__ PairColumns(const Finish& f, uint32_t i, uint32_t all, int n)
        : gate(f, i, n), gated(f, i + all, n) {}
};
template <typename O, int N>
__device__ __forceinline__ void finish_pair(const Finish& f, const PairColumns<O, N>& cols, uint64_t j, uint32_t i, uint32_t all,
                                            float (&g)[N], float (&u)[N], int n) {
    if (f.p_scale) {
        const float qs = f.q_scale[j];
#pragma unroll
        for (int c = 0; c < N; ++c) g[c] *= qs * cols.gate.scale.v[c], u[c] *= qs * cols.gated.scale.v[c];
    }
    if (f.bias)
#pragma unroll
        for (int c = 0; c < N; ++c) g[c] += (float)cols.gate.bias.v[c], u[c] += (float)cols.gated.bias.v[c];
    if (f.pre) {
        Pack<O, N> a, b;
#pragma unroll
        for (int c = 0; c < N; ++c) a.v[c] = (O)g[c], b.v[c] = (O)u[c];
        O* pre = (O*)f.pre + j * f.pre_stride + i;
        store_result(pre, a, n, f.stream);
        store_result(pre + all, b, n, f.stream);
    }
    activate<sizeof(O) == 4>(f.act, g);
    Pack<O, N> y;
#pragma unroll
    for (int c = 0; c < N; ++c) y.v[c] = (O)(g[c] * u[c]);
    store_result((O*)f.out + j * f.out_stride + i, y, n, f.stream);
}

constexpr int kStepBytes = 128;  // of k in a step
constexpr int kRowChunks = kStepBytes / 16;

// Byte of chunk c of a tile's row in LDS.
__device__ __forceinline__ uint32_t chunk_at(uint32_t row, uint32_t c) {
    return row * kStepBytes + ((c ^ (row >> 1 & 7u)) << 4);
}

// v moved `bytes` towards its start, zeros behind it.
__device__ __forceinline__ u4 shift_down(u4 v, uint32_t bytes) {
    const u4 zero = {0, 0, 0, 0};
    if (bytes >= 16) v = zero;
    if (bytes & 8) v = u4{v[2], v[3], 0, 0};
    if (bytes & 4) v = u4{v[1], v[2], v[3], 0};
    const uint32_t by = bytes & 3;
    return u4{__builtin_amdgcn_alignbyte(v[1], v[0], by), __builtin_amdgcn_alignbyte(v[2], v[1], by),
              __builtin_amdgcn_alignbyte(v[3], v[2], by), __builtin_amdgcn_alignbyte(0u, v[3], by)};
}

// Row r of a tile of pairs, 16 rows that gate before the 16 that they gate, is its result pair_row(r)'s.  A wave carries
// eight rows at a time, and every turn of four waves or eight starts at a multiple of 32: so all of its rows gate, or none.
__device__ __forceinline__ uint32_t pair_row(uint32_t r) { return r / 32 * 16 + r % 16; }
__device__ __forceinline__ uint32_t pair_half() { return wave_index() >> 1 & 1; }

// A step's R rows of one operand on their way from memory to LDS, the
// block's THREADS threads sharing them.  Where a row or k ends inside a
// vector, the vector that ends there is read, and moved into place on its way
// to LDS: no load waits for another (element by element, each behind its own
// condition, 20 x 650 x 650 took 33 us backward, so 13).  Rows shorter than a
// vector (few) are read by elements.
template <typename E, bool ACROSS, int R, int THREADS>
struct TileLoad;

template <typename E, int R, int THREADS>
struct TileLoad<E, false, R, THREADS> {
    static constexpr int CE = 16 / sizeof(E), KE = kStepBytes / sizeof(E), N = R * kRowChunks / THREADS;
    static_assert(R * kRowChunks % THREADS == 0, "every thread carries whole chunks");
    const E* base;       // the tile's first row at the first step's k
    uint32_t off[N];     // elements
    bool few;            // k is shorter than a chunk
    struct Regs {
        u4 r[N];
    };
    static __device__ __forceinline__ uint32_t first_k(int n) { return (n * THREADS + threadIdx.x) % kRowChunks * CE; }

    __device__ void start(const void* p, uint64_t stride, uint32_t row0, uint32_t rows, uint32_t k0, uint32_t k) {
        base = (const E*)p + (uint64_t)row0 * stride + k0;
        few = k < (uint32_t)CE;
#pragma unroll
        for (int n = 0; n < N; ++n) {  // rows past the end repeat the last one; their results are dropped
            const uint32_t id = n * THREADS + threadIdx.x;
            off[n] = min(id / kRowChunks, rows - row0 - 1) * (uint32_t)stride + first_k(n);
        }
    }
    // Of a pair of operands `rows` apart: result row0 is the tile's first (see pair_row).
    __device__ void start_pair(const void* p, uint64_t stride, uint32_t row0, uint32_t rows, uint32_t k0, uint32_t k) {
        base = (const E*)p + ((uint64_t)row0 + (uint64_t)pair_half() * rows) * stride + k0;
        few = k < (uint32_t)CE;
#pragma unroll
        for (int n = 0; n < N; ++n)
            off[n] = min(pair_row((n * THREADS + threadIdx.x) / kRowChunks), rows - row0 - 1) * (uint32_t)stride + first_k(n);
    }
    __device__ __forceinline__ bool always_whole() const { return true; }
    __device__ __forceinline__ void load_whole(Regs& g, uint32_t step) const {
        const E* at = base + (uint64_t)step * KE;
#pragma unroll
        for (int n = 0; n < N; ++n) g.r[n] = bits_as<u4>(load_pack<CE>(at + off[n]));
    }
    __device__ __forceinline__ void load(Regs& g, uint32_t step, uint32_t k_left) const {
        if (k_left >= (uint32_t)KE) return load_whole(g, step);
        const E* at = base + (uint64_t)step * KE;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int have = (int)k_left - (int)first_k(n);
            if (few)
                g.r[n] = bits_as<u4>(load_some<CE>(at + off[n], have));
            else
                g.r[n] = bits_as<u4>(load_pack<CE>(at + off[n] + min(have - CE, 0)));
        }
    }
    __device__ __forceinline__ void store(const Regs& g, char* lds, uint32_t k_left) const {
        const bool end = k_left < (uint32_t)KE && !few;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const uint32_t id = n * THREADS + threadIdx.x;
            u4 v = g.r[n];
            if (end) v = shift_down(v, (uint32_t)max((int)first_k(n) + CE - (int)k_left, 0) * (uint32_t)sizeof(E));
            *(u4*)(lds + chunk_at(id / kRowChunks, id % kRowChunks)) = v;
        }
    }
};

template <typename E, int R, int THREADS>
struct TileLoad<E, true, R, THREADS> {
    // an item: one chunk of k of four neighbouring rows of the tile
    static constexpr int CE = 16 / sizeof(E), KE = kStepBytes / sizeof(E);
    static constexpr int ITEMS = R / 4 * kRowChunks, N = (ITEMS + THREADS - 1) / THREADS;
    const E* base;
    uint64_t stride;
    uint32_t rows;       // of the operand from the tile's first on
    bool few, edge;      // the operand has fewer than four rows; the tile has rows past its end
    struct Regs {
        Pack<E, 4> r[N][CE];
    };

    static __device__ __forceinline__ uint32_t group(int n) { return (n * THREADS + threadIdx.x) % (R / 4); }
    static __device__ __forceinline__ uint32_t chunk(int n) { return (n * THREADS + threadIdx.x) / (R / 4); }
    // how far the item's vector of four rows lies before the item
    __device__ __forceinline__ int before(int n) const { return max((int)group(n) * 4 + 4 - (int)rows, 0); }

    __device__ void start(const void* p, uint64_t st, uint32_t row0, uint32_t all, uint32_t k0, uint32_t) {
        stride = st;
        base = (const E*)p + (uint64_t)k0 * st + row0;
        rows = min(all - row0, (uint32_t)R);
        few = all < 4;
        edge = rows < (uint32_t)R;
    }
    __device__ __forceinline__ bool always_whole() const { return !few; }
    __device__ __forceinline__ void load_whole(Regs& g, uint32_t step) const {
        const E* at = base + (uint64_t)step * KE * stride;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (N * THREADS > ITEMS && chunk(n) >= (uint32_t)kRowChunks) continue;
            const int64_t off = (int64_t)(chunk(n) * CE * (uint32_t)stride + group(n) * 4) - before(n);
#pragma unroll
            for (int e = 0; e < CE; ++e) g.r[n][e] = load_pack<4>(at + (uint64_t)e * stride + off);
        }
    }
    __device__ __forceinline__ void load(Regs& g, uint32_t step, uint32_t k_left) const {
        const E* at = base + (uint64_t)step * KE * stride;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (N * THREADS > ITEMS && chunk(n) >= (uint32_t)kRowChunks) continue;
#pragma unroll
            for (int e = 0; e < CE; ++e) {
                const uint32_t k = chunk(n) * CE + e;
                const E* row = at + (uint64_t)min(k, k_left - 1) * stride + group(n) * 4;  // past the end of k the last again
                if (few)
                    g.r[n][e] = load_some<4>(row, (int)rows - (int)(group(n) * 4));
                else
                    g.r[n][e] = load_pack<4>(row - before(n));
            }
        }
    }
    __device__ __forceinline__ void store(const Regs& g, char* lds, uint32_t k_left) const {
        const bool end = k_left < (uint32_t)KE;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (N * THREADS > ITEMS && chunk(n) >= (uint32_t)kRowChunks) continue;
            Pack<E, 4> r[CE];
#pragma unroll
            for (int e = 0; e < CE; ++e) r[e] = g.r[n][e];
            if (edge && !few) {
#pragma unroll
                for (int e = 0; e < CE; ++e) r[e] = moved(r[e], before(n));
            }
            if (end) {
#pragma unroll
                for (int e = 0; e < CE; ++e)
                    if (chunk(n) * CE + e >= k_left) r[e] = Pack<E, 4>{};
            }
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                Pack<E, CE> c;
#pragma unroll
                for (int e = 0; e < CE; ++e) c.v[e] = r[e].v[m];
                *(u4*)(lds + chunk_at(group(n) * 4 + m, chunk(n))) = bits_as<u4>(c);
            }
        }
    }
    // r with its first `by` elements gone; what fills the end is a row past the operand's, whose results are dropped
    static __device__ __forceinline__ Pack<E, 4> moved(const Pack<E, 4>& r, int by) {
        if constexpr (sizeof(E) == 2) {
            return bits_as<Pack<E, 4>>(bits_as<uint64_t>(r) >> (by * 16 & 63));
        } else {
            Pack<E, 4> m = r;
            if (by & 2) m.v[0] = m.v[2], m.v[1] = m.v[3];
            if (by & 1) m.v[0] = m.v[1], m.v[1] = m.v[2], m.v[2] = m.v[3];
            return m;
        }
    }
};

// WI x WJ waves of NI x NJ 16 x 16 results each.
template <int WI_, int WJ_, int NI_, int NJ_, int DEEP_ = 2>
struct Tile {
    static constexpr int WI = WI_, WJ = WJ_, NI = NI_, NJ = NJ_, DEEP = DEEP_;  // DEEP: steps in LDS, where they go straight there
    static constexpr int BI = WI * NI * 16, BJ = WJ * NJ * 16, kThreads = WI * WJ * kWave;
    static constexpr int kStage = (BI + BJ) * kStepBytes;           // bytes of LDS of one step
    static constexpr int kLds = 2 * kStage;
    static_assert(WI * WJ * NI * 16 * 16 * 4 <= kLds, "the epilogue's rows fit where the operands were");
};
typedef Tile<2, 4, 8, 4> TileBig;    // 256 x 256
typedef Tile<2, 4, 8, 3> TileLong;   // 256 x 192
typedef Tile<2, 4, 8, 2> TileWide;   // 256 x 128
typedef Tile<2, 2, 4, 4> TileMid;    // 128 x 128
typedef Tile<2, 2, 2, 2, 4> TileSmall;  // 64 x 64; four deep: 256 x 4096 x 4096 took 47 us with two, 23 with four

// The tile of block b: blocks go to the eight dies in turn, so each die is
// given a run of neighbouring tiles, and a run goes through 8 tiles along j
// before the next along i, so that the operands' rows are shared in its L2.
__device__ __forceinline__ void tile_of(const GemmArgs& a, uint32_t b, uint32_t& ti, uint32_t& tj) {
    const uint32_t n = a.tiles_i * a.tiles_j, x = b % 8, per = n / 8, rest = n % 8;
    const uint32_t t = x * per + min(x, rest) + b / 8;
    constexpr uint32_t kRun = 8;
    const uint32_t g = t / (kRun * a.tiles_i), wide = min(kRun, a.tiles_j - g * kRun), in = t - g * kRun * a.tiles_i;
    ti = in / wide;
    tj = g * kRun + in % wide;
}

// The block's sums to their results.  A wave's go through LDS, 16 rows j of
// all its i at a time, so that it reads and writes whole runs of memory.
template <typename E, typename O, typename TL, bool PAIR = false>
__device__ __forceinline__ void store_tile(const GemmArgs& a, typename Mma<E>::Sum (&acc)[TL::NI][TL::NJ], char* lds,
                                           uint32_t i0, uint32_t j0, uint32_t split) {
    const uint32_t wave = wave_index(), lane = lane_id(), wi = wave % TL::WI, wj = wave / TL::WI;
    constexpr int W = TL::NI * 16;  // results of a row
    float* rows = (float*)(lds + wave * (W * 16 * 4));
    constexpr int kPer = 8, kResults = PAIR ? W / 2 : W, kLanes = kResults / kPer, kAtOnce = kWave / kLanes;
    const uint32_t col = lane % kLanes * kPer, i = i0 + wi * kResults + col;
    const int n = i < a.I ? (int)min(a.I - i, (uint32_t)kPer) : 0;
    const std::conditional_t<PAIR, PairColumns<O, kPer>, Columns<O, kPer>> cols = [&] {
        if constexpr (PAIR)
            return PairColumns<O, kPer>(a.fin, i, a.I, a.part ? 0 : n);
        else
            return Columns<O, kPer>(a.fin, i, a.part ? 0 : n);
    }();
#pragma unroll
    for (int j = 0; j < TL::NJ; ++j) {
#pragma unroll
        for (int i = 0; i < TL::NI; ++i) {
            const uint32_t col = i * 16 + (lane >> 4) * 4, row = lane & 15;
            *(f4*)(rows + row * W + (col ^ ((row & 7) << 2))) = bits_as<f4>(acc[i][j]);
        }
        wave_lds_sync();
#pragma unroll 1
        for (uint32_t r = lane / kLanes; r < 16; r += kAtOnce) {
            const uint32_t row = j0 + (wj * TL::NJ + j) * 16 + r;
            const auto get = [&](uint32_t from, float (&s)[kPer]) {
                const f4 lo = *(const f4*)(rows + r * W + (from ^ ((r & 7) << 2)));
                const f4 hi = *(const f4*)(rows + r * W + ((from + 4) ^ ((r & 7) << 2)));
#pragma unroll
                for (int c = 0; c < 4; ++c) s[c] = lo[c], s[c + 4] = hi[c];
            };
            const auto put = [&](const float (&s)[kPer], uint64_t to) {
                Pack<float, kPer> v;
#pragma unroll
                for (int c = 0; c < kPer; ++c) v.v[c] = s[c];
                store_some<kPer>(a.part + to, v, n);
            };
            const auto whole = [&](float (&s)[kPer]) {
                if constexpr (sizeof(E) == 1)
#pragma unroll
                    for (int c = 0; c < kPer; ++c) s[c] = (float)bits_as<int>(s[c]);
            };
            float s[kPer];
            if constexpr (PAIR) {
                float u[kPer];
                get(col / 16 * 32 + col % 16, s);
                get(col / 16 * 32 + col % 16 + 16, u);
                if (row < a.J && n > 0) {
                    if (a.part) {
                        const uint64_t to = ((uint64_t)split * a.J + row) * 2 * a.I + i;
                        put(s, to);
                        put(u, to + a.I);
                    } else {
                        whole(s);
                        whole(u);
                        finish_pair<O, kPer>(a.fin, cols, row, i, a.I, s, u, n);
                    }
                }
            } else {
                get(col, s);
                if (row < a.J && n > 0) {
                    if (a.part) {
                        put(s, ((uint64_t)split * a.J + row) * a.I + i);
                    } else {
                        whole(s);
                        finish<O, kPer>(a.fin, cols, row, i, s, n);
                    }
                }
            }
        }
        wave_lds_sync();
    }
}

// Tile `block` of a product, its share `split` of k, through registers; lds holds TL::kLds bytes.
template <typename E, typename O, bool PA, bool QA, typename TL, bool PAIR = false, int SETS = 2>
__device__ __forceinline__ void gemm_staged(const GemmArgs& a, uint32_t block, uint32_t split, char* lds) {
    using M = Mma<E>;
    constexpr uint32_t KE = kStepBytes / sizeof(E);
    uint32_t ti, tj;
    tile_of(a, block, ti, tj);
    const uint32_t i0 = ti * (PAIR ? TL::BI / 2 : TL::BI), j0 = tj * TL::BJ;
    const uint32_t k0 = split * a.steps * KE;
    const uint32_t k_end = min((uint64_t)a.K, (uint64_t)k0 + (uint64_t)a.steps * KE);
    const uint32_t steps = k_end > k0 ? (k_end - k0 + KE - 1) / KE : 0;

    TileLoad<E, PA, TL::BI, TL::kThreads> lp;
    TileLoad<E, QA, TL::BJ, TL::kThreads> lq;
    if constexpr (PAIR)
        lp.start_pair(a.p, a.p_stride, i0, a.I, k0, a.K);
    else
        lp.start(a.p, a.p_stride, i0, a.I, k0, a.K);
    lq.start(a.q, a.q_stride, j0, a.J, k0, a.K);
    typename M::Sum acc[TL::NI][TL::NJ];
#pragma unroll
    for (int i = 0; i < TL::NI; ++i)
#pragma unroll
        for (int j = 0; j < TL::NJ; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][j][r] = 0;

    const uint32_t wave = wave_index(), lane = lane_id();
    const uint32_t wi = wave % TL::WI, wj = wave / TL::WI;
    // this lane's row and chunk of a fragment: bits 1 to 3 of the row set the chunk's place, those of 16 rows on do not
    const uint32_t at = chunk_at(lane & 15, lane >> 4);
    const uint32_t p_at = wi * TL::NI * 16 * kStepBytes + at;
    const uint32_t q_at = TL::BI * kStepBytes + wj * TL::NJ * 16 * kStepBytes + at;

    typename decltype(lp)::Regs rp[SETS];
    typename decltype(lq)::Regs rq[SETS];
    const uint32_t left = k_end > k0 ? k_end - k0 : 0;
    const uint32_t whole = lp.always_whole() && lq.always_whole() ? left / KE : 0;  // steps whose every load is a vector
    const auto load = [&](int set, uint32_t s) {
        if (s >= steps) return;
        lp.load(rp[set], s, left - s * KE);
        lq.load(rq[set], s, left - s * KE);
    };
    const auto store = [&](int set, uint32_t s, uint32_t k_left) {
        char* to = lds + (s & 1) * TL::kStage;
        lp.store(rp[set], to, k_left);
        lq.store(rq[set], to + TL::BI * kStepBytes, k_left);
    };
    const auto multiply = [&](uint32_t s, int c) {
        const char* now = lds + (s & 1) * TL::kStage;
        u4 p[TL::NI], q[TL::NJ];
#pragma unroll
        for (int i = 0; i < TL::NI; ++i)
            p[i] = *(const u4*)(now + ((p_at ^ (c << 6)) + i * 16 * kStepBytes));
#pragma unroll
        for (int j = 0; j < TL::NJ; ++j)
            q[j] = *(const u4*)(now + ((q_at ^ (c << 6)) + j * 16 * kStepBytes));
#pragma unroll
        for (int i = 0; i < TL::NI; ++i)
#pragma unroll
            for (int j = 0; j < TL::NJ; ++j) acc[i][j] = M::multiply(p[i], q[j], acc[i][j]);
    };
    // step s multiplies what LDS holds, stores step s + 1, loaded SETS steps
    // ago, to the other half, and loads into its registers anew
    if (steps) {
        load(0, 0);
        store(0, 0, left);
#pragma unroll
        for (int d = 0; d < SETS; ++d) load(d, d + 1);
    }
    __syncthreads();
    uint32_t s = 0;
    for (; s + 2 * SETS < whole; s += SETS)
#pragma unroll
        for (int d = 0; d < SETS; ++d) {
            multiply(s + d, 0);
            store(d, s + d + 1, KE);
            lp.load_whole(rp[d], s + d + 1 + SETS);
            lq.load_whole(rq[d], s + d + 1 + SETS);
            multiply(s + d, 1);
            __syncthreads();
        }
#pragma unroll 1
    for (; s < steps; s += SETS)
#pragma unroll
        for (int d = 0; d < SETS; ++d) {
            if (s + d >= steps) break;
            multiply(s + d, 0);
            if (s + d + 1 < steps) store(d, s + d + 1, left - (s + d + 1) * KE);
            load(d, s + d + 1 + SETS);
            multiply(s + d, 1);
            __syncthreads();
        }

    store_tile<E, O, TL, PAIR>(a, acc, lds, i0, j0, split);
}

template <typename E, typename O, bool PA, bool QA, typename TL, bool PAIR = false>
__global__ __launch_bounds__(TL::kThreads, 2) void k_gemm(GemmArgs a) {
    __shared__ __align__(16) char lds[TL::kLds];
    gemm_staged<E, O, PA, QA, TL, PAIR>(a, blockIdx.x, blockIdx.y, lds);
}

// ---- The same product with operands that memory instructions place in LDS ----
//
// For 16- and 8-bit operands whose rows start at 16-byte boundaries and whose
// last 16 bytes may be read whole (along k with zeros behind the end of k):
// the caller's where their sizes are so, else copies made by k_pad.
// LDS has room for DEEP steps, two for the larger tiles.  While step s is
// multiplied, the next DEEP - 1 are on their way from memory straight into
// LDS, in no register; one barrier, behind the last reads of step s, both
// shows that step s + 1 has come for every wave and frees the room of step s
// for step s + DEEP.  Each fragment is read
// right behind the last use of the one whose registers it takes.
//
// Along k a row's eight 16-byte chunks change places by bits 1 to 3 of the row:
// the 16 lanes that a 16-byte read serves at once take their rows from both
// halves of a fragment (bits 0 to 2 cost a second turn for every read).
// Across k the tile lies in LDS as in memory, a row for each k, and the
// transposing LDS read gives each lane four k of one row; pairs of 16-byte
// chunks change places by the low bits of k.  A load puts its lanes' data
// side by side, so the places are chosen by what each lane fetches.
static __device__ const u4 zero_chunk = {0, 0, 0, 0};  // what lanes past the end of k fetch

// 16 bytes from base + off to each lane's place after lds_at (uniform).  The
// instruction writes no register; load_wait says when its data is there.  (The
// compiler's builtin would have it wait for all of them before the next read
// of LDS.  m0 is reserved: the compiler sets it before each use of its own.)
__device__ __forceinline__ void fetch(const void* base, uint32_t off, uint32_t lds_at) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds_at)
                 : "memory");
}
__device__ __forceinline__ void fetch_far(const void* at, uint32_t lds_at) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(at), "s"(lds_at)
                 : "memory");
}
// Until at most N fetches of this wave are under way and its LDS reads are done; then until all waves are here.
template <int N>
__device__ __forceinline__ void load_wait() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <typename E, bool ACROSS, int R, int THREADS>
struct TileFetch {
    static constexpr int kBytes = R * kStepBytes, N = kBytes / (THREADS * 16), KE = kStepBytes / sizeof(E);
    static constexpr int CE = 16 / sizeof(E);
    static constexpr int kRowBytes = ACROSS ? R * (int)sizeof(E) : kStepBytes;
    static constexpr int kUnits = kRowBytes / 32;  // across: pairs of chunks of a k
    static_assert(kBytes % (THREADS * 16) == 0 && (!ACROSS || sizeof(E) == 2));
    const E* base;      // the tile's first row at the first step's k
    uint64_t per_step;  // bytes
    uint32_t stride;
    uint32_t off[N];    // bytes

    // k and row, in elements of the tile, of the chunk that this lane fetches with its n-th load
    static __device__ __forceinline__ uint32_t at(int n) {
        return (n * (THREADS / kWave) + wave_index()) * kWave * 16 + lane_id() * 16;
    }
    // The 32 lanes that a transposing read serves at once take k to k + 3 and k + 8 to k + 11 of one pair of chunks: eight
    // runs of 32 bytes, one on each eighth of the banks.  (Tiles of 64 rows turn by half the banks with every k.)
    static __device__ __forceinline__ uint32_t place(uint32_t k) {
        static_assert(!ACROSS || kUnits == 4 || kUnits == 8 || kUnits == 16, "exclusive-or stays within a row");
        return kUnits >= 8 ? (k & 3) << 1 | (k >> 3 & 1) : (k >> 1 & 1) | (k >> 3 & 1) << 1;
    }
    static __device__ __forceinline__ uint32_t row_place(uint32_t row) {
        return row >> 1 & 7;
    }
    static __device__ __forceinline__ uint32_t k_of(int n) {
        if constexpr (ACROSS) return at(n) / kRowBytes;
        const uint32_t row = at(n) / kStepBytes;
        return ((at(n) / 16 % (kStepBytes / 16)) ^ row_place(row)) * CE;
    }
    static __device__ __forceinline__ uint32_t row_of(int n) {
        if constexpr (!ACROSS) return at(n) / kStepBytes;
        const uint32_t chunk = at(n) % kRowBytes / 16;
        return ((chunk >> 1) ^ place(k_of(n))) * 16 + (chunk & 1) * 8;
    }
    __device__ void start(const void* p, uint64_t st, uint32_t row0, uint32_t rows, uint32_t k0) {
        stride = (uint32_t)st;
        base = (const E*)p + (ACROSS ? (uint64_t)k0 * st + row0 : (uint64_t)row0 * st + k0);
        per_step = (ACROSS ? KE * st : KE) * sizeof(E);
        // rows past the end repeat the last; their results are dropped
        const uint32_t last = ACROSS ? (rows + CE - 1) / CE * CE - row0 - CE : rows - row0 - 1;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const uint32_t r = min(row_of(n), last);
            off[n] = (ACROSS ? k_of(n) * stride + r : r * stride + k_of(n)) * (uint32_t)sizeof(E);
        }
    }
    // Of a pair of operands `rows` apart, along k: result row0 is the tile's first (see pair_row).
    __device__ void start_pair(const void* p, uint64_t st, uint32_t row0, uint32_t rows, uint32_t k0) {
        static_assert(!ACROSS && THREADS % 256 == 0);
        stride = (uint32_t)st;
        base = (const E*)p + ((uint64_t)row0 + (uint64_t)pair_half() * rows) * st + k0;
        per_step = KE * sizeof(E);
#pragma unroll
        for (int n = 0; n < N; ++n)
            off[n] = (min(pair_row(row_of(n)), rows - row0 - 1) * stride + k_of(n)) * (uint32_t)sizeof(E);
    }
    template <bool WHOLE>
    __device__ __forceinline__ void issue(uint32_t step, uint32_t k_left, uint32_t lds_at) const {
        const char* from = (const char*)base + step * per_step;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const uint32_t to = lds_at + (n * (THREADS / kWave) + wave_index()) * kWave * 16;
            if (WHOLE)
                fetch(from, off[n], to);
            else
                fetch_far(k_of(n) < k_left ? (const void*)(from + off[n]) : &zero_chunk, to);
        }
    }
    // This lane's part of the address of its fragment of 16 rows, 16 bytes of k a lane, number c of the step.
    static __device__ __forceinline__ uint32_t lane_at(int c) {
        const uint32_t l = lane_id();
        if constexpr (ACROSS) {
            const uint32_t k = c * 32 + (l >> 4) * 8 + l % 16 / 4;
            return k * kRowBytes + (place(k) << 5) + l % 4 * 8;
        }
        const uint32_t row = l & 15;
        return row * kStepBytes + (((c * 4 + (l >> 4)) ^ row_place(row)) << 4);
    }
    // The fragment of rows row0 (a multiple of 16) on; lane is lane_at(c), the tile starts at `tile` in LDS.
    static __device__ __forceinline__ u4 fragment(const char* tile, uint32_t row0, uint32_t lane) {
        if constexpr (ACROSS) {
            // 16 rows are a pair of chunks; a k's row is a power of two of them, so the exclusive-or keeps to it
            typedef short s4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s4 lds_s4;
            const char* p = tile + (lane ^ (row0 / 16 << 5));
            u4 v;
            const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)p);
            const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(p + 4 * kRowBytes));
            __builtin_memcpy(&v, &lo, 8);
            __builtin_memcpy((char*)&v + 8, &hi, 8);
            return v;
        }
        return *(const u4*)(tile + row0 * kStepBytes + lane);
    }
};

// A copy of an operand's rows at 16-byte boundaries, zeros behind their ends: 16 bytes a thread.
template <typename E>
__global__ __launch_bounds__(kBlock) void k_pad(const E* from, uint64_t stride, uint64_t rows, uint32_t columns, E* to) {
    constexpr uint32_t CE = 16 / sizeof(E);
    const uint32_t per_row = (columns + CE - 1) / CE;
    const uint64_t all = rows * per_row;
    for (uint64_t t = (uint64_t)blockIdx.x * kBlock + threadIdx.x; t < all; t += (uint64_t)gridDim.x * kBlock) {
        const uint64_t row = t / per_row;
        const uint32_t c = (uint32_t)(t - row * per_row) * CE;
        store_pack<CE>(to + t * CE, load_some<CE>(from + row * stride + c, (int)(columns - c)));
    }
}

// Tile `block` of a product, its share `split` of k; lds holds TL::DEEP steps.
template <typename E, typename O, bool PA, bool QA, typename TL, bool PAIR = false>
__device__ __forceinline__ void gemm_fetch(const GemmArgs& a, uint32_t block, uint32_t split, char* lds) {
    using M = Mma<E>;
    using FP = TileFetch<E, PA, TL::BI, TL::kThreads>;
    using FQ = TileFetch<E, QA, TL::BJ, TL::kThreads>;
    static_assert(FP::kBytes + FQ::kBytes == TL::kStage);
    constexpr int DEEP = TL::DEEP, kLoads = FP::N + FQ::N;
    uint32_t ti, tj;
    tile_of(a, block, ti, tj);
    const uint32_t i0 = ti * (PAIR ? TL::BI / 2 : TL::BI), j0 = tj * TL::BJ;
    const uint32_t k0 = split * a.steps * FP::KE;
    const uint32_t k_end = min((uint64_t)a.K, (uint64_t)k0 + (uint64_t)a.steps * FP::KE);
    const uint32_t left = k_end > k0 ? k_end - k0 : 0, steps = (left + FP::KE - 1) / FP::KE, whole = left / FP::KE;
    FP fp;
    FQ fq;
    if constexpr (PAIR)
        fp.start_pair(a.p, a.p_stride, i0, a.I, k0);
    else
        fp.start(a.p, a.p_stride, i0, a.I, k0);
    fq.start(a.q, a.q_stride, j0, a.J, k0);
    typename M::Sum acc[TL::NI][TL::NJ];
#pragma unroll
    for (int i = 0; i < TL::NI; ++i)
#pragma unroll
        for (int j = 0; j < TL::NJ; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][j][r] = 0;

    const uint32_t wave = wave_index(), wi = wave % TL::WI, wj = wave / TL::WI;
    const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    uint32_t p_at[2], q_at[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) p_at[c] = FP::lane_at(c), q_at[c] = FQ::lane_at(c);
    const auto issue = [&](uint32_t s) {
        if (s >= steps) return;
        const uint32_t to = lds_at + s % DEEP * TL::kStage;
        if (s < whole) {
            fp.template issue<true>(s, 0, to);
            fq.template issue<true>(s, 0, to + FP::kBytes);
        } else {
            fp.template issue<false>(s, left - s * FP::KE, to);
            fq.template issue<false>(s, left - s * FP::KE, to + FP::kBytes);
        }
    };
    u4 p[TL::NI], qa[TL::NJ], qb[TL::NJ];
    const auto read_p = [&](uint32_t s, int c, int i) {
        p[i] = FP::fragment(lds + s % DEEP * TL::kStage, (wi * TL::NI + i) * 16, p_at[c]);
    };
    const auto read_q = [&](uint32_t s, int c, int j) {
        return FQ::fragment(lds + s % DEEP * TL::kStage + FP::kBytes, (wj * TL::NJ + j) * 16, q_at[c]);
    };
    // The products of p and q; each fragment of group nc of step ns is read behind the last use of the one whose
    // place it takes.  `before` comes before the first read, more(m) behind product m.
    const auto group = [&](uint32_t ns, int nc, u4 (&nq)[TL::NJ], const u4 (&q)[TL::NJ], auto before, auto more) {
#pragma unroll
        for (int i = 0; i < TL::NI; ++i) {
#pragma unroll
            for (int j = 0; j < TL::NJ; ++j) {
                acc[i][j] = M::multiply(p[i], q[j], acc[i][j]);
                more(i * TL::NJ + j);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (i == 0) before();
            read_p(ns, nc, i);
#pragma unroll
            for (int j = 0; j < TL::NJ; ++j)
                if (min(j, TL::NI - 1) == i) nq[j] = read_q(ns, nc, j);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const auto nothing = [] {};
    const auto no_more = [](int) {};
    if (steps) {
#pragma unroll 1
        for (uint32_t d = 0; d < DEEP; ++d) issue(d);
        if (steps >= DEEP)
            load_wait<(DEEP - 1) * kLoads>();
        else
            load_wait<0>();
#pragma unroll
        for (int i = 0; i < TL::NI; ++i) read_p(0, 0, i);
#pragma unroll
        for (int j = 0; j < TL::NJ; ++j) qa[j] = read_q(0, 0, j);
    }
    uint32_t s = 0;
    for (; s + DEEP < whole; ++s) {
        group(s, 1, qb, qa, nothing, no_more);
        const char* from_p = (const char*)fp.base + (s + DEEP) * fp.per_step;
        const char* from_q = (const char*)fq.base + (s + DEEP) * fq.per_step;
        const uint32_t to = lds_at + s % DEEP * TL::kStage;
        // the loads are spread over the group: side by side they would hold up its reads of LDS
        group(s + 1, 0, qa, qb, [] { load_wait<(DEEP - 2) * kLoads>(); }, [&](int m) {
            constexpr int kRoom = TL::NI * TL::NJ - TL::NJ;
#pragma unroll
            for (int d = 0; d < kLoads; ++d) {
                if (TL::NJ + d * kRoom / kLoads != m) continue;
                if (d < FP::N)
                    fetch(from_p, fp.off[d], to + (d * (TL::kThreads / kWave) + wave) * kWave * 16);
                else
                    fetch(from_q, fq.off[d - FP::N],
                          to + FP::kBytes + ((d - FP::N) * (TL::kThreads / kWave) + wave) * kWave * 16);
            }
        });
    }
#pragma unroll 1
    for (; s < steps; ++s) {
        group(s, 1, qb, qa, nothing, no_more);
#pragma unroll
        for (int i = 0; i < TL::NI; ++i)
#pragma unroll
            for (int j = 0; j < TL::NJ; ++j) acc[i][j] = M::multiply(p[i], qb[j], acc[i][j]);
        if (s + 1 < steps) {
            load_wait<0>();
            issue(s + DEEP);
#pragma unroll
            for (int i = 0; i < TL::NI; ++i) read_p(s + 1, 0, i);
#pragma unroll
            for (int j = 0; j < TL::NJ; ++j) qa[j] = read_q(s + 1, 0, j);
        }
    }
    __syncthreads();
    store_tile<E, O, TL, PAIR>(a, acc, lds, i0, j0, split);
}

template <typename E, typename O, bool PA, bool QA, typename TL, bool PAIR = false>
__global__ __launch_bounds__(TL::kThreads) void k_gemm_fetch(GemmArgs a) {
    __shared__ __align__(1024) char lds[TL::DEEP * TL::kStage];
    gemm_fetch<E, O, PA, QA, TL, PAIR>(a, blockIdx.x, blockIdx.y, lds);
}

// The two products of a small layer's backward pass in one launch: blocks
// below `first` take the input's gradient, the others the weight's.
template <typename E, bool DIRECT>
__global__ __launch_bounds__(TileSmall::kThreads, DIRECT ? 1 : 2) void k_gemm_pair(GemmArgs dx, GemmArgs dw, uint32_t first) {
    __shared__ __align__(1024) char lds[DIRECT ? TileSmall::DEEP * TileSmall::kStage : TileSmall::kLds];
    const bool is_dx = blockIdx.x < first;
    if constexpr (DIRECT) {
        if (is_dx)
            gemm_fetch<E, E, true, false, TileSmall>(dx, blockIdx.x, 0, lds);
        else
            gemm_fetch<E, float, true, true, TileSmall>(dw, blockIdx.x - first, 0, lds);
    } else {
        if (is_dx)
            gemm_staged<E, E, true, false, TileSmall>(dx, blockIdx.x, 0, lds);
        else
            gemm_staged<E, float, true, true, TileSmall>(dw, blockIdx.x - first, 0, lds);
    }
}

// Joins the splits' sums, four results a thread.
template <typename E, typename O, bool PAIR = false>
__global__ __launch_bounds__(kBlock) void k_join(GemmArgs a, uint32_t splits) {
    const uint32_t per_row = (a.I + 3) / 4;
    const uint64_t all = (uint64_t)per_row * a.J, wide = PAIR ? 2ull * a.I : a.I;
    for (uint64_t t = (uint64_t)blockIdx.x * kBlock + threadIdx.x; t < all; t += (uint64_t)gridDim.x * kBlock) {
        const uint64_t j = t / per_row;
        const uint32_t i = (uint32_t)(t - j * per_row) * 4;
        const int n = (int)min(a.I - i, 4u);
        const auto join = [&](const float* p, float (&s)[4]) {
            if constexpr (sizeof(E) == 1) {
                int v[4] = {0, 0, 0, 0};
                for (uint32_t k = 0; k < splits; ++k) {
                    const Pack<float, 4> x = load_some<4>(p + (uint64_t)k * a.J * wide, n);
#pragma unroll
                    for (int c = 0; c < 4; ++c) v[c] += bits_as<int>(x.v[c]);
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) s[c] = (float)v[c];
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c) s[c] = 0.0f;
#pragma unroll 4
                for (uint32_t k = 0; k < splits; ++k) {
                    const Pack<float, 4> x = load_some<4>(p + (uint64_t)k * a.J * wide, n);
#pragma unroll
                    for (int c = 0; c < 4; ++c) s[c] += x.v[c];
                }
            }
        };
        const float* p = a.part + j * wide + i;
        float s[4];
        join(p, s);
        if constexpr (PAIR) {
            float u[4];
            join(p + a.I, u);
            finish_pair<O, 4>(a.fin, PairColumns<O, 4>(a.fin, i, a.I, n), j, i, a.I, s, u, n);
        } else {
            finish<O, 4>(a.fin, Columns<O, 4>(a.fin, i, n), j, i, s, n);
        }
    }
}

// At most 16 rows of Q (single tokens): a block takes 16 rows of P, its eight
// waves a share of k each, straight from memory, and joins their sums.  Bound
// by reading P once.
constexpr int kThinRows = 16, kThinWaves = 8, kThinDeep = 8;
template <typename E, typename O, bool PAIR = false>
__global__ __launch_bounds__(kThinWaves* kWave) void k_thin(GemmArgs a) {
    using M = Mma<E>;
    constexpr int H = PAIR ? 2 : 1;  // rows of P of a result
    __shared__ f4 lds[H][kThinWaves][kWave];
    constexpr uint32_t CE = 16 / sizeof(E), KE = 4 * CE;  // k of one instruction
    const uint32_t wave = wave_index(), lane = lane_id();
    const uint32_t i0 = blockIdx.x * kThinRows;
    const E* p = (const E*)a.p + (uint64_t)min(i0 + lane % 16, a.I - 1) * a.p_stride + lane / 16 * CE;
    const E* q = (const E*)a.q + (uint64_t)min(lane % 16, a.J - 1) * a.q_stride + lane / 16 * CE;
    const uint64_t apart = (uint64_t)a.I * a.p_stride;
    const uint32_t whole = a.K / KE, share = (whole + kThinWaves - 1) / kThinWaves;
    uint32_t s = min(wave * share, whole);
    const uint32_t end = min(s + share, whole);
    typename M::Sum acc[H];
#pragma unroll
    for (int h = 0; h < H; ++h) acc[h] = typename M::Sum{0, 0, 0, 0};
    for (; s + kThinDeep <= end; s += kThinDeep) {
        u4 x[H][kThinDeep], y[kThinDeep];
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int d = 0; d < kThinDeep; ++d) x[h][d] = bits_as<u4>(load_pack<CE>(p + h * apart + (uint64_t)(s + d) * KE));
#pragma unroll
        for (int d = 0; d < kThinDeep; ++d) y[d] = bits_as<u4>(load_pack<CE>(q + (uint64_t)(s + d) * KE));
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int d = 0; d < kThinDeep; ++d) acc[h] = M::multiply(x[h][d], y[d], acc[h]);
    }
    for (; s < end; ++s) {
        const u4 y = bits_as<u4>(load_pack<CE>(q + (uint64_t)s * KE));
#pragma unroll
        for (int h = 0; h < H; ++h)
            acc[h] = M::multiply(bits_as<u4>(load_pack<CE>(p + h * apart + (uint64_t)s * KE)), y, acc[h]);
    }
    if (wave == kThinWaves - 1 && whole * KE < a.K) {  // what is left of k
        const int have = (int)(a.K - whole * KE) - (int)(lane / 16 * CE);
        const u4 y = bits_as<u4>(load_some<CE>(q + (uint64_t)whole * KE, have));
#pragma unroll
        for (int h = 0; h < H; ++h)
            acc[h] = M::multiply(bits_as<u4>(load_some<CE>(p + h * apart + (uint64_t)whole * KE, have)), y, acc[h]);
    }
#pragma unroll
    for (int h = 0; h < H; ++h) lds[h][wave][lane] = bits_as<f4>(acc[h]);
    __syncthreads();
    if (wave != 0) return;
    const uint32_t i = i0 + lane / 16 * 4, j = lane % 16;
    if (i >= a.I || j >= a.J) return;
    const auto join = [&](int h, float (&v)[4]) {
        if constexpr (sizeof(E) == 1) {
            int t[4] = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < kThinWaves; ++w)
#pragma unroll
                for (int c = 0; c < 4; ++c) t[c] += bits_as<int>(lds[h][w][lane][c]);
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = (float)t[c];
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = 0.0f;
#pragma unroll
            for (int w = 0; w < kThinWaves; ++w)
#pragma unroll
                for (int c = 0; c < 4; ++c) v[c] += lds[h][w][lane][c];
        }
    };
    const int n = (int)min(a.I - i, 4u);
    float v[4];
    join(0, v);
    if constexpr (PAIR) {
        float u[4];
        join(1, u);
        finish_pair<O, 4>(a.fin, PairColumns<O, 4>(a.fin, i, a.I, n), j, i, a.I, v, u, n);
    } else {
        finish<O, 4>(a.fin, Columns<O, 4>(a.fin, i, n), j, i, v, n);
    }
}

// Limits and scratch of the layers that take these products.
constexpr uint64_t kLinearRoom = 8ull << 20;  // floats of partial sums of a product
constexpr uint32_t kLinearMaxDim = 1u << 22, kLinearMaxInt8 = 1u << 17;
constexpr uint64_t kLinearPad = 512ull << 20; // bytes of padded copies, at most
constexpr uint32_t kBiasParts = 256;          // partial sums of the bias's gradient

// Which operands lie across k.
enum GemmForm { kAlong = 0, kPAcross = 1, kBothAcross = 2 };

// Scratch of a product: `floats` for sums where k is split (at GemmArgs::part),
// and room for padded copies of operands (none: null).
struct GemmRoom {
    uint64_t floats;
    char* pad;
    uint64_t pad_bytes;
};

// Whether a product of I x J results is one that can be launched: a dispatch
// holds less than 2^32 threads, and the middle tile serves every form.
constexpr uint32_t kProductTile = 128, kProductThreads = 256;
inline bool product_fits(uint64_t I, uint64_t J) {
    return ((I + kProductTile - 1) / kProductTile) * ((J + kProductTile - 1) / kProductTile) * kProductThreads <= 0xFFFFFFFFull;
}

// One product that fits.  Operand types: E is O's type, or int8 with kAlong.
template <typename E, typename O, int FORM>
hipError_t launch_gemm(GemmArgs a, const GemmRoom& room, hipStream_t st);

// One product of a gated layer, both operands along k: I results of 2 I rows of P, whose product_fits.
template <typename E, typename O>
hipError_t launch_gated(const GemmArgs& a, const GemmRoom& room, hipStream_t st);

// The products of a layer's backward pass in its type T, each where it is given.
template <typename T>
hipError_t launch_backward(const GemmArgs* dx, const GemmArgs* dw, const GemmRoom& room, hipStream_t st);

}  // namespace gd
