// Device-side building blocks of the operators around the compressor: element
// types, loads and stores at element alignment, reductions over a row.
#pragma once

#include "gd_device.hpp"

namespace gd {

typedef __bf16 bf16;
typedef _Float16 f16;

// N consecutive elements at p, which is aligned to one element only: one
// memory instruction per 16 bytes (the hardware takes any address).
template <typename T, int N>
struct Pack {
    T v[N];
};
template <int N, typename T>
__device__ __forceinline__ Pack<T, N> load_pack(const T* p) {
    Pack<T, N> r;
    __builtin_memcpy(&r, p, sizeof r);
    return r;
}
template <int N, typename T>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, N>& r) {
    __builtin_memcpy(p, &r, sizeof r);
}
// The first `n` of them (0 for the others), where fewer than N are there.
template <int N, typename T>
__device__ __forceinline__ Pack<T, N> load_some(const T* p, int n) {
    if (n >= N) return load_pack<N>(p);
    Pack<T, N> r;
#pragma unroll
    for (int i = 0; i < N; ++i) r.v[i] = i < n ? p[i] : (T)0.0f;
    return r;
}
template <int N, typename T>
__device__ __forceinline__ void store_some(T* p, const Pack<T, N>& r, int n) {
    if (n >= N) {
        store_pack<N>(p, r);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < n) p[i] = r.v[i];
}

// store_some for results that nothing reads back soon.
template <int N, typename T>
__device__ __forceinline__ void store_stream(T* p, const Pack<T, N>& r, int n) {
    if (n < N) {
        store_some<N>(p, r, n);
        return;
    }
    typedef uint32_t words __attribute__((ext_vector_type(4), aligned(2)));
    static_assert(sizeof(r) % 16 == 0 && alignof(T) >= 2);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(r) / 16); ++i) {
        words v;
        __builtin_memcpy(&v, (const char*)&r + i * 16, 16);
        __builtin_nontemporal_store(v, (words*)p + i);
    }
}

// Sum over the threads of one row: WAVES consecutive waves of the block, in a
// fixed order, in every thread.  lds holds one double per wave of the block;
// every thread of the block calls it, with a barrier after the last use of
// lds by an earlier call.
template <int WAVES>
__device__ __forceinline__ double row_sum(double v, double* lds) {
    v = wave_sum(v);
    if constexpr (WAVES > 1) {
        const uint32_t w = wave_index();
        if (lane_id() == 0) lds[w] = v;
        __syncthreads();
        v = 0.0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) v += lds[w / WAVES * WAVES + i];
    }
    return v;
}

// Two such sums behind one barrier.
template <int WAVES>
__device__ __forceinline__ void row_sums(double& a, double& b, double* lds_a, double* lds_b) {
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (WAVES > 1) {
        const uint32_t w = wave_index();
        if (lane_id() == 0) lds_a[w] = a, lds_b[w] = b;
        __syncthreads();
        a = b = 0.0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) a += lds_a[w / WAVES * WAVES + i], b += lds_b[w / WAVES * WAVES + i];
    }
}

// Up to four such sums behind one barrier, each wave's shares joined by 16 lanes a sum (all of them read by every
// thread would take 64 registers for four sums of eight waves).
template <int WAVES, int N, int LDS>
__device__ __forceinline__ void row_sums(double (&v)[N], double (&lds)[N][LDS]) {
    static_assert(N <= 4 && WAVES <= 16);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = wave_sum(v[k]);
    if constexpr (WAVES > 1) {
        const uint32_t w = wave_index(), k = lane_id() / 16, from = lane_id() % 16;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (lane_id() == 0) lds[i][w] = v[i];
        __syncthreads();
        double s = -0.0;
        if (k < (uint32_t)N && from < (uint32_t)WAVES) s = lds[k][w / WAVES * WAVES + from];
        s += dpp_f64<0x111, 0xF>(s);  // row_shr:1
        s += dpp_f64<0x112, 0xF>(s);  // row_shr:2
        s += dpp_f64<0x114, 0xF>(s);  // row_shr:4
        s += dpp_f64<0x118, 0xF>(s);  // row_shr:8
        const uint64_t bits = (uint64_t)__double_as_longlong(s);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t lo = lane_value((uint32_t)bits, i * 16 + 15), hi = lane_value((uint32_t)(bits >> 32), i * 16 + 15);
            v[i] = __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
        }
    }
}

// Largest of unsigned words over the threads of one row, likewise.
template <int WAVES>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t* lds) {
    v = lane_value(wave_incl_max(v), kWave - 1);
    if constexpr (WAVES > 1) {
        const uint32_t w = wave_index();
        if (lane_id() == 0) lds[w] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) v = max(v, lds[w / WAVES * WAVES + i]);
    }
    return v;
}

// Scale and step of a row stored in 8 bits, from its largest magnitude's bit
// pattern (the order of the patterns puts infinities and NaN last, so the
// scale of a row that holds one is not finite).  The step is 127 times the
// rounded reciprocal, one rounding each: what 127.0 / max is in torch, so
// codes equal those of the elementary operations bit for bit.  (127 / max
// rounded once puts 1.4e-4 of a bfloat16 row's codes, halves of the largest
// magnitude most of them, on the other side of the middle.)  Rows below
// 2^-119, whose step would overflow, are stored as zeros.
struct RowScale {
    float scale, step;
};
__device__ __forceinline__ RowScale row_scale(uint32_t max_bits) {
    const float big = __uint_as_float(max_bits);
    return {big / 127.0f, big >= 0x1p-119f ? 127.0f * (1.0f / big) : 0.0f};
}
__device__ __forceinline__ int8_t quantise(float y, float step) {
    return (int8_t)fminf(fmaxf(rintf(y * step), -127.0f), 127.0f);  // a NaN gives -127, under a NaN scale
}

// out[c] (+)= sum over p of part[p][c], p < parts, in 64 bits and a fixed order.
hipError_t launch_sum_parts(const float* part, uint32_t parts, uint64_t columns, float* out, bool accumulate,
                            hipStream_t st);

}  // namespace gd
