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

// a in the lower half of the lanes and b in the upper, each with what its other half holds added: two sums over 64 lanes
// become one over 32.
__device__ __forceinline__ double halves_joined(double a, double b) {
    const uint64_t x = (uint64_t)__double_as_longlong(a), y = (uint64_t)__double_as_longlong(b);
    const auto lo = __builtin_amdgcn_permlane32_swap((uint32_t)x, (uint32_t)y, false, false);
    const auto hi = __builtin_amdgcn_permlane32_swap((uint32_t)(x >> 32), (uint32_t)(y >> 32), false, false);
    return __longlong_as_double((long long)((uint64_t)hi[0] << 32 | lo[0])) +
           __longlong_as_double((long long)((uint64_t)hi[1] << 32 | lo[1]));
}
// The same by rows of 16 lanes: a in the even ones and b in the odd.
__device__ __forceinline__ double rows_joined(double a, double b) {
    const uint64_t x = (uint64_t)__double_as_longlong(a), y = (uint64_t)__double_as_longlong(b);
    const auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)y, false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(x >> 32), (uint32_t)(y >> 32), false, false);
    return __longlong_as_double((long long)((uint64_t)hi[0] << 32 | lo[0])) +
           __longlong_as_double((long long)((uint64_t)hi[1] << 32 | lo[1]));
}

// Two or four such sums behind one barrier.  The sums share the steps over a
// wave's lanes, which end with one sum to 16 or 32 of them (four sums one by
// one took a quarter of the layer norm's backward pass), and 16 lanes a sum join
// the waves' shares (read by every thread they would take 64 registers).
template <int WAVES, int N, int LDS>
__device__ __forceinline__ void row_sums(double (&v)[N], double (&lds)[N][LDS]) {
    static_assert((N == 2 || N == 4) && WAVES <= 16);
    double s = N == 2 ? halves_joined(v[0], v[1]) : rows_joined(halves_joined(v[0], v[N / 2]), halves_joined(v[1], v[N - 1]));
    s += dpp_f64<0x111, 0xF>(s);  // row_shr:1
    s += dpp_f64<0x112, 0xF>(s);  // row_shr:2
    s += dpp_f64<0x114, 0xF>(s);  // row_shr:4
    s += dpp_f64<0x118, 0xF>(s);  // row_shr:8
    if (N == 2) s += dpp_f64<0x142, 0xA>(s);  // row_bcast:15, rows 1 and 3
    constexpr int kSpan = kWave / N;          // sum i is in the last lane of the i-th span
    const auto spread = [&](double x, int span) {
        const uint64_t bits = (uint64_t)__double_as_longlong(x);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int from = (i + 1) * span - 1;
            const uint32_t lo = lane_value((uint32_t)bits, from), hi = lane_value((uint32_t)(bits >> 32), from);
            v[i] = __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
        }
    };
    if constexpr (WAVES == 1) {
        spread(s, kSpan);
    } else {
        const uint32_t w = wave_index(), lane = lane_id(), k = lane / 16, from = lane % 16;
        if (lane % kSpan == kSpan - 1) lds[lane / kSpan][w] = s;
        __syncthreads();
        s = -0.0;
        if (k < (uint32_t)N && from < (uint32_t)WAVES) s = lds[k][w / WAVES * WAVES + from];
        s += dpp_f64<0x111, 0xF>(s);
        s += dpp_f64<0x112, 0xF>(s);
        if (WAVES > 4) s += dpp_f64<0x114, 0xF>(s);
        if (WAVES > 8) s += dpp_f64<0x118, 0xF>(s);
        // the shares lie in the first WAVES lanes of 16; their sum is in the last of those
        const uint64_t bits = (uint64_t)__double_as_longlong(s);
        constexpr int kLast = WAVES > 8 ? 15 : WAVES > 4 ? 7 : 3;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t lo = lane_value((uint32_t)bits, i * 16 + kLast), hi = lane_value((uint32_t)(bits >> 32), i * 16 + kLast);
            v[i] = __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
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
