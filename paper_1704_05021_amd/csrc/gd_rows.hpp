// Shapes of the kernels that take whole rows: norms, and rows in 8 bits.
#pragma once

#include <type_traits>

#include "gd.h"
#include "gd_ops.hpp"

namespace gd {

template <int WAVES>
struct NormShape {
    static constexpr int kThreads = WAVES * kWave < kBlock ? kBlock : WAVES * kWave;
    static constexpr int kRow = WAVES * kWave;          // threads of a row
    static constexpr int kRows = kThreads / kRow;       // rows of a block
};

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
