// The matrix products of layers in f32.
#include <algorithm>

#include "gd_gemm_launch.hpp"

namespace gd {
template hipError_t launch_gemm<float, float, kAlong>(GemmArgs, uint64_t, hipStream_t);
template hipError_t launch_gemm<float, float, kPAcross>(GemmArgs, uint64_t, hipStream_t);
template hipError_t launch_gemm<float, float, kBothAcross>(GemmArgs, uint64_t, hipStream_t);
template hipError_t launch_gemm<int8_t, float, kAlong>(GemmArgs, uint64_t, hipStream_t);
}  // namespace gd
