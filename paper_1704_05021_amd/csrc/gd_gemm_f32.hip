// The matrix products of layers in f32.
#include <algorithm>

#include "gd_gemm_launch.hpp"

namespace gd {
template hipError_t launch_gemm<float, float, kAlong>(GemmArgs, const GemmRoom&, hipStream_t);
template hipError_t launch_backward<float>(const GemmArgs*, const GemmArgs*, const GemmRoom&, hipStream_t);
template hipError_t launch_gemm<int8_t, float, kAlong>(GemmArgs, const GemmRoom&, hipStream_t);
template hipError_t launch_gated<float, float>(const GemmArgs&, const GemmRoom&, hipStream_t);
template hipError_t launch_gated<int8_t, float>(const GemmArgs&, const GemmRoom&, hipStream_t);
}  // namespace gd
