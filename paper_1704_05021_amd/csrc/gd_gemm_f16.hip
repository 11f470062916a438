// The matrix products of layers in f16.
#include <algorithm>

#include "gd_gemm_launch.hpp"

namespace gd {
template hipError_t launch_gemm<f16, f16, kAlong>(GemmArgs, const GemmRoom&, hipStream_t);
template hipError_t launch_backward<f16>(const GemmArgs*, const GemmArgs*, const GemmRoom&, hipStream_t);
template hipError_t launch_gemm<int8_t, f16, kAlong>(GemmArgs, const GemmRoom&, hipStream_t);
template hipError_t launch_gated<f16, f16>(const GemmArgs&, const GemmRoom&, hipStream_t);
template hipError_t launch_gated<int8_t, f16>(const GemmArgs&, const GemmRoom&, hipStream_t);
}  // namespace gd
