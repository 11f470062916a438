// The matrix products of layers in bf16.
#include <algorithm>

#include "gd_gemm_launch.hpp"

namespace gd {
template hipError_t launch_gemm<bf16, bf16, kAlong>(GemmArgs, const GemmRoom&, hipStream_t);
template hipError_t launch_backward<bf16>(const GemmArgs*, const GemmArgs*, const GemmRoom&, hipStream_t);
template hipError_t launch_gemm<int8_t, bf16, kAlong>(GemmArgs, const GemmRoom&, hipStream_t);
}  // namespace gd
