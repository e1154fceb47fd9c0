#include "prefix_kernel.cuh"

namespace wise {
cudaError_t launch_prefix_d128(bool fp16, const PfxLaunch& L) { return launch_prefix_for_dim<128>(fp16, L); }
}  // namespace wise
