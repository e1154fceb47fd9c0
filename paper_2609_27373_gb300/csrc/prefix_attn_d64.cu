#include "prefix_kernel.cuh"

namespace wise {
cudaError_t launch_prefix_d64(bool fp16, const PfxLaunch& L) { return launch_prefix_for_dim<64>(fp16, L); }
}  // namespace wise
