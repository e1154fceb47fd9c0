#include "quant_attn_kernel.cuh"

namespace wise {
cudaError_t launch_quant_attn_d96(const QaLaunch& L) { return launch_quant_attn_for_dim<96>(L); }
}  // namespace wise
