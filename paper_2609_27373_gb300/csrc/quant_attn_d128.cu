#include "quant_attn_kernel.cuh"

namespace wise {
cudaError_t launch_quant_attn_d128(const QaLaunch& L) { return launch_quant_attn_for_dim<128>(L); }
}  // namespace wise
