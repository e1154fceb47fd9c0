// Host side of the attention over a paged cache of 8 or 4 bits: workspace and
// the choice of the kernel instance.
#include "quant_attn.cuh"

namespace wise {

size_t quant_attn_workspace(const PrefixParams& p, int sm_count) {
  return qa_work(nullptr, p.batch, p.n_groups, p.cache.n_kv_heads, p.q_len * p.group, p.head_dim, sm_count).bytes;
}

int launch_quant_attn(const PrefixParams& p, void* workspace, int sm_count, cudaStream_t stream) {
  const CacheView& c = p.cache;
  QaLaunch L;
  L.p.cache = c;
  L.p.plane = c.pool + (long long)p.layer * c.plane_bytes;
  L.p.batch = p.batch;
  L.p.q_len = p.q_len;
  L.p.n_groups = p.n_groups;
  L.p.rows = p.q_len * p.group;
  L.p.rows_inv = 65536 / L.p.rows + 1;
  L.p.q_len_inv = 65536 / p.q_len + 1;
  L.p.chunks = (L.p.rows + kQaRows - 1) / kQaRows;
  L.p.per_tile = p.n_groups > 0 && L.p.rows * 2 <= kQaRows ? kQaRows / L.p.rows : 0;
  L.p.fp16 = p.fp16;
  L.p.scale_log2 = p.scale_log2;
  L.p.Q = p.Q;
  L.p.O = p.O;
  L.p.slots = p.slots;
  L.p.n_new = p.n_new;
  L.p.group_start = p.group_start;
  L.p.prefix_lens = p.prefix_lens;
  L.p.work = qa_work(workspace, p.batch, p.n_groups, c.n_kv_heads, L.p.rows, p.head_dim, sm_count);
  L.p.wait_ns = wait_limit_ns();
  L.grid = sm_count;
  // The wide instance takes 64 rows at a time, the narrow one half a step's time
  // for at most 16 (32 x 12K tokens, 4 rows: 105 us against 145; 16 x 4K in 8
  // bits 103 against 127).  Sharing prefixes needs the wide one: 64 on a shared
  // 32K prefix take 116 us in it, 501 each by itself in the narrow one.
  L.wide = L.p.rows > 16 || L.p.per_tile > 0;
  L.stream = stream;
  cudaError_t e;
  switch (p.head_dim) {
    case 64: e = launch_quant_attn_d64(L); break;
    case 96: e = launch_quant_attn_d96(L); break;
    default: e = launch_quant_attn_d128(L); break;
  }
  return e == cudaSuccess ? WISE_OK : WISE_ERR_CUDA;
}

}  // namespace wise
