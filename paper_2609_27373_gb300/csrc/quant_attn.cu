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
  // bits 103 against 127).  Prefix items need the wide one, and both lines of the
  // plan are walked in one launch, so own items run there too as soon as groups are
  // given: what is shared is known on the device alone.  With 4 rows a request and
  // 4 bits (us with groups, without): 64 requests of about 256 tokens behind 512
  // shared ones 51, 33, behind 2K 59, 51, behind 8K 65, 139, behind 32K 106, 496;
  // 32 of about 8K behind 40 (nothing is shared) 107, 82, behind 2K 116, 91, behind
  // 8K 126, 135; 4 of about 10K behind 8K 35, 30, behind 32K 43, 53.
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
