// Host side of the attention over the paged cache: workspace, tensor maps and
// the choice of the kernel instance.
#include "prefix_attn.cuh"

namespace wise {

size_t prefix_attn_workspace(const PrefixParams& p, int sm_count) {
  return pfx_work(nullptr, p.batch, p.n_groups, p.cache.n_kv_heads, p.q_len * p.group, p.head_dim, sm_count).bytes;
}

int launch_prefix_attn(const PrefixParams& p, void* workspace, int sm_count, cudaStream_t stream) {
  const CacheView& c = p.cache;
  PfxLaunch L;
  L.p.cache = c;
  L.p.batch = p.batch;
  L.p.q_len = p.q_len;
  L.p.n_heads = p.n_heads;
  L.p.group = p.group;
  L.p.n_groups = p.n_groups;
  L.p.rows = p.q_len * p.group;
  L.p.per_tile = kPfxRows / L.p.rows;
  L.p.scale_log2 = p.scale_log2;
  L.p.slots = p.slots;
  L.p.n_new = p.n_new;
  L.p.group_start = p.group_start;
  L.p.prefix_lens = p.prefix_lens;
  L.p.work = pfx_work(workspace, p.batch, p.n_groups, c.n_kv_heads, L.p.rows, p.head_dim, sm_count);
  L.p.wait_ns = wait_limit_ns();
  L.O = p.O;
  L.grid = sm_count;
  L.stream = stream;
  const uint8_t* keys = c.pool + 2 * (long long)p.layer * c.plane_bytes;
  const long long outer = (long long)c.n_pages * c.n_kv_heads;
  if (!make_tile_map(&L.mapK, keys, p.fp16, p.head_dim, c.page, outer, c.page) ||
      !make_tile_map(&L.mapV, keys + c.plane_bytes, p.fp16, p.head_dim, c.page, outer, c.page) ||
      !make_query_map(&L.mapQ, p.Q, p.fp16, p.head_dim, L.p.rows, c.n_kv_heads, p.batch, L.p.per_tile) ||
      !make_query_map(&L.mapQ1, p.Q, p.fp16, p.head_dim, L.p.rows, c.n_kv_heads, p.batch, 1))
    return WISE_ERR_CUDA;
  cudaError_t e;
  switch (p.head_dim) {
    case 64: e = launch_prefix_d64(p.fp16, L); break;
    case 96: e = launch_prefix_d96(p.fp16, L); break;
    default: e = launch_prefix_d128(p.fp16, L); break;
  }
  return e == cudaSuccess ? WISE_OK : WISE_ERR_CUDA;
}

}  // namespace wise
