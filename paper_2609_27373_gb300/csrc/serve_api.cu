// Host side of the serving calls declared in include/wise.h: argument checks
// and launches of the paged cache's operations, the attention over it and the
// verification of drafted tokens.
#include <math.h>
#include <string.h>

#include "internal.cuh"
#include "prefix_attn.cuh"
#include "wise.h"

namespace wise {
namespace {

constexpr int kMaxVocab = 1 << 18; // weights of 2^40 at most add up within 2^58
constexpr int kMaxDraft = 1024;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
bool ok32(const void* p) { return p && aligned(p, 4); }

// The checks that need no device; `pool` says whether the call touches pages.
int check_cache(const wise_cache_t* c, bool pool, CacheView* v) {
  if (!c) return WISE_ERR_INVALID_ARG;
  if (c->n_pages <= 0 || c->n_slots <= 0 || c->max_pages <= 0 || c->n_layers <= 0 || c->n_kv_heads <= 0 ||
      c->page <= 0 || c->head_dim <= 0)
    return WISE_ERR_INVALID_ARG;
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return WISE_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128) return WISE_ERR_UNSUPPORTED;
  if (c->dtype != WISE_BF16 && c->dtype != WISE_FP16) return WISE_ERR_UNSUPPORTED;
  if (c->n_slots > kMaxSlots || (long long)c->max_pages * c->page > (1LL << 30) ||
      (long long)c->n_pages * c->n_kv_heads > INT32_MAX || c->n_pages >= (1 << 30) - 1 || c->n_kv_heads > (1 << 14) || c->n_layers > (1 << 20))
    return WISE_ERR_UNSUPPORTED;
  if (!ok32(c->table) || !ok32(c->lens) || !ok32(c->refs)) return WISE_ERR_INVALID_ARG;
  if (pool && (!c->pool || !aligned(c->pool, 16))) return WISE_ERR_INVALID_ARG;
  v->n_pages = c->n_pages;
  v->page = c->page;
  v->page_shift = c->page == 16 ? 4 : c->page == 32 ? 5 : c->page == 64 ? 6 : 7;
  v->n_slots = c->n_slots;
  v->max_pages = c->max_pages;
  v->n_planes = 2 * c->n_layers;
  v->row_bytes = c->head_dim * 2;
  v->head_bytes = v->row_bytes * c->page;
  v->page_bytes = v->head_bytes * c->n_kv_heads;
  v->plane_bytes = (long long)v->page_bytes * c->n_pages;
  v->n_kv_heads = c->n_kv_heads;
  v->pool = reinterpret_cast<uint8_t*>(c->pool);
  v->table = c->table;
  v->lens = c->lens;
  v->refs = c->refs;
  v->max_len = c->max_pages * c->page;
  return WISE_OK;
}

int result(cudaError_t e) { return e == cudaSuccess ? WISE_OK : WISE_ERR_CUDA; }

// Shape checks of the attention (everything but the device pointers).
int check_prefix(const wise_cache_t* cache, const wise_prefix_t* sh, PrefixParams* p) {
  int rc = check_cache(cache, true, &p->cache);
  if (rc != WISE_OK) return rc;
  if (!sh || sh->batch < 0 || sh->q_len < 0 || sh->n_heads <= 0 || sh->n_groups < 0 || !(sh->scale >= 0.0f) ||
      isinf(sh->scale))
    return WISE_ERR_INVALID_ARG;
  if (sh->n_heads % cache->n_kv_heads != 0) return WISE_ERR_UNSUPPORTED;
  const int group = sh->n_heads / cache->n_kv_heads;
  if (sh->batch > kPfxMaxBatch || (long long)sh->q_len * group > kPfxRows || sh->n_groups > sh->batch ||
      sh->n_groups > kPfxMaxGroups)
    return WISE_ERR_UNSUPPORTED;
  // Key tiles of all requests and kv heads are counted in 32 bits.
  const long long max_tiles = ((long long)cache->max_pages * cache->page + kPfxKeys - 1) / kPfxKeys;
  if ((long long)sh->batch * cache->n_kv_heads * (max_tiles + 1) > (1LL << 30)) return WISE_ERR_UNSUPPORTED;
  p->batch = sh->batch;
  p->q_len = sh->q_len;
  p->n_heads = sh->n_heads;
  p->group = group;
  p->n_groups = sh->n_groups;
  p->head_dim = cache->head_dim;
  p->fp16 = cache->dtype == WISE_FP16;
  const float scale = sh->scale > 0.0f ? sh->scale : 1.0f / sqrtf((float)cache->head_dim);
  p->scale_log2 = scale * 1.4426950408889634f;
  return WISE_OK;
}

}  // namespace
}  // namespace wise

using namespace wise;

extern "C" int wise_kv_fork(const wise_cache_t* cache, const int32_t* src, const int32_t* dst, int n,
                            cudaStream_t stream) {
  CacheView v;
  int rc = check_cache(cache, false, &v);
  if (rc != WISE_OK) return rc;
  if (n < 0) return WISE_ERR_INVALID_ARG;
  if (n == 0) return WISE_OK;
  if (n > kMaxSlots) return WISE_ERR_UNSUPPORTED;
  if (!ok32(src) || !ok32(dst)) return WISE_ERR_INVALID_ARG;
  int sms;
  if ((rc = current_device(&sms, &v.status)) != WISE_OK) return rc;
  return result(launch_kv_fork(v, src, dst, n, stream));
}

extern "C" size_t wise_kv_workspace(const wise_cache_t* cache, int n) {
  CacheView v;
  if (check_cache(cache, false, &v) != WISE_OK || n < 0) return 0;
  // A few counters; extend: the free pages it may take, the need of each entry
  // and three words per copied page; compact: two lists of pages.
  return (size_t)4 * (2 * (size_t)v.n_pages + 4 * (size_t)n + 4);
}

extern "C" int wise_kv_extend(const wise_cache_t* cache, const int32_t* slots, const int32_t* n_new, int n,
                              int32_t* granted, void* workspace, cudaStream_t stream) {
  CacheView v;
  int rc = check_cache(cache, true, &v);
  if (rc != WISE_OK) return rc;
  if (n < 0) return WISE_ERR_INVALID_ARG;
  if (n == 0) return WISE_OK;
  if (n > kMaxSlots) return WISE_ERR_UNSUPPORTED;
  if (!ok32(slots) || !ok32(n_new) || !ok32(granted) || !workspace || !aligned(workspace, 16))
    return WISE_ERR_INVALID_ARG;
  int sms;
  if ((rc = current_device(&sms, &v.status)) != WISE_OK) return rc;
  return result(
      launch_kv_extend(v, slots, n_new, n, granted, reinterpret_cast<int32_t*>(workspace), sms, stream));
}

extern "C" int wise_kv_write(const wise_cache_t* cache, int layer, const int32_t* slots, const int32_t* n_new,
                             int batch, int q_len, const void* K, const void* V, cudaStream_t stream) {
  CacheView v;
  int rc = check_cache(cache, true, &v);
  if (rc != WISE_OK) return rc;
  if (layer < 0 || layer >= cache->n_layers || batch < 0 || q_len < 0) return WISE_ERR_INVALID_ARG;
  if (batch == 0 || q_len == 0) return WISE_OK;
  if (batch > kMaxSlots || (long long)batch * q_len > (1LL << 30) / cache->n_kv_heads) return WISE_ERR_UNSUPPORTED;
  if (!ok32(slots) || !aligned(n_new, 4) || !K || !V || !aligned(K, 16) || !aligned(V, 16))
    return WISE_ERR_INVALID_ARG;
  int sms;
  if ((rc = current_device(&sms, &v.status)) != WISE_OK) return rc;
  return result(launch_kv_write(v, layer, slots, n_new, batch, q_len, K, V, sms, stream));
}

extern "C" int wise_kv_drop(const wise_cache_t* cache, const int32_t* slots, const int32_t* n_drop, int n,
                            cudaStream_t stream) {
  CacheView v;
  int rc = check_cache(cache, false, &v);
  if (rc != WISE_OK) return rc;
  if (n < 0) return WISE_ERR_INVALID_ARG;
  if (n == 0) return WISE_OK;
  if (n > kMaxSlots) return WISE_ERR_UNSUPPORTED;
  if (!ok32(slots) || !ok32(n_drop)) return WISE_ERR_INVALID_ARG;
  int sms;
  if ((rc = current_device(&sms, &v.status)) != WISE_OK) return rc;
  return result(launch_kv_drop(v, slots, n_drop, n, stream));
}

extern "C" int wise_kv_compact(const wise_cache_t* cache, int32_t* remap, int32_t* n_live, void* workspace,
                               cudaStream_t stream) {
  CacheView v;
  int rc = check_cache(cache, true, &v);
  if (rc != WISE_OK) return rc;
  if (!ok32(remap) || !ok32(n_live) || !workspace || !aligned(workspace, 16)) return WISE_ERR_INVALID_ARG;
  int sms;
  if ((rc = current_device(&sms, &v.status)) != WISE_OK) return rc;
  return result(launch_kv_compact(v, remap, n_live, reinterpret_cast<int32_t*>(workspace), sms, stream));
}

extern "C" size_t wise_prefix_attn_workspace(const wise_cache_t* cache, const wise_prefix_t* shape) {
  PrefixParams p;
  if (check_prefix(cache, shape, &p) != WISE_OK || p.batch == 0 || p.q_len == 0) return 0;
  int sms;
  int* status;
  if (current_device(&sms, &status) != WISE_OK) return 0;
  return prefix_attn_workspace(p, sms);
}

extern "C" int wise_prefix_attn(const wise_cache_t* cache, int layer, const wise_prefix_t* shape, const void* Q,
                                const int32_t* slots, const int32_t* n_new, const int32_t* group_start,
                                const int32_t* prefix_lens, void* O, void* workspace, size_t workspace_bytes,
                                cudaStream_t stream) {
  PrefixParams p;
  int rc = check_prefix(cache, shape, &p);
  if (rc != WISE_OK) return rc;
  if (layer < 0 || layer >= cache->n_layers) return WISE_ERR_INVALID_ARG;
  if (p.batch == 0 || p.q_len == 0) return WISE_OK;
  if (!Q || !O || !aligned(Q, 16) || !aligned(O, 16) || !ok32(slots) || !aligned(n_new, 4))
    return WISE_ERR_INVALID_ARG;
  if (p.n_groups > 0 && (!ok32(group_start) || !ok32(prefix_lens))) return WISE_ERR_INVALID_ARG;
  int sms;
  if ((rc = current_device(&sms, &p.cache.status)) != WISE_OK) return rc;
  const size_t need = prefix_attn_workspace(p, sms);
  if (workspace_bytes < need || (need > 0 && (!workspace || !aligned(workspace, 16)))) return WISE_ERR_INVALID_ARG;
  p.layer = layer;
  p.Q = Q;
  p.O = O;
  p.slots = slots;
  p.n_new = n_new;
  p.group_start = group_start;
  p.prefix_lens = prefix_lens;
  return launch_prefix_attn(p, workspace, sms, stream);
}

extern "C" int wise_verify_draft(int batch, int k_max, int vocab, int dtype, const void* p, const void* q,
                                 const int32_t* draft, const int32_t* n_draft, const float* u_accept,
                                 const float* u_sample, int32_t* accepted, int32_t* tokens, cudaStream_t stream) {
  if (batch < 0 || k_max < 0 || vocab <= 0) return WISE_ERR_INVALID_ARG;
  if (dtype != WISE_BF16 && dtype != WISE_FP16 && dtype != WISE_FP32) return WISE_ERR_UNSUPPORTED;
  if (batch > kMaxSlots || k_max > kMaxDraft || vocab > kMaxVocab) return WISE_ERR_UNSUPPORTED;
  if (batch == 0) return WISE_OK;
  const size_t size = dtype == WISE_FP32 ? 4 : 2;
  if (!p || !aligned(p, size) || !ok32(u_sample) || !ok32(accepted) || !ok32(tokens) || !aligned(n_draft, 4))
    return WISE_ERR_INVALID_ARG;
  if (k_max > 0 && (!q || !aligned(q, size) || !ok32(draft) || !ok32(u_accept))) return WISE_ERR_INVALID_ARG;
  VerifyParams vp;
  int rc;
  if ((rc = current_device(&vp.sm_count, &vp.status)) != WISE_OK) return rc;
  vp.batch = batch;
  vp.k_max = k_max;
  vp.vocab = vocab;
  vp.p = p;
  vp.q = q;
  vp.draft = draft;
  vp.n_draft = n_draft;
  vp.u_accept = u_accept;
  vp.u_sample = u_sample;
  vp.accepted = accepted;
  vp.tokens = tokens;
  return result(launch_verify_draft(dtype, vp, stream));
}
