// The cache behind the compression: checks of a call, and its workspace.
#include <cmath>

#include "cache_internal.h"

namespace tc {

int make_cache_plan(const tc_cache* c, CachePlan* plan) {
  if (!c) return TC_ERR_NULL;
  if (!known_dtype(c->dtype)) return TC_ERR_DTYPE;
  if (c->batch < 0 || c->batch > (1 << 16) || c->n_heads < 1 || c->n_heads > 1024 || c->n_kv_heads < 1 || c->n_heads % c->n_kv_heads != 0 ||
      (c->head_dim != 64 && c->head_dim != 128) || c->n_query < 1 || c->n_query > (1 << 20) || c->capacity < 1 || c->capacity > (1 << 24) ||
      c->max_len < 0 || c->max_len > c->capacity || c->n_prefixes < 0 || c->prefix_len < 0 || c->prefix_len > (1 << 24) ||
      (c->n_prefixes > 0 ? c->batch % c->n_prefixes != 0 : c->prefix_len > 0))
    return TC_ERR_SHAPE;
  if (!(c->softmax_scale >= 0.f) || !std::isfinite(c->softmax_scale) || c->budget < 0 || c->budget > c->capacity || c->n_sink < 0 ||
      c->n_recent < 0 || (c->budget > 0 && (int64_t)c->n_sink + c->n_recent > c->budget))
    return TC_ERR_PARAM;
  CachePlan& q = *plan;
  q.B = c->batch; q.H = c->n_heads; q.Hk = c->n_kv_heads; q.G = q.H / q.Hk; q.dh = c->head_dim; q.T = c->n_query;
  q.cap = c->capacity; q.max_len = c->max_len > 0 ? c->max_len : c->capacity;
  q.images = c->prefix_len > 0 ? c->n_prefixes : 0; q.each = q.images > 0 ? q.B / q.images : 0; q.P = c->prefix_len;
  q.esize = elem_size(c->dtype);
  q.R = q.G * q.T;
  q.scale = c->softmax_scale > 0.f ? c->softmax_scale : 1.0f / std::sqrt((float)q.dh);
  if ((long long)q.B * q.H * q.T > (1LL << 31) - 1) return TC_ERR_SHAPE;  // rows are counted in 32 bits
  q.budget = c->budget; q.sink = c->n_sink; q.recent = c->n_recent;
  const size_t a = attention_bytes(q), e = evict_bytes(q);
  q.total = align256((a > e ? a : e) + 256);
  return TC_OK;
}

}  // namespace tc

using namespace tc;

extern "C" size_t tc_cache_workspace_bytes(const tc_cache* c) {
  CachePlan pl;
  return make_cache_plan(c, &pl) == TC_OK ? pl.total : 0;
}
