// Geometry, layout and device view of a grouped-query cache, shared by the C
// entry points that take one (pask_api.cpp, pask_prompt_api.cpp).
#pragma once

#include "pask_host.h"

namespace pask {

inline bool valid_geom(const pask_geom* g) {
  if (!g) return false;
  if (g->max_batch < 1 || g->max_batch > 65535) return false;
  if (g->n_layers < 1 || g->n_layers > PASK_MAX_LAYERS) return false;
  if (g->n_kv_heads < 1 || g->n_kv_heads > 8 || g->n_q_heads < g->n_kv_heads) return false;
  if (g->n_q_heads % g->n_kv_heads != 0) return false;
  const int gs = g->n_q_heads / g->n_kv_heads;
  if (gs != 1 && gs != 2 && gs != 4 && gs != 8) return false;
  if (g->head_dim != 64 && g->head_dim != 128) return false;
  if (g->page_tokens != PASK_PAGE_TOKENS) return false;
  if (g->max_tokens_per_seq < 1 || g->max_tokens_per_seq > (1 << 28)) return false;
  if (g->hi_pages < 0 || g->lo_pages < 0) return false;
  if (g->recent_window < 0 || g->recent_window > g->max_tokens_per_seq) return false;
  const int64_t ring = (int64_t)g->max_batch * g->n_layers * ((g->recent_window + PASK_PAGE_TOKENS - 1) / PASK_PAGE_TOKENS);
  if (ring + g->hi_pages > INT32_MAX) return false;
  return true;
}

inline CacheDims dims_of(const pask_geom* g) {
  const uint64_t D = (uint64_t)g->head_dim, H = (uint64_t)g->n_kv_heads;
  return CacheDims{g->max_batch, g->n_layers, g->max_tokens_per_seq, g->recent_window, g->hi_pages, g->lo_pages,
                   H * 2 * PASK_PAGE_TOKENS * D * 2,
                   H * 2 * (PASK_PAGE_TOKENS * (D / 2) + PASK_PAGE_TOKENS * (D / PASK_QGROUP) * 2)};
}

// Layout of a cache buffer; false when the geometry is unsupported.
inline bool layout_of(const pask_geom* g, pask_cache_layout* L) {
  if (!valid_geom(g)) return false;
  *L = layout_regions(dims_of(g));
  return true;
}

inline CacheView view_of(const pask_cache* c) {
  const CacheDims d = dims_of(&c->geom);
  CacheView v = view_regions(c->base, layout_regions(d), d);
  v.n_kv_heads = c->geom.n_kv_heads;
  v.head_dim = c->geom.head_dim;
  return v;
}

inline int check_cache(const pask_cache* c) {
  if (!c || !c->base) return PASK_E_ARG;
  if (!valid_geom(&c->geom)) return PASK_E_SHAPE;
  if (!aligned(c->base, 256)) return PASK_E_ARG;
  pask_cache_layout L;
  layout_of(&c->geom, &L);
  if (c->bytes < L.total_bytes) return PASK_E_CAPACITY;
  return PASK_OK;
}

}  // namespace pask
