// Host side of the latent-attention C ABI (pask_latent.h): argument checks,
// cache layout and launch planning.  Every check runs before the first HIP
// call of an entry point.
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <memory>
#include <new>

#include <hip/hip_runtime_api.h>

#include "pask_host.h"
#include "pask_latent_internal.h"

namespace {

using pask::align_up;
using pask::aligned;
using pask::CacheView;

constexpr int kTileSlots = 32;

bool valid_geom(const pask_latent_geom* g) {
  if (!g) return false;
  if (g->max_batch < 1 || g->max_batch > 65535) return false;
  if (g->n_layers < 1 || g->n_layers > PASK_MAX_LAYERS) return false;
  if (g->n_q_heads < 1 || g->n_q_heads > PASK_LATENT_MAX_HEADS) return false;
  if (g->rank != 128 && g->rank != 256 && g->rank != 512) return false;
  if (g->rope_dim != 32 && g->rope_dim != 64) return false;
  if (g->page_tokens != PASK_PAGE_TOKENS) return false;
  if (g->max_tokens_per_seq < 1 || g->max_tokens_per_seq > (1 << 28)) return false;
  return g->hi_pages >= 0 && g->lo_pages >= 0;
}

// Bytes of one entry, DROP, LOW, HIGH.
void entry_bytes(const pask_latent_geom& g, int64_t m[3]) {
  m[PASK_DROP] = 0;
  m[PASK_RETAIN_LOW] = g.rank / 2 + 2 * (g.rank / PASK_QGROUP) + 2 * g.rope_dim;
  m[PASK_RETAIN_HIGH] = 2 * (g.rank + g.rope_dim);
}

pask::CacheDims dims_of(const pask_latent_geom& g) {
  int64_t m[3];
  entry_bytes(g, m);
  return pask::CacheDims{g.max_batch, g.n_layers, g.max_tokens_per_seq, 0, g.hi_pages, g.lo_pages,
                         (uint64_t)(PASK_PAGE_TOKENS * m[PASK_RETAIN_HIGH]),
                         (uint64_t)(PASK_PAGE_TOKENS * m[PASK_RETAIN_LOW])};
}

pask_cache_layout layout_of(const pask_latent_geom& g) { return pask::layout_regions(dims_of(g)); }

CacheView view_of(const pask_latent_cache* c) {
  const pask::CacheDims d = dims_of(c->geom);
  return pask::view_regions(c->base, pask::layout_regions(d), d);
}

int check_cache(const pask_latent_cache* c) {
  if (!c || !c->base) return PASK_E_ARG;
  if (!valid_geom(&c->geom)) return PASK_E_SHAPE;
  if (!aligned(c->base, 256)) return PASK_E_ARG;
  return c->bytes < layout_of(c->geom).total_bytes ? PASK_E_CAPACITY : PASK_OK;
}

int check_policy(const pask_policy* p, const pask_latent_cache* c) {
  const int st = pask::check_policy_layers(p, c->geom.n_layers);
  if (st != PASK_OK) return st;
  if (p->recent_window != 0) return PASK_E_UNSUPPORTED;
  return pask::check_policy_groups(p);
}

int check_call(const pask_latent_cache* cache, int32_t layer, int32_t batch) {
  if (layer < 0 || layer >= cache->geom.n_layers) return PASK_E_SHAPE;
  return batch < 1 || batch > cache->geom.max_batch ? PASK_E_SHAPE : PASK_OK;
}

int debug_check(const char* where, hipError_t e, const pask_latent_cache* cache, hipStream_t stream) {
  const void* word = cache->base;                  // the status word opens the buffer
  return pask::debug_check_words(where, e == hipSuccess ? PASK_OK : PASK_E_HIP, &word, 1, stream);
}

int workers_for(const pask_latent_geom& g, int32_t batch, int32_t max_ctx_hint) {
  const int64_t hint = max_ctx_hint < 1 ? g.max_tokens_per_seq : std::min(max_ctx_hint, g.max_tokens_per_seq);
  // both stores of a sequence may end in a part of a tile
  return pask::latent_workers(g.n_q_heads, batch * ((hint + kTileSlots - 1) / kTileSlots + 1));
}

// Two partial results per workgroup (its first sequence and its last), and two
// words per sequence that say where its partials are.
struct WsLayout {
  uint64_t ml_off, seq_off, total;
};
WsLayout ws_layout(const pask_latent_geom& g, int32_t batch, int workers) {
  const uint64_t rows = 2ull * workers * 16 * pask::latent_head_tiles(g.n_q_heads);
  WsLayout w;
  w.ml_off = align_up(rows * g.rank * 4, pask::kAlignSmall);
  w.seq_off = align_up(w.ml_off + rows * 8, pask::kAlignSmall);
  w.total = align_up(w.seq_off + (uint64_t)batch * 8, pask::kAlignSmall);
  return w;
}

pask::LatentAppendArgs append_args(const pask_policy* policy, pask_latent_cache* cache, int32_t layer, int32_t batch,
                                   const int32_t* n_new, int32_t max_new, const uint8_t* tags, const void* c,
                                   const void* r, uint32_t flags) {
  pask::LatentAppendArgs a;
  a.base.cv = view_of(cache);
  a.base.tab = pask::column_of(policy, layer);
  a.base.n_new = n_new;
  a.base.tags = tags;
  a.base.states = nullptr;
  a.base.k = static_cast<const uint16_t*>(c);
  a.base.v = static_cast<const uint16_t*>(r);
  a.base.layer = layer;
  a.base.batch = batch;
  a.base.max_new = max_new;
  a.base.flags = flags;
  a.rank = cache->geom.rank;
  a.rope = cache->geom.rope_dim;
  return a;
}

bool rows_ok(const void* p) { return p && aligned(p, 16); }

// The kernels' exponentials are in base 2.
float scale_log2(float softmax_scale) { return (float)((double)softmax_scale * 1.4426950408889634); }
bool scale_ok(float softmax_scale) { return isfinite(softmax_scale) && isfinite(scale_log2(softmax_scale)); }

int check_prompt(int32_t batch, int32_t n_heads, int32_t nope_dim, int32_t rope_dim, int32_t v_dim, int32_t max_q,
                 int32_t total_q, int32_t total_k, const int32_t* cu_q, const int32_t* cu_k, const float* lse,
                 float softmax_scale) {
  if (batch < 1 || batch > 65535 || n_heads < 1 || n_heads > PASK_LATENT_MAX_HEADS) return PASK_E_SHAPE;
  if ((nope_dim != 64 && nope_dim != 128) || (v_dim != 64 && v_dim != 128) || (rope_dim != 32 && rope_dim != 64))
    return PASK_E_SHAPE;
  if (max_q < 0 || total_q < 0 || total_k < 0 || !scale_ok(softmax_scale)) return PASK_E_ARG;
  if (!cu_q || !cu_k || !aligned(cu_q, 4) || !aligned(cu_k, 4) || !aligned(lse, 4)) return PASK_E_ARG;
  return PASK_OK;
}

// Prompts with queries, their sizes and offsets checked (check_prompt); pos: null, or the keys' positions.
int prompt_attn(const char* where, int32_t batch, int32_t n_heads, int32_t nope_dim, int32_t rope_dim, int32_t v_dim,
                int32_t max_q, int32_t total_q, int32_t total_k, const int32_t* cu_q, const int32_t* cu_k,
                const int32_t* pos, const int32_t* q_first, const void* q, const void* kv, const void* r, void* out,
                float* lse, float softmax_scale, hipStream_t stream) {
  if (!rows_ok(q) || !rows_ok(out)) return PASK_E_ARG;
  if (total_k > 0 && (!rows_ok(kv) || !rows_ok(r))) return PASK_E_ARG;
  pask::LatentPromptArgs a;
  a.q = static_cast<const uint16_t*>(q);
  a.kv = static_cast<const uint16_t*>(kv);
  a.r = static_cast<const uint16_t*>(r);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.cu_q = cu_q;
  a.cu_k = cu_k;
  a.pos = pos;
  a.q_first = q_first;
  a.scale_log2 = scale_log2(softmax_scale);
  a.batch = batch;
  a.heads = n_heads;
  a.nope = nope_dim;
  a.rope = rope_dim;
  a.v = v_dim;
  a.max_q = std::min(max_q, total_q);
  a.total_q = total_q;
  a.total_k = total_k;
  if (pask::latent_prompt_blocks(a) > (1 << 23) - 1) return PASK_E_SHAPE;   // a launch holds 2^32 - 1 threads
  const hipError_t e = pask::launch_latent_prompt(a, stream);
  return pask::debug_check_words(where, e == hipSuccess ? PASK_OK : PASK_E_HIP, nullptr, 0, stream);
}

}  // namespace

extern "C" {

int pask_latent_cache_layout_query(const pask_latent_geom* geom, pask_cache_layout* out) {
  if (!geom || !out) return PASK_E_ARG;
  if (!valid_geom(geom)) return PASK_E_SHAPE;
  *out = layout_of(*geom);
  return PASK_OK;
}

size_t pask_latent_cache_bytes(const pask_latent_geom* geom) {
  return valid_geom(geom) ? (size_t)layout_of(*geom).total_bytes : 0;
}

int pask_latent_cache_reset(pask_latent_cache* cache, hipStream_t stream) {
  const int st = check_cache(cache);
  if (st != PASK_OK) return st;
  return debug_check("pask_latent_cache_reset", pask::launch_reset(view_of(cache), cache->geom.max_batch, stream),
                     cache, stream);
}

int pask_latent_cache_init(pask_latent_cache* cache, const pask_latent_geom* geom, void* base, size_t bytes,
                           hipStream_t stream) {
  if (!cache || !geom || !base) return PASK_E_ARG;
  if (!valid_geom(geom)) return PASK_E_SHAPE;
  if (!aligned(base, 256)) return PASK_E_ARG;
  if (bytes < pask_latent_cache_bytes(geom)) return PASK_E_CAPACITY;
  cache->geom = *geom;
  cache->base = base;
  cache->bytes = bytes;
  return pask_latent_cache_reset(cache, stream);
}

int pask_latent_append(const pask_policy* policy, pask_latent_cache* cache, int32_t layer, int32_t batch,
                       const int32_t* n_new_dev, int32_t max_new, const uint8_t* tags_dev, const void* c_dev,
                       const void* r_dev, uint32_t flags, hipStream_t stream) {
  int st = check_cache(cache);
  if (st == PASK_OK) st = check_policy(policy, cache);
  if (st == PASK_OK) st = check_call(cache, layer, batch);
  if (st != PASK_OK) return st;
  if (max_new < 0 || max_new > cache->geom.max_tokens_per_seq) return PASK_E_SHAPE;
  if (!pask::append_fits(max_new, 0)) return PASK_E_SHAPE;
  if (flags & ~(uint32_t)PASK_APPEND_KEEP_ALL) return PASK_E_ARG;
  if (!rows_ok(c_dev) || !rows_ok(r_dev)) return PASK_E_ARG;
  if (!tags_dev && !(flags & PASK_APPEND_KEEP_ALL)) return PASK_E_ARG;
  if (n_new_dev && !aligned(n_new_dev, 4)) return PASK_E_ARG;
  if (max_new == 0) return PASK_OK;
  return debug_check("pask_latent_append",
                     pask::launch_latent_append(append_args(policy, cache, layer, batch, n_new_dev, max_new, tags_dev,
                                                            c_dev, r_dev, flags),
                                                stream),
                     cache, stream);
}

int pask_latent_read(const pask_latent_cache* cache, int32_t layer, int32_t batch, int32_t rows, void* c_dev,
                     void* r_dev, int32_t* pos_dev, int32_t* cu_dev, hipStream_t stream) {
  int st = check_cache(cache);
  if (st == PASK_OK) st = check_call(cache, layer, batch);
  if (st != PASK_OK) return st;
  if ((int64_t)batch * cache->geom.max_tokens_per_seq > INT32_MAX) return PASK_E_SHAPE;
  if (rows < 0 || !cu_dev || !aligned(cu_dev, 4) || !aligned(pos_dev, 4)) return PASK_E_ARG;
  if (rows > 0 && (!rows_ok(c_dev) || !rows_ok(r_dev))) return PASK_E_ARG;
  pask::LatentReadArgs a;
  a.cv = view_of(cache);
  a.c = static_cast<uint16_t*>(c_dev);
  a.r = static_cast<uint16_t*>(r_dev);
  a.pos = pos_dev;
  a.cu = cu_dev;
  a.layer = layer;
  a.batch = batch;
  a.rows = rows;
  a.rank = cache->geom.rank;
  a.rope = cache->geom.rope_dim;
  return debug_check("pask_latent_read", pask::launch_latent_read(a, stream), cache, stream);
}

size_t pask_latent_workspace_bytes(const pask_latent_geom* geom, int32_t batch, int32_t max_ctx_hint) {
  if (!valid_geom(geom) || batch < 1 || batch > geom->max_batch) return 0;
  return (size_t)ws_layout(*geom, batch, workers_for(*geom, batch, max_ctx_hint)).total;
}

int pask_latent_decode_attn(const pask_policy* policy, pask_latent_cache* cache, int32_t layer, int32_t batch,
                            const void* q_dev, void* out_dev, float* lse_dev, const uint8_t* tags_new_dev,
                            const void* c_new_dev, const void* r_new_dev, float softmax_scale, int32_t max_ctx_hint,
                            void* ws_dev, size_t ws_bytes, hipStream_t stream) {
  int st = check_cache(cache);
  if (st == PASK_OK) st = check_policy(policy, cache);
  if (st == PASK_OK) st = check_call(cache, layer, batch);
  if (st != PASK_OK) return st;
  const pask_latent_geom& g = cache->geom;
  if (!rows_ok(q_dev) || !rows_ok(out_dev) || !aligned(lse_dev, 4)) return PASK_E_ARG;
  if (tags_new_dev && (!rows_ok(c_new_dev) || !rows_ok(r_new_dev))) return PASK_E_ARG;
  if (!scale_ok(softmax_scale)) return PASK_E_ARG;
  const int workers = workers_for(g, batch, max_ctx_hint);
  const WsLayout w = ws_layout(g, batch, workers);
  if (!ws_dev || !aligned(ws_dev, 256)) return PASK_E_ARG;
  if (ws_bytes < w.total) return PASK_E_CAPACITY;
  if (tags_new_dev &&
      pask::launch_latent_append(append_args(policy, cache, layer, batch, nullptr, 1, tags_new_dev, c_new_dev,
                                             r_new_dev, 0),
                                 stream) != hipSuccess)
    return PASK_E_HIP;
  uint8_t* ws = static_cast<uint8_t*>(ws_dev);
  pask::LatentAttnArgs a;
  a.cv = view_of(cache);
  a.q = static_cast<const uint16_t*>(q_dev);
  a.out = static_cast<uint16_t*>(out_dev);
  a.lse = lse_dev;
  a.ws_o = reinterpret_cast<float*>(ws);
  a.ws_ml = reinterpret_cast<float*>(ws + w.ml_off);
  a.ws_seq = reinterpret_cast<int32_t*>(ws + w.seq_off);
  a.scale_log2 = scale_log2(softmax_scale);
  a.layer = layer;
  a.batch = batch;
  a.heads = g.n_q_heads;
  a.rank = g.rank;
  a.rope = g.rope_dim;
  a.workers = workers;
  return debug_check("pask_latent_decode_attn", pask::launch_latent_attention(a, stream), cache, stream);
}

int pask_latent_prompt_attn(int32_t batch, int32_t n_heads, int32_t nope_dim, int32_t rope_dim, int32_t v_dim,
                            int32_t max_q, int32_t total_q, int32_t total_k, const int32_t* cu_q_dev,
                            const int32_t* cu_k_dev, const void* q_dev, const void* kv_dev, const void* r_dev,
                            void* out_dev, float* lse_dev, float softmax_scale, hipStream_t stream) {
  const int st = check_prompt(batch, n_heads, nope_dim, rope_dim, v_dim, max_q, total_q, total_k, cu_q_dev, cu_k_dev,
                              lse_dev, softmax_scale);
  if (st != PASK_OK || max_q == 0 || total_q == 0) return st;
  return prompt_attn("pask_latent_prompt_attn", batch, n_heads, nope_dim, rope_dim, v_dim, max_q, total_q, total_k,
                     cu_q_dev, cu_k_dev, nullptr, nullptr, q_dev, kv_dev, r_dev, out_dev, lse_dev, softmax_scale,
                     stream);
}

int pask_latent_prompt_attn_pos(int32_t batch, int32_t n_heads, int32_t nope_dim, int32_t rope_dim, int32_t v_dim,
                                int32_t max_q, int32_t total_q, int32_t total_k, const int32_t* cu_q_dev,
                                const int32_t* cu_k_dev, const int32_t* pos_dev, const int32_t* q_first_dev,
                                const void* q_dev, const void* kv_dev, const void* r_dev, void* out_dev,
                                float* lse_dev, float softmax_scale, hipStream_t stream) {
  const int st = check_prompt(batch, n_heads, nope_dim, rope_dim, v_dim, max_q, total_q, total_k, cu_q_dev, cu_k_dev,
                              lse_dev, softmax_scale);
  if (st != PASK_OK) return st;
  if (!q_first_dev || !aligned(q_first_dev, 4) || !aligned(pos_dev, 4)) return PASK_E_ARG;
  if (total_k > 0 && !pos_dev) return PASK_E_ARG;
  if (max_q == 0 || total_q == 0) return PASK_OK;
  return prompt_attn("pask_latent_prompt_attn_pos", batch, n_heads, nope_dim, rope_dim, v_dim, max_q, total_q, total_k,
                     cu_q_dev, cu_k_dev, pos_dev, q_first_dev, q_dev, kv_dev, r_dev, out_dev, lse_dev, softmax_scale,
                     stream);
}

int pask_latent_cache_stats(const pask_policy* policy, const pask_latent_cache* cache, int32_t batch,
                            pask_stats* out, hipStream_t stream) {
  int st = check_cache(cache);
  if (st == PASK_OK) st = check_policy(policy, cache);
  if (st == PASK_OK) st = check_call(cache, 0, batch);
  if (st != PASK_OK) return st;
  if (!out) return PASK_E_ARG;
  const pask_latent_geom& g = cache->geom;
  const pask_cache_layout L = layout_of(g);
  const size_t words = (size_t)batch * g.n_layers * pask::kCounterStride;
  std::unique_ptr<int32_t[]> cnt(new (std::nothrow) int32_t[words]);
  if (!cnt) return PASK_E_CAPACITY;
  uint32_t status[4];
  const uint8_t* base = static_cast<const uint8_t*>(cache->base);
  if (hipMemcpyAsync(status, base + L.status_off, sizeof(status), hipMemcpyDeviceToHost, stream) != hipSuccess ||
      hipMemcpyAsync(cnt.get(), base + L.counters_off, words * 4, hipMemcpyDeviceToHost, stream) != hipSuccess ||
      hipStreamSynchronize(stream) != hipSuccess)
    return PASK_E_HIP;
  pask_stats s;
  memset(&s, 0, sizeof(s));
  for (size_t i = 0; i < words; i += pask::kCounterStride) {
    const int32_t* c = &cnt[i];
    s.n_entries += c[pask::kCntPos];
    s.n_high += c[pask::kCntHi];
    s.n_low += c[pask::kCntLo];
    s.n_drop += c[pask::kCntDrop];
    s.n_forced_high += c[pask::kCntForced];
    s.n_lost += c[pask::kCntLost];
  }
  int64_t m[3];
  entry_bytes(g, m);
  s.bytes_high = s.n_high * m[PASK_RETAIN_HIGH];
  s.bytes_low = s.n_low * m[PASK_RETAIN_LOW];
  s.hi_pages_used = std::min<int64_t>(status[2], g.hi_pages);
  s.lo_pages_used = std::min<int64_t>(status[3], g.lo_pages);
  const double full = (double)m[PASK_RETAIN_HIGH];
  const int64_t gov_high = s.n_high - s.n_forced_high, gov = gov_high + s.n_low + s.n_drop;
  const int64_t all = s.n_high + s.n_low + s.n_drop;
  s.c_kv_governed = gov > 0 ? ((double)gov_high * full + (double)s.bytes_low) / ((double)gov * full) : NAN;
  s.c_kv_all = all > 0 ? (double)(s.bytes_high + s.bytes_low) / ((double)all * full) : NAN;
  s.device_flags = status[0];
  *out = s;
  return status[0] ? PASK_E_DEVICE_FLAG : PASK_OK;
}

}  // extern "C"
