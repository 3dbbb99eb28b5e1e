// Host side of pask_prompt.h: argument checks, rotary frequencies and launch
// planning.  Every check runs before the first HIP call of an entry point.
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>

#include <hip/hip_runtime_api.h>

#include "pask_geom.h"
#include "pask_prompt_internal.h"

namespace {

using pask::align_up;
using pask::aligned;

constexpr double kTwoPi = 6.283185307179586476925;

int check_rope_shape(int32_t head_dim, int32_t rot_first, int32_t rot_dim) {
  if (head_dim < 2 || head_dim > PASK_ROPE_MAX_HEAD_DIM) return PASK_E_SHAPE;
  if (rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > 2 * PASK_ROPE_MAX_PAIRS) return PASK_E_SHAPE;
  return rot_first < 0 || rot_first > head_dim - rot_dim ? PASK_E_SHAPE : PASK_OK;
}

int check_rope(const pask_rope* r) {
  if (!r || check_rope_shape(r->head_dim, r->rot_first, r->rot_dim) != PASK_OK) return PASK_E_ARG;
  if (r->layout != PASK_ROPE_HALF && r->layout != PASK_ROPE_INTERLEAVED) return PASK_E_ARG;
  if (!isfinite(r->magnitude)) return PASK_E_ARG;
  for (int i = 0; i < r->rot_dim / 2; ++i)
    if (!isfinite(r->turns[i])) return PASK_E_ARG;
  return PASK_OK;
}

int check_rope_rows(const pask_rope& r, int32_t heads, const void* in, int64_t in_stride, const void* out,
                    int64_t out_stride) {
  if (heads == 0) return PASK_OK;
  if (!in || !out || !aligned(in, 2) || !aligned(out, 2)) return PASK_E_ARG;
  const int64_t row = (int64_t)heads * r.head_dim;
  if (in_stride < row || out_stride < row || in_stride > ((int64_t)1 << 40) || out_stride > ((int64_t)1 << 40))
    return PASK_E_ARG;
  return in == out && in_stride != out_stride ? PASK_E_ARG : PASK_OK;
}

int32_t hint_of(const pask_geom& g, int32_t max_ctx_hint) {
  return max_ctx_hint < 1 || max_ctx_hint > g.max_tokens_per_seq ? g.max_tokens_per_seq : max_ctx_hint;
}

pask::PromptCut cut_of(const pask_geom& g, int32_t batch, int32_t max_q, int32_t max_ctx_hint) {
  return pask::prompt_cut(batch, max_q, g.n_q_heads / g.n_kv_heads, g.n_kv_heads, g.head_dim, hint_of(g, max_ctx_hint));
}

struct WsLayout {
  uint64_t ml_off, total;
};
// Per (sequence, KV head, piece) and row an output, then a reference and a sum.
WsLayout ws_layout(const pask_geom& g, int32_t batch, int32_t max_q, int32_t pieces) {
  WsLayout w = {0, 0};
  if (pieces <= 1) return w;
  const uint64_t rows = (uint64_t)batch * g.n_q_heads * pieces * max_q;
  w.ml_off = align_up(rows * g.head_dim * 4, pask::kAlignSmall);
  w.total = align_up(w.ml_off + rows * 8, pask::kAlignSmall);
  return w;
}

}  // namespace

extern "C" {

int pask_rope_init(pask_rope* out, int32_t head_dim, int32_t rot_first, int32_t rot_dim, int32_t layout, double base,
                   int32_t scaling, double factor, int32_t original_len, double low_turns, double high_turns,
                   float magnitude) {
  if (!out) return PASK_E_ARG;
  const int st = check_rope_shape(head_dim, rot_first, rot_dim);
  if (st != PASK_OK) return st;
  if (layout != PASK_ROPE_HALF && layout != PASK_ROPE_INTERLEAVED) return PASK_E_ARG;
  if (scaling < PASK_ROPE_PLAIN || scaling > PASK_ROPE_PARTS) return PASK_E_ARG;
  if (!isfinite(base) || !(base > 0.0) || !isfinite(magnitude)) return PASK_E_ARG;
  if (scaling != PASK_ROPE_PLAIN && (!isfinite(factor) || factor < 1.0)) return PASK_E_ARG;
  const bool parts = scaling == PASK_ROPE_PARTS;
  if (parts && (original_len < 1 || !isfinite(high_turns) || !(low_turns >= 0.0) || !(low_turns < high_turns)))
    return PASK_E_ARG;
  pask_rope r;
  memset(&r, 0, sizeof(r));
  r.head_dim = head_dim;
  r.rot_first = rot_first;
  r.rot_dim = rot_dim;
  r.layout = layout;
  r.magnitude = magnitude;
  if (scaling == PASK_ROPE_BASE && rot_dim > 2) base *= pow(factor, (double)rot_dim / (rot_dim - 2));
  for (int i = 0; i < rot_dim / 2; ++i) {
    const double turns = pow(base, -2.0 * i / rot_dim) / kTwoPi;
    double keep = scaling == PASK_ROPE_LINEAR ? 0.0 : 1.0;   // the part of the frequency that is not scaled
    if (parts) keep = std::min(1.0, std::max(0.0, (turns * original_len - low_turns) / (high_turns - low_turns)));
    r.turns[i] = keep == 1.0 ? turns : keep * turns + (1.0 - keep) * turns / factor;
    if (!isfinite(r.turns[i])) return PASK_E_ARG;
  }
  *out = r;
  return PASK_OK;
}

int pask_rope_apply(const pask_rope* rope, int32_t batch, int32_t max_new, const int32_t* n_new_dev,
                    const int32_t* first_dev, int64_t first_stride, const int32_t* pos_dev, int32_t n_q_heads,
                    const void* q_in, int64_t q_in_stride, void* q_out, int64_t q_out_stride, int32_t n_k_heads,
                    const void* k_in, int64_t k_in_stride, void* k_out, int64_t k_out_stride, hipStream_t stream) {
  int st = check_rope(rope);
  if (st != PASK_OK) return st;
  if (batch < 0 || max_new < 0 || (int64_t)batch * max_new > INT32_MAX) return PASK_E_SHAPE;
  if (n_q_heads < 0 || n_k_heads < 0 || n_q_heads > PASK_ROPE_MAX_HEADS || n_k_heads > PASK_ROPE_MAX_HEADS)
    return PASK_E_SHAPE;
  if ((pos_dev != nullptr) == (first_dev != nullptr) || (first_dev && first_stride < 0)) return PASK_E_ARG;
  if (!aligned(pos_dev, 4) || !aligned(first_dev, 4) || !aligned(n_new_dev, 4)) return PASK_E_ARG;
  st = check_rope_rows(*rope, n_q_heads, q_in, q_in_stride, q_out, q_out_stride);
  if (st != PASK_OK) return st;
  st = check_rope_rows(*rope, n_k_heads, k_in, k_in_stride, k_out, k_out_stride);
  if (st != PASK_OK) return st;
  if (batch == 0 || max_new == 0 || n_q_heads + n_k_heads == 0) return PASK_OK;
  pask::RopeArgs a;
  memset(&a, 0, sizeof(a));
  a.rope = *rope;
  a.q = {static_cast<const uint16_t*>(q_in), static_cast<uint16_t*>(q_out), q_in_stride, q_out_stride};
  a.k = {static_cast<const uint16_t*>(k_in), static_cast<uint16_t*>(k_out), k_in_stride, k_out_stride};
  a.n_new = n_new_dev;
  a.first = first_dev;
  a.pos = pos_dev;
  a.first_stride = first_stride;
  a.batch = batch;
  a.max_new = max_new;
  a.q_heads = n_q_heads;
  a.k_heads = n_k_heads;
  return pask::debug_check_words("pask_rope_apply", pask::launch_rope(a, stream) == hipSuccess ? PASK_OK : PASK_E_HIP,
                                 nullptr, 0, stream);
}

size_t pask_prompt_workspace_bytes(const pask_geom* geom, int32_t batch, int32_t max_q, int32_t max_ctx_hint) {
  if (!pask::valid_geom(geom) || batch < 1 || batch > geom->max_batch) return 0;
  if (max_q < 1 || max_q > geom->max_tokens_per_seq) return 0;
  return (size_t)ws_layout(*geom, batch, max_q, cut_of(*geom, batch, max_q, max_ctx_hint).pieces).total;
}

int pask_prompt_attn(const pask_cache* cache, int32_t layer, int32_t batch, int32_t max_q, const int32_t* n_q_dev,
                     const int32_t* first_dev, const void* q_dev, void* out_dev, float* lse_dev, float softmax_scale,
                     int32_t max_ctx_hint, void* ws_dev, size_t ws_bytes, hipStream_t stream) {
  int st = pask::check_cache(cache);
  if (st != PASK_OK) return st;
  const pask_geom& g = cache->geom;
  if (layer < 0 || layer >= g.n_layers) return PASK_E_SHAPE;
  if (batch < 1 || batch > g.max_batch) return PASK_E_SHAPE;
  if (max_q < 0 || max_q > g.max_tokens_per_seq) return PASK_E_SHAPE;
  if (!q_dev || !aligned(q_dev, 16) || !out_dev || !aligned(out_dev, 16)) return PASK_E_ARG;
  if (!aligned(n_q_dev, 4) || !aligned(first_dev, 4) || !aligned(lse_dev, 4)) return PASK_E_ARG;
  const float scale_log2 = (float)((double)softmax_scale * 1.4426950408889634);
  if (!isfinite(softmax_scale) || !isfinite(scale_log2)) return PASK_E_ARG;
  if (max_q == 0) return PASK_OK;
  const pask::PromptCut cut = cut_of(g, batch, max_q, max_ctx_hint);
  const WsLayout w = ws_layout(g, batch, max_q, cut.pieces);
  if (w.total && (!ws_dev || !aligned(ws_dev, 256))) return PASK_E_ARG;
  if (ws_bytes < w.total) return PASK_E_CAPACITY;
  pask::PromptArgs a;
  a.cv = pask::view_of(cache);
  a.q = static_cast<const uint16_t*>(q_dev);
  a.out = static_cast<uint16_t*>(out_dev);
  a.lse = lse_dev;
  a.n_q = n_q_dev;
  a.first = first_dev;
  a.ws_o = static_cast<float*>(ws_dev);
  a.ws_ml = reinterpret_cast<float*>(static_cast<uint8_t*>(ws_dev) + w.ml_off);
  a.scale_log2 = scale_log2;
  a.layer = layer;
  a.batch = batch;
  a.max_q = max_q;
  a.n_q_heads = g.n_q_heads;
  a.pieces = cut.pieces;
  if (pask::prompt_blocks(a, cut) >= (1 << 23)) return PASK_E_SHAPE;
  const void* word = cache->base;                  // the status word opens the buffer
  return pask::debug_check_words("pask_prompt_attn",
                                 pask::launch_prompt(a, cut, stream) == hipSuccess ? PASK_OK : PASK_E_HIP, &word, 1,
                                 stream);
}

}  // extern "C"
