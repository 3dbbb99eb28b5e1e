// Internal declarations shared by the C entry points of pask_prompt.h
// (pask_prompt_api.cpp) and their gfx950 kernels (pask_rope.hip,
// pask_prompt.hip).
#pragma once

#include "pask_internal.h"
#include "pask_prompt.h"

namespace pask {

// Rows of one tensor: heads of head_dim elements behind each other, rows `in` (`out`) elements apart.
struct RopeRows {
  const uint16_t* src;
  uint16_t* dst;
  int64_t in, out;
};

struct RopeArgs {
  pask_rope rope;
  RopeRows q, k;
  const int32_t* n_new;     // [batch] or null (all max_new)
  const int32_t* first;     // position of sequence b's first row at first[b * first_stride], or null:
  const int32_t* pos;       // [batch * max_new]
  int64_t first_stride;
  int32_t batch, max_new, q_heads, k_heads;
  // set at launch
  int32_t pieces;           // 16-byte chunks (or pairs of them), or pairs of elements and single ones, of a head
  int32_t rot_pieces;       // the first of them: those of the rotated part
  int32_t tokens;           // rows a workgroup takes
  int32_t q_copies, k_copies;   // the other pieces are copied (0 in place)
};

hipError_t launch_rope(const RopeArgs& a, hipStream_t s);

struct PromptArgs {
  CacheView cv;
  const uint16_t* q;        // bf16 bits [batch][max_q][Hq][D]
  uint16_t* out;            // the same
  float* lse;               // [batch][max_q][Hq] or null
  const int32_t* n_q;       // [batch] or null (all max_q)
  const int32_t* first;     // [batch] or null (the queries are the last tokens)
  float* ws_o;              // [batch][Hkv][pieces][rows][D], rows = max_q * G
  float* ws_ml;             // [batch][Hkv][pieces][rows][2]  (reference in log2 units, sum)
  float scale_log2;         // softmax_scale * log2(e)
  int32_t layer, batch, max_q, n_q_heads;
  int32_t pieces;           // parts the keys of a tile are cut into; 1: written out directly
};

// How a call is cut: rows (query, head of the group) of a workgroup's tile, and pieces of its keys.
struct PromptCut {
  int32_t rows, pieces;
};
PromptCut prompt_cut(int32_t batch, int32_t max_q, int32_t group, int32_t n_kv_heads, int32_t head_dim,
                     int32_t max_ctx_hint);
int64_t prompt_blocks(const PromptArgs& a, const PromptCut& c);   // workgroups of the attention kernel

hipError_t launch_prompt(const PromptArgs& a, const PromptCut& c, hipStream_t s);

}  // namespace pask
