// Declarations shared by the latent entry points (pask_latent_api.cpp) and
// their kernels.  Not part of the public interface.
#pragma once

#include "pask_internal.h"
#include "pask_latent.h"

namespace pask {

struct LatentAppendArgs {
  AppendArgs base;          // cache, table, tags and counts; k holds the latents, v the rotary keys
  int32_t rank, rope;
};

struct LatentReadArgs {
  CacheView cv;
  uint16_t* c;              // bf16 bits [rows][rank]
  uint16_t* r;              // [rows][rope]
  int32_t* pos;             // [rows] or null
  int32_t* cu;              // [batch + 1]
  int32_t layer, batch, rows, rank, rope;
};

struct LatentAttnArgs {
  CacheView cv;
  const uint16_t* q;        // bf16 bits [batch][heads][rank + rope]
  uint16_t* out;            // [batch][heads][rank]
  float* lse;               // [batch][heads] or null
  float* ws_o;              // [2 workers][tile heads][rank]
  float* ws_ml;             // [2 workers][tile heads][2]  (max in log2 units, sum)
  int32_t* ws_seq;          // [batch][2]: first partial and number of partials (0: written by its worker)
  float scale_log2;         // softmax_scale * log2(e)
  int32_t layer, batch, heads, rank, rope, workers;
};

struct LatentPromptArgs {
  const uint16_t* q;        // bf16 bits [total_q][heads][nope + rope]
  const uint16_t* kv;       // [total_k][heads][nope + v]
  const uint16_t* r;        // [total_k][rope]
  uint16_t* out;            // [total_q][heads][v]
  float* lse;               // [total_q][heads] or null
  const int32_t* cu_q;
  const int32_t* cu_k;
  const int32_t* pos;       // [total_k] positions of the keys, or null: the queries are the last of their keys
  const int32_t* q_first;   // [batch] position of each sequence's first query, with pos
  float scale_log2;
  int32_t batch, heads, nope, rope, v, max_q, total_q, total_k;
};

// Head tiles (16 heads) the decode kernel is built for: 1, 2, 4 or 8.
inline int latent_head_tiles(int heads) { return heads <= 16 ? 1 : heads <= 32 ? 2 : heads <= 64 ? 4 : 8; }
// Workgroups of the decode kernel; at most `tiles` (of 32 slots, and one per sequence).
int latent_workers(int heads, int64_t tiles);

hipError_t launch_latent_append(const LatentAppendArgs& a, hipStream_t s);   // chooses the one-token kernel
hipError_t launch_latent_read(const LatentReadArgs& a, hipStream_t s);
hipError_t launch_latent_attention(const LatentAttnArgs& a, hipStream_t s);
hipError_t launch_latent_prompt(const LatentPromptArgs& a, hipStream_t s);
int64_t latent_prompt_blocks(const LatentPromptArgs& a);   // workgroups it launches

}  // namespace pask
