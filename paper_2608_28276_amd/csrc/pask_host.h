// Host-side pieces shared by the C entry points (pask_api.cpp and
// pask_latent_api.cpp): the layout of a cache buffer and its device view, the
// policy checks, and the debug check after a call.
#pragma once

#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <atomic>

#include <hip/hip_runtime_api.h>

#include "pask_internal.h"
#include "pask_pages.h"

namespace pask {

constexpr uint64_t kAlignSmall = 256;
constexpr uint64_t kAlignPool = 4096;

inline uint64_t align_up(uint64_t x, uint64_t a) { return (x + a - 1) / a * a; }
inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// What the regions of a cache buffer depend on; sizes checked by the caller.
struct CacheDims {
  int32_t max_batch, n_layers, max_tokens, window, hi_pages, lo_pages;
  uint64_t hi_page_bytes, lo_page_bytes;
};

inline pask_cache_layout layout_regions(const CacheDims& g) {
  pask_cache_layout L;
  memset(&L, 0, sizeof(L));
  const uint64_t B = (uint64_t)g.max_batch, NL = (uint64_t)g.n_layers;
  const uint64_t T = (uint64_t)g.max_tokens, W = (uint64_t)g.window;
  L.max_pages = (int32_t)((T + PASK_PAGE_TOKENS - 1) / PASK_PAGE_TOKENS);
  L.counter_stride = kCounterStride;
  L.ring_pages = (int32_t)(B * NL * ((W + PASK_PAGE_TOKENS - 1) / PASK_PAGE_TOKENS));
  L.staging_stride = (int32_t)(T + W + 4);
  L.hi_page_bytes = g.hi_page_bytes;
  L.lo_page_bytes = g.lo_page_bytes;
  uint64_t off = 0;
  L.status_off = off;
  off = align_up(off + 16, kAlignSmall);
  L.counters_off = off;
  off = align_up(off + B * NL * kCounterStride * 4, kAlignSmall);
  L.block_table_off = off;
  off = align_up(off + B * NL * 2 * (uint64_t)L.max_pages * 4, kAlignSmall);
  L.index_list_off = off;
  off = align_up(off + B * NL * 2 * T * 4, kAlignSmall);
  L.staging_off = off;
  off = align_up(off + B * (uint64_t)L.staging_stride * 4, kAlignSmall);
  L.budget_off = off;
  off = align_up(off + sizeof(BudgetTable), kAlignSmall);
  L.ring_act_off = off;
  off = align_up(off + B * NL * W, kAlignPool);
  L.hi_pool_off = off;
  off = align_up(off + ((uint64_t)L.ring_pages + g.hi_pages) * L.hi_page_bytes, kAlignPool);
  L.lo_pool_off = off;
  off = align_up(off + (uint64_t)g.lo_pages * L.lo_page_bytes, kAlignPool);
  L.total_bytes = off;
  return L;
}

// The device view of a buffer laid out so; n_kv_heads and head_dim are the caller's.
inline CacheView view_regions(void* buffer, const pask_cache_layout& L, const CacheDims& g) {
  uint8_t* base = static_cast<uint8_t*>(buffer);
  CacheView v;
  v.status = reinterpret_cast<uint32_t*>(base + L.status_off);
  v.counters = reinterpret_cast<int32_t*>(base + L.counters_off);
  v.block_table = reinterpret_cast<int32_t*>(base + L.block_table_off);
  v.index_list = reinterpret_cast<int32_t*>(base + L.index_list_off);
  v.staging = reinterpret_cast<int32_t*>(base + L.staging_off);
  v.budget = reinterpret_cast<BudgetTable*>(base + L.budget_off);
  v.ring_act = base + L.ring_act_off;
  v.hi_pool = base + L.hi_pool_off;
  v.lo_pool = base + L.lo_pool_off;
  v.n_layers = g.n_layers;
  v.n_kv_heads = 1;
  v.head_dim = 0;
  v.max_tokens = g.max_tokens;
  v.max_pages = L.max_pages;
  v.hi_pages = L.ring_pages + g.hi_pages;
  v.hi_base = L.ring_pages;
  v.window = g.window;
  v.ring_pp = (g.window + PASK_PAGE_TOKENS - 1) / PASK_PAGE_TOKENS;
  v.staging_stride = L.staging_stride;
  v.lo_pages = g.lo_pages;
  v.hi_page_bytes = (uint32_t)L.hi_page_bytes;
  v.lo_page_bytes = (uint32_t)L.lo_page_bytes;
  return v;
}

// The policy by itself, and against a cache's number of layers.
inline int check_policy_layers(const pask_policy* p, int32_t n_layers) {
  if (!p) return PASK_E_ARG;
  if (p->n_tags < 1 || p->n_tags > PASK_MAX_TAGS || p->n_groups < 1 || p->n_groups > PASK_MAX_GROUPS)
    return PASK_E_POLICY;
  if ((int32_t)p->n_layers != n_layers) return PASK_E_SHAPE;
  return PASK_OK;
}
inline int check_policy_groups(const pask_policy* p) {
  for (uint32_t l = 0; l < p->n_layers; ++l)
    if (p->group_of_layer[l] >= p->n_groups) return PASK_E_POLICY;
  if (p->n_states > PASK_MAX_STATES) return PASK_E_POLICY;
  return PASK_OK;
}

inline TableColumn column_of(const pask_policy* p, int layer) {
  TableColumn t;
  memset(&t, 0, sizeof(t));
  const int c = p->group_of_layer[layer];
  for (uint32_t z = 0; z < p->n_tags; ++z) {
    t.a0[z] = p->action[z][c];
    t.amin[z] = p->floor_[z][c];
  }
  t.n_tags = p->n_tags;
  t.n_sink = p->n_sink;
  t.group = (uint32_t)c;
  return t;
}

// PASK_DEBUG set to anything but "" or "0" when the library is first used
// turns on a check after every entry point that launches kernels: it waits for
// the stream, turns a launch or execution error into PASK_E_HIP, and writes to
// stderr the entry point with the HIP error, or with the cache's device status
// flags when they differ from the last ones reported.  A failure is then named
// by the call that caused it, not by a later synchronisation.  Calls on a
// stream that is being captured into a graph are not checked.  Off by default:
// each check costs a host round trip.
inline bool debug_on() {
  static const bool on = [] {
    const char* e = getenv("PASK_DEBUG");
    return e && e[0] && strcmp(e, "0") != 0;
  }();
  return on;
}

// status: the device status words of the caches of the call.
inline int debug_check_words(const char* where, int st, const void* const* status, int n, hipStream_t stream) {
  if (st != PASK_OK || !debug_on()) return st;
  hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
  hipError_t e = hipStreamIsCapturing(stream, &cs);
  if (e == hipSuccess && cs != hipStreamCaptureStatusNone) return st;
  if (e == hipSuccess) e = hipStreamSynchronize(stream);
  if (e == hipSuccess) e = hipGetLastError();
  if (e != hipSuccess) {
    fprintf(stderr, "pask: %s: %s\n", where, hipGetErrorString(e));
    return PASK_E_HIP;
  }
  static std::atomic<uint32_t> reported{0};
  for (int i = 0; i < n; ++i) {
    uint32_t word = 0;
    if (hipMemcpyAsync(&word, status[i], sizeof(word), hipMemcpyDeviceToHost, stream) != hipSuccess ||
        hipStreamSynchronize(stream) != hipSuccess) {
      fprintf(stderr, "pask: %s: status word not readable\n", where);
      return PASK_E_HIP;
    }
    if (word != 0 && reported.exchange(word) != word)
      fprintf(stderr, "pask: %s: device status flags 0x%x\n", where, word);
  }
  return st;
}

}  // namespace pask
