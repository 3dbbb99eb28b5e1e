// How many pages a bulk append reaches, for its launch and for the checks before it.
#pragma once

#include <stdint.h>

#include <algorithm>

#include "pask.h"

namespace pask {

// Most pages that n new slots of one sequence can reach in its two stores: m
// consecutive slots reach at most (m + 14) / 16 + 1.
inline int pack_pages(int n) { return (n + 28) / PASK_PAGE_TOKENS + 2; }

// Most workgroups (256 threads) of one sequence that a kernel of a bulk append
// is launched with: the pages, or the window's slots.  A launch holds 2^32 - 1
// threads, and one that fails after the plan has counted the tokens leaves
// entries whose pages nobody wrote.
inline bool append_fits(int32_t max_new, int32_t window) {
  return std::max(pack_pages(max_new + window), std::min(max_new, window)) < 1 << 24;
}

}  // namespace pask
