// gfx950 kernels that persist latents and rotary keys by the table, and read
// them back.
//
//   latent_pack  after the plan kernel of the bulk append has slotted the
//                call's tokens: HIGH rows copied, LOW latents quantised (int4,
//                one fp16 scale per 32 elements), whole pages at a time.
//   latent_step  decision, slot and write of one token per sequence.
//   latent_read  the persisted entries of a layer as dense rows in position
//                order, packed over the batch.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pask_latent_device.h"

namespace pask {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

// A 16-byte piece of an entry: step i (32 elements), quarter q of it (8
// elements), slot t of the page.  Thread by thread in this order neighbours
// touch 64 bytes of a row, and a wave all of step i in a page.
struct Piece {
  int i, q, t;
};
__device__ __forceinline__ Piece piece(int x) { return Piece{x >> 6, x & 3, (x >> 2) & 15}; }
// Its chunk in a HIGH page, and in the rotary keys of either (i from 0 there).
__device__ __forceinline__ int chunk_of(const Piece& p) { return 64 * p.i + 16 * p.q + latent_swap(p.q, p.t); }

// The int4 codes of a quarter, in page order, with the scale of the 32
// elements that this lane and the three beside it hold.
__device__ __forceinline__ uint32_t low_word(const uint4& x, uint16_t& sbits) {
  uint32_t mb = abs_max_bits8(x);
  mb = max(mb, (uint32_t)__shfl_xor((int)mb, 1));
  mb = max(mb, (uint32_t)__shfl_xor((int)mb, 2));
  float s, inv;
  bool plain;
  sbits = quant_scale_bf16(__uint_as_float(mb << 16), s, inv, plain);
  uint32_t cb[8];
  code_bytes8(x, s, inv, plain, cb);
  return low_bytes4((cb[4] << 4) | cb[0], (cb[5] << 4) | cb[1], (cb[6] << 4) | cb[2], (cb[7] << 4) | cb[3]);
}

// Block (k, b) fills page k of the pages of sequence b that this call's slots
// reach, HIGH's first, then LOW's (the plan kernel left the counts before the
// call in the staging words).  Each slot's input row comes from the index
// list.  Every 16-byte piece and every scale belongs to one slot, so slots of
// earlier calls in a page that was already open are not touched.  The memory
// bounds it: 32 prompts of 500-8,000 tokens at rank 512, most kept as LOW, take 34 us; streaming
// stores of the pages, which are read soon, make writing and reading them back
// 103 us in place of 82, streaming loads of the rows 89.
template <int R, int P>
__global__ __launch_bounds__(kThreads) void latent_pack_kernel(AppendArgs a) {
  using PG = LatentPage<R, P>;
  __shared__ int s_src[kPage];                     // input row of each slot, -1: none of this call
  const CacheView& cv = a.cv;
  const int b = blockIdx.y, tid = (int)threadIdx.x;
  const int32_t* stg = cv.staging + (size_t)b * cv.staging_stride + cv.staging_stride - 4;
  const int32_t* cnt = counters_of(cv, b, a.layer);
  const int p0 = stg[2];
  int k = (int)blockIdx.x;
  const int n_hi = cnt[kCntHi] > stg[0] ? (cnt[kCntHi] + kPage - 1) / kPage - stg[0] / kPage : 0;
  const int st = k < n_hi ? kHi : kLo;
  k -= st == kHi ? 0 : n_hi;
  const int n0 = stg[st], n1 = cnt[st];
  const int pidx = n0 / kPage + k;
  const int t0 = max(n0 - pidx * kPage, 0), t1 = min(n1 - pidx * kPage, kPage);
  if (t0 >= t1) return;                            // block-uniform: no new slot here
  const int page = block_table_of(cv, b, a.layer, st)[pidx];
  if (tid < kPage) {
    int j = -1;
    if (tid >= t0 && tid < t1) {
      const int row = index_list_of(cv, b, a.layer, st)[pidx * kPage + tid] - p0;
      if (row >= 0 && row < a.max_new) j = row;
    }
    s_src[tid] = j;
  }
  __syncthreads();
  const uint16_t* c = a.k + (size_t)b * a.max_new * R;
  const uint16_t* r = a.v + (size_t)b * a.max_new * P;
  uint8_t* pg = st == kHi ? cv.hi_pool + (size_t)page * PG::kHiBytes : cv.lo_pool + (size_t)page * PG::kLoBytes;
  uint8_t* rope = pg + (st == kHi ? 1024 * PG::RI : PG::kRopeAt);
  constexpr int kItems = (PG::KI + kWaves - 1) / kWaves;
  uint4 v[kItems];                                 // all loads before the first store
#pragma unroll
  for (int u = 0; u < kItems; ++u) {
    const Piece p = piece(tid + u * kThreads);
    const int j = p.i < PG::KI ? s_src[p.t] : -1;
    const uint16_t* src = p.i < PG::RI ? c + (size_t)j * R + 32 * p.i : r + (size_t)j * P + 32 * (p.i - PG::RI);
    v[u] = j >= 0 ? *reinterpret_cast<const uint4*>(src + 8 * p.q) : make_uint4(0u, 0u, 0u, 0u);
  }
#pragma unroll
  for (int u = 0; u < kItems; ++u) {
    Piece p = piece(tid + u * kThreads);           // p.i is the same for a wave
    if (p.i >= PG::KI) continue;
    const bool there = s_src[p.t] >= 0;
    if (p.i >= PG::RI) {
      p.i -= PG::RI;
      if (there) *reinterpret_cast<uint4*>(rope + chunk_of(p) * 16) = v[u];
    } else if (st == kHi) {
      if (there) *reinterpret_cast<uint4*>(pg + chunk_of(p) * 16) = v[u];
    } else {
      uint16_t sbits;
      const uint32_t w = low_word(v[u], sbits);
      const int g = 16 * p.i + p.t;
      if (there) *reinterpret_cast<uint32_t*>(pg + g * 16 + 4 * p.q) = w;
      if (there && p.q == 0) *reinterpret_cast<uint16_t*>(pg + PG::kScales + 2 * g) = sbits;
    }
  }
}

// One token per sequence: thread 0 of the block decides and slots it, the
// block writes it (decide; a page is taken from the pool by the token that
// opens it).  The row's pieces are loaded before the decision is known.
template <int R, int P>
__global__ __launch_bounds__(128) void latent_step_kernel(AppendArgs a) {
  using PG = LatentPage<R, P>;
  __shared__ int s_code, s_page;
  const CacheView& cv = a.cv;
  const int b = blockIdx.x, tid = (int)threadIdx.x;
  const uint16_t* c = a.k + (size_t)b * R;
  const uint16_t* r = a.v + (size_t)b * P;
  constexpr int kChunks = 4 * PG::KI;
  static_assert(kChunks <= 128, "a chunk per thread");
  uint4 mine = make_uint4(0u, 0u, 0u, 0u);
  if (tid < 4 * PG::RI) mine = reinterpret_cast<const uint4*>(c)[tid];
  else if (tid < kChunks) mine = reinterpret_cast<const uint4*>(r)[tid - 4 * PG::RI];
  if (tid == 0) {
    uint32_t flags = 0;
    int32_t* cnt = counters_of(cv, b, a.layer);
    const int pos = cnt[kCntPos], slots[2] = {cnt[kCntHi], cnt[kCntLo]};
    const unsigned cursors[2] = {cv.status[2], cv.status[3]};
    int code = -1, page = -1;
    if (pos >= cv.max_tokens) {
      flags |= PASK_FLAG_SEQ_CAPACITY;
      cnt[kCntLost] += 1;
    } else {
      bool forced, bad;
      const int tag = a.tags ? (int)a.tags[b] : 0;
      const int act = decide(a.tab.a0, a.tab.amin, a.tab.n_tags, a.tab.n_sink, (a.flags & kKeepAll) != 0u, tag, pos,
                             forced, bad);
      if (bad) flags |= PASK_FLAG_BAD_TAG;
      cnt[kCntPos] = pos + 1;
      if (act == kDrop) {
        cnt[kCntDrop] += 1;
      } else {
        const int st = act == kHigh ? kHi : kLo, slot = slots[st];
        int32_t* entry = block_table_of(cv, b, a.layer, st) + slot / kPage;
        bool stored = true;
        if (slot % kPage == 0) {
          // A pool that was full when the call began keeps its cursor (append_plan_kernel).
          const unsigned pages = (unsigned)(st == kHi ? cv.hi_pages : cv.lo_pages);
          const unsigned pid = cursors[st] >= pages ? cursors[st] : atomicAdd(&cv.status[2 + st], 1u);
          stored = pid < pages;
          page = (int)pid;
          if (stored) *entry = page;
        } else {
          page = *entry;
        }
        if (stored) {
          index_list_of(cv, b, a.layer, st)[slot] = pos;
          cnt[st] = slot + 1;
          if (forced) cnt[kCntForced] += 1;
          code = (st << 30) | slot;
        } else {
          flags |= st == kHi ? PASK_FLAG_HI_POOL_EXHAUSTED : PASK_FLAG_LO_POOL_EXHAUSTED;
          cnt[kCntLost] += 1;
        }
      }
    }
    if (flags) atomicOr(cv.status, flags);
    s_code = code;
    s_page = page;
  }
  __syncthreads();
  if (s_code < 0) return;
  const int t = (s_code & 0x3FFFFFFF) % kPage, i = tid >> 2, q = tid & 3;
  const int at = chunk_of(Piece{i, q, t});
  if ((s_code >> 30) == kHi) {
    if (tid < kChunks)
      *reinterpret_cast<uint4*>(cv.hi_pool + (size_t)s_page * PG::kHiBytes + at * 16) = mine;
    return;
  }
  uint8_t* pg = cv.lo_pool + (size_t)s_page * PG::kLoBytes;
  uint16_t sbits;
  const uint32_t w = low_word(mine, sbits);
  if (tid < 4 * PG::RI) {
    const int g = 16 * i + t;
    *reinterpret_cast<uint32_t*>(pg + g * 16 + 4 * q) = w;
    if (q == 0) *reinterpret_cast<uint16_t*>(pg + PG::kScales + 2 * g) = sbits;
  } else if (tid < kChunks) {
    *reinterpret_cast<uint4*>(pg + PG::kRopeAt + (at - 64 * PG::RI) * 16) = mine;
  }
}

// Block (x, b) takes pages x, x + gridDim.x, ... of sequence b, HIGH's first.
// A slot's row is cu[b] + its slot + the entries of the other store at lower
// positions: of the position's predecessors those that are neither in this
// store nor kept nowhere, so between position - slot - (positions not kept)
// and position - slot, found among these.  A page's bytes are loaded first.
// The memory bounds it: 64 sequences of 100-12,000 tokens at rank 256 (327 MB in
// and out) take 96 us from memory, 61 with the pages in the last-level cache.
// Rows are stored past the caches: with plain stores, which evict pages still
// to be read, 109 and 107.  At most 16,384 blocks: with 4,096 the longest
// sequences' run alone at the end (131 us).  The blocks a compute unit holds,
// named for the compiler, which then issues a page's loads sooner (111 us
// without); at rank 512 more than five would spill (write and read 32 prompts:
// 83 us, 123 with eight).  Each block sums the counts of the sequences before its
// own, which is nothing at 1,024 sequences (13 MB in 10 us) and much at tens of
// thousands (65,535 of 20 tokens, 839 MB: 2.1 ms, with 60 layers between a
// sequence's counters and the next's 10.9).
template <int R, int P>
__global__ __launch_bounds__(kThreads, R >= 512 ? 5 : 8) void latent_read_kernel(LatentReadArgs a) {
  using PG = LatentPage<R, P>;
  __shared__ int s_cu[kWaves];
  __shared__ int s_row[2][kPage];
  const CacheView& cv = a.cv;
  const int b = blockIdx.y, tid = (int)threadIdx.x;
  int before = 0;
  for (int x = tid; x < b; x += kThreads) {
    const int32_t* o = counters_of(cv, x, a.layer);
    before += o[kCntHi] + o[kCntLo];
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) before += __shfl_xor(before, off);
  if ((tid & 63) == 0) s_cu[tid >> 6] = before;
  const int32_t* cnt = counters_of(cv, b, a.layer);
  const int n[2] = {cnt[kCntHi], cnt[kCntLo]};
  const int gone = cnt[kCntPos] - n[0] - n[1];     // positions not kept
  __syncthreads();
  int cu = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) cu += s_cu[w];
  if (blockIdx.x == 0 && tid == 0) {
    if (b == 0) a.cu[0] = 0;
    a.cu[b + 1] = cu + n[0] + n[1];
  }
  const int np_hi = (n[0] + kPage - 1) / kPage, np = np_hi + (n[1] + kPage - 1) / kPage;
  int turn = 0;
  for (int k = blockIdx.x; k < np; k += gridDim.x, turn ^= 1) {
    const int st = k < np_hi ? kHi : kLo, pidx = st == kHi ? k : k - np_hi;
    const int m = min(kPage, n[st] - pidx * kPage);
    const int page = block_table_of(cv, b, a.layer, st)[pidx];
    const int slot = pidx * kPage + (tid >> 4);    // 16 lanes for each
    const int pos = tid >> 4 < m ? index_list_of(cv, b, a.layer, st)[slot] : 0;
    const uint8_t* pg =
        st == kHi ? cv.hi_pool + (size_t)page * PG::kHiBytes : cv.lo_pool + (size_t)page * PG::kLoBytes;
    const uint8_t* rope = pg + (st == kHi ? 1024 * PG::RI : PG::kRopeAt);
    constexpr int kItems = (PG::KI + kWaves - 1) / kWaves;
    uint4 v[kItems];
    uint16_t s[kItems];
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
      Piece p = piece(tid + u * kThreads);         // p.i is the same for a wave
      if (p.i >= PG::KI) continue;
      if (p.i >= PG::RI) {
        p.i -= PG::RI;
        v[u] = *reinterpret_cast<const uint4*>(rope + chunk_of(p) * 16);
      } else if (st == kHi) {
        v[u] = *reinterpret_cast<const uint4*>(pg + chunk_of(p) * 16);
      } else {
        const int g = 16 * p.i + p.t;
        v[u].x = *reinterpret_cast<const uint32_t*>(pg + g * 16 + 4 * p.q);
        s[u] = *reinterpret_cast<const uint16_t*>(pg + PG::kScales + 2 * g);
      }
    }
    int row = -1;
    if (tid >> 4 < m) {
      const int most = pos - slot;
      row = cu + slot + entries_below(index_list_of(cv, b, a.layer, 1 - st), max(0, most - gone),
                                      min(n[1 - st], most), pos);
      if (row >= a.rows) row = -1;
    }
    if ((tid & 15) == 0) {
      s_row[turn][tid >> 4] = row;
      if (row >= 0 && a.pos) a.pos[row] = pos;
    }
    __syncthreads();                               // this turn's rows; the ones before last have been used
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
      const Piece p = piece(tid + u * kThreads);
      if (p.i >= PG::KI) continue;
      const int to = s_row[turn][p.t];
      const bool latent = p.i < PG::RI;
      uint16_t* dst = latent ? a.c + (size_t)to * R + 32 * p.i : a.r + (size_t)to * P + 32 * (p.i - PG::RI);
      const uint4 x = latent && st == kLo ? low_values(v[u].x, half_value(s[u])) : v[u];
      if (to >= 0) stream_store16(reinterpret_cast<uint8_t*>(dst + 8 * p.q), x);
    }
  }
}

// f(std::integral_constant-like tag) for the page type of (rank, rope).
template <typename F>
void with_page(int rank, int rope, F f) {
  if (rope == 32) {
    if (rank == 128) f(LatentPage<128, 32>{});
    else if (rank == 256) f(LatentPage<256, 32>{});
    else f(LatentPage<512, 32>{});
  } else {
    if (rank == 128) f(LatentPage<128, 64>{});
    else if (rank == 256) f(LatentPage<256, 64>{});
    else f(LatentPage<512, 64>{});
  }
}

}  // namespace

hipError_t launch_latent_append(const LatentAppendArgs& la, hipStream_t s) {
  const AppendArgs& a = la.base;
  if (a.max_new == 1 && a.n_new == nullptr) {
    with_page(la.rank, la.rope, [&](auto pg) {
      using PG = decltype(pg);
      latent_step_kernel<PG::kRank, PG::kRope><<<dim3(a.batch), dim3(128), 0, s>>>(a);
    });
    return hipGetLastError();
  }
  const hipError_t e = launch_append_plan(a, s);
  if (e != hipSuccess) return e;
  const dim3 grid(pack_pages(a.max_new), a.batch);
  with_page(la.rank, la.rope, [&](auto pg) {
    using PG = decltype(pg);
    latent_pack_kernel<PG::kRank, PG::kRope><<<grid, dim3(kThreads), 0, s>>>(a);
  });
  return hipGetLastError();
}

hipError_t launch_latent_read(const LatentReadArgs& a, hipStream_t s) {
  const int most = a.cv.max_pages + 1;             // pages of a sequence: both stores may end in a part
  const int per = std::max(1, std::min(most, 16384 / a.batch));
  with_page(a.rank, a.rope, [&](auto pg) {
    using PG = decltype(pg);
    latent_read_kernel<PG::kRank, PG::kRope><<<dim3(per, a.batch), dim3(kThreads), 0, s>>>(a);
  });
  return hipGetLastError();
}

}  // namespace pask
