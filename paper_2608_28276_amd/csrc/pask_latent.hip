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

constexpr int kThreads = 256;

// The int4 codes of a 32-element group (x[q]: elements 8q .. 8q + 7) in page
// order, and its scale's bits.
__device__ __forceinline__ uint4 low_group(const uint4 (&x)[4], uint16_t& sbits) {
  uint32_t mb = 0u;
#pragma unroll
  for (int q = 0; q < 4; ++q) mb = max(mb, abs_max_bits8(x[q]));
  float s, inv;
  bool plain;
  sbits = quant_scale_bf16(__uint_as_float(mb << 16), s, inv, plain);
  uint32_t w[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t cb[8];
    code_bytes8(x[q], s, inv, plain, cb);
    w[q] = low_bytes4((cb[4] << 4) | cb[0], (cb[5] << 4) | cb[1], (cb[6] << 4) | cb[2],
                      (cb[7] << 4) | cb[3]);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Block (k, b) fills page k of the pages of sequence b that this call's slots
// reach, HIGH's first, then LOW's (the plan kernel left the counts before the
// call in the staging words).  Each slot's input row comes from the index
// list.  Every 16-byte piece and every scale belongs to one slot, so slots of
// earlier calls in a page that was already open are not touched.
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
  auto rope_chunk = [&](int x, uint8_t* dst) {     // chunk x of the page's rotary keys
    const int q = (x >> 4) & 3, t = latent_swap(q, x & 15), j = s_src[t];
    if (j < 0) return;
    *reinterpret_cast<uint4*>(dst + x * 16) =
        *reinterpret_cast<const uint4*>(r + (size_t)j * P + 32 * (x >> 6) + 8 * q);
  };
  if (st == kHi) {
    uint8_t* pg = cv.hi_pool + (size_t)page * PG::kHiBytes;
    for (int x = tid; x < 64 * PG::RI; x += kThreads) {
      const int q = (x >> 4) & 3, t = latent_swap(q, x & 15), j = s_src[t];
      if (j >= 0)
        *reinterpret_cast<uint4*>(pg + x * 16) =
            *reinterpret_cast<const uint4*>(c + (size_t)j * R + 32 * (x >> 6) + 8 * q);
    }
    for (int x = tid; x < PG::kRopeChunks; x += kThreads) rope_chunk(x, pg + 1024 * PG::RI);
    return;
  }
  uint8_t* pg = cv.lo_pool + (size_t)page * PG::kLoBytes;
  for (int x = tid; x < PG::kGroups; x += kThreads) {
    const int j = s_src[x & 15];
    if (j < 0) continue;
    const uint4* src = reinterpret_cast<const uint4*>(c + (size_t)j * R + 32 * (x >> 4));
    const uint4 v[4] = {src[0], src[1], src[2], src[3]};
    uint16_t sbits;
    *reinterpret_cast<uint4*>(pg + x * 16) = low_group(v, sbits);
    *reinterpret_cast<uint16_t*>(pg + PG::kScales + 2 * x) = sbits;
  }
  for (int x = tid; x < PG::kRopeChunks; x += kThreads) rope_chunk(x, pg + PG::kRopeAt);
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
          const unsigned pid = atomicAdd(&cv.status[2 + st], 1u);
          stored = pid < (unsigned)(st == kHi ? cv.hi_pages : cv.lo_pages);
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
  const int at = 64 * i + 16 * q + latent_swap(q, t);          // the piece's chunk in a HIGH page
  if ((s_code >> 30) == kHi) {
    if (tid < kChunks)
      *reinterpret_cast<uint4*>(cv.hi_pool + (size_t)s_page * PG::kHiBytes + at * 16) = mine;
    return;
  }
  uint8_t* pg = cv.lo_pool + (size_t)s_page * PG::kLoBytes;
  if (tid < PG::RI) {                                          // a 32-element group per thread
    const uint4* src = reinterpret_cast<const uint4*>(c) + 4 * tid;
    const uint4 v[4] = {src[0], src[1], src[2], src[3]};
    uint16_t sbits;
    *reinterpret_cast<uint4*>(pg + (16 * tid + t) * 16) = low_group(v, sbits);
    *reinterpret_cast<uint16_t*>(pg + PG::kScales + 2 * (16 * tid + t)) = sbits;
  }
  if (tid >= 4 * PG::RI && tid < kChunks) *reinterpret_cast<uint4*>(pg + PG::kRopeAt + (at - 64 * PG::RI) * 16) = mine;
}

// Entries of list[0..n) below x (the list ascends).
__device__ __forceinline__ int entries_below(const int32_t* list, int n, int x) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int m = (lo + hi) >> 1;
    if (list[m] < x) lo = m + 1;
    else hi = m;
  }
  return lo;
}

// Block (x, b) takes pages x, x + gridDim.x, ... of sequence b, HIGH's first.
// A slot's row is cu[b] + its slot + the entries of the other store at lower
// positions.
template <int R, int P>
__global__ __launch_bounds__(kThreads) void latent_read_kernel(LatentReadArgs a) {
  using PG = LatentPage<R, P>;
  __shared__ int s_cu;
  __shared__ int s_row[kPage];
  const CacheView& cv = a.cv;
  const int b = blockIdx.y, tid = (int)threadIdx.x;
  if (tid == 0) s_cu = 0;
  __syncthreads();
  int before = 0;
  for (int x = tid; x < b; x += kThreads) {
    const int32_t* o = counters_of(cv, x, a.layer);
    before += o[kCntHi] + o[kCntLo];
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) before += __shfl_xor(before, off);
  if ((tid & 63) == 0 && before) atomicAdd(&s_cu, before);
  __syncthreads();
  const int32_t* cnt = counters_of(cv, b, a.layer);
  const int n[2] = {cnt[kCntHi], cnt[kCntLo]};
  const int cu = s_cu;
  if (blockIdx.x == 0 && tid == 0) {
    if (b == 0) a.cu[0] = 0;
    a.cu[b + 1] = cu + n[0] + n[1];
  }
  const int np_hi = (n[0] + kPage - 1) / kPage, np = np_hi + (n[1] + kPage - 1) / kPage;
  for (int k = blockIdx.x; k < np; k += gridDim.x) {
    const int st = k < np_hi ? kHi : kLo, pidx = st == kHi ? k : k - np_hi;
    const int m = min(kPage, n[st] - pidx * kPage);
    const int page = block_table_of(cv, b, a.layer, st)[pidx];
    __syncthreads();                               // the rows of the page before are used
    if (tid < kPage) {
      int row = -1;
      if (tid < m) {
        const int slot = pidx * kPage + tid;
        const int pos = index_list_of(cv, b, a.layer, st)[slot];
        row = cu + slot + entries_below(index_list_of(cv, b, a.layer, 1 - st), n[1 - st], pos);
        if (row >= a.rows) row = -1;
        else if (a.pos) a.pos[row] = pos;
      }
      s_row[tid] = row;
    }
    __syncthreads();
    auto rope_chunk = [&](int x, const uint8_t* src) {
      const int q = (x >> 4) & 3, row = s_row[latent_swap(q, x & 15)];
      if (row >= 0)
        *reinterpret_cast<uint4*>(a.r + (size_t)row * P + 32 * (x >> 6) + 8 * q) =
            *reinterpret_cast<const uint4*>(src + x * 16);
    };
    if (st == kHi) {
      const uint8_t* pg = cv.hi_pool + (size_t)page * PG::kHiBytes;
      for (int x = tid; x < 64 * PG::RI; x += kThreads) {
        const int q = (x >> 4) & 3, row = s_row[latent_swap(q, x & 15)];
        if (row >= 0)
          *reinterpret_cast<uint4*>(a.c + (size_t)row * R + 32 * (x >> 6) + 8 * q) =
              *reinterpret_cast<const uint4*>(pg + x * 16);
      }
      for (int x = tid; x < PG::kRopeChunks; x += kThreads) rope_chunk(x, pg + 1024 * PG::RI);
    } else {
      const uint8_t* pg = cv.lo_pool + (size_t)page * PG::kLoBytes;
      for (int x = tid; x < PG::kGroups; x += kThreads) {
        const int row = s_row[x & 15];
        if (row < 0) continue;
        const uint4 w = *reinterpret_cast<const uint4*>(pg + x * 16);
        const float s = half_value(*reinterpret_cast<const uint16_t*>(pg + PG::kScales + 2 * x));
        uint4* dst = reinterpret_cast<uint4*>(a.c + (size_t)row * R + 32 * (x >> 4));
        dst[0] = low_values(w.x, s);
        dst[1] = low_values(w.y, s);
        dst[2] = low_values(w.z, s);
        dst[3] = low_values(w.w, s);
      }
      for (int x = tid; x < PG::kRopeChunks; x += kThreads) rope_chunk(x, pg + PG::kRopeAt);
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
  const int per = std::max(1, std::min(most, 4096 / a.batch));
  with_page(a.rank, a.rope, [&](auto pg) {
    using PG = decltype(pg);
    latent_read_kernel<PG::kRank, PG::kRope><<<dim3(per, a.batch), dim3(kThreads), 0, s>>>(a);
  });
  return hipGetLastError();
}

}  // namespace pask
