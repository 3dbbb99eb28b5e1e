// gfx950 kernels of the attention of many query tokens over the mixed cache:
// bf16 pages, int4 pages and the recent window, causal by position, keys cut
// into pieces where there are few queries.
#include <hip/hip_runtime.h>

#include <float.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "pask_latent_device.h"
#include "pask_prompt_internal.h"

namespace pask {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kStepKeys = 64, kStepPages = kStepKeys / kPage;
// The reference of a row's weights lies kBelow under a maximum (in base 2) and
// moves only when a score exceeds it by more than kHeadroom: weights stay below
// 2^15, which fp16 holds, and the largest is 2^8 or more, so that what fp16
// cannot tell from 0 is 2^-33 of it.  bf16 and fp32 are as precise there as
// below 1, and the sums stay below the largest fp32 for values that sum to less
// than 2^112, the bound that the header gives.
constexpr float kHeadroom = 15.0f, kBelow = 8.0f;
constexpr int kAhead = 4;                          // score operands read ahead of their product
constexpr float kLn2 = 0.6931471805599453f;

// D[32x32] += A[32x16] B[16x32]: lane l holds A[l % 32][8 (l / 32) ..], B[8 (l / 32) ..][l % 32], and
// D[8 (r / 4) + 4 (l / 32) + r % 4][l % 32], r < 16.
__device__ __forceinline__ f32x16_t mfma(uint4 a, uint4 b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0,
                                                 0, 0);
}
__device__ __forceinline__ f32x16_t mfma_half(uint4 a, uint4 b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0,
                                                0);
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {   // round to nearest even
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){lo, hi}, f16x2_t));
}

// The kinds of pages a sequence's keys come from, in the order they are taken.
enum Kind { kLowPages = 0, kHighPages = 1, kWindowPages = 2 };

// What the keys of one (sequence, layer) are, seen from queries at positions.
struct Keys {
  const int32_t* list[2];                          // positions of the LOW and HIGH entries, ascending
  const int32_t* table[2];                         // their pages
  int n[2];                                        // entries
  int n_pos, ring_slots, ring_turn;                // positions; slots of the window in use; slot of the next position
  int ring_page;                                   // first page of the window
};

__device__ __forceinline__ Keys keys_of(const CacheView& cv, int b, int layer) {
  Keys k;
  const int32_t* cnt = counters_of(cv, b, layer);
  k.list[kLowPages] = index_list_of(cv, b, layer, kLo);
  k.list[kHighPages] = index_list_of(cv, b, layer, kHi);
  k.table[kLowPages] = block_table_of(cv, b, layer, kLo);
  k.table[kHighPages] = block_table_of(cv, b, layer, kHi);
  k.n[kLowPages] = cnt[kCntLo];
  k.n[kHighPages] = cnt[kCntHi];
  k.n_pos = cnt[kCntPos];
  k.ring_slots = min(k.n_pos, cv.window);
  k.ring_turn = cv.window ? k.n_pos % cv.window : 0;
  k.ring_page = (int)sl_index(cv, b, layer) * cv.ring_pp;
  return k;
}
// The sequence that has the b-th most entries, so that a call whose workgroups
// take turns begins with the longest, where the sequences are few enough to rank
// in a wave's lanes (64 drafts behind 1,024-8,192 entries: bf16 235 us in the
// sequences' own order, 209 so, int4 175 and 139; 16 equal prompts 107 and 111).
// Larger batches keep their order: 96 drafts take 208 us, 186 where the caller has
// put the longest first, 96 turns of 4-64 tokens 253 and 198.
__device__ __forceinline__ int by_length(const PromptArgs& a, int b) {
  if (a.batch == 1 || a.batch > 64 || gridDim.x <= 256) return b;
  const int lane = (int)threadIdx.x & 63;
  const int32_t* cnt = counters_of(a.cv, min(lane, a.batch - 1), a.layer);
  const int n = lane < a.batch ? cnt[kCntHi] + cnt[kCntLo] : -1;
  int before = 0;
  for (int y = 0; y < a.batch; ++y) {
    const int other = __builtin_amdgcn_readlane(n, y);
    before += other > n || (other == n && y < lane);
  }
  return __builtin_amdgcn_readfirstlane((int)__ffsll((unsigned long long)__ballot(lane < a.batch && before == b)) - 1);
}
// Position held by slot s of the window; INT64_MAX for a slot not in use.
__device__ __forceinline__ long long ring_position(const Keys& k, int window, int s) {
  if (s >= k.ring_slots) return INT64_MAX;
  return (long long)k.n_pos - k.ring_turn + s - (s < k.ring_turn ? 0 : window);
}
// Entries of a list at position p or before.  An entry is one position, so no
// more than the positions behind p lie behind it, and no more than p + 1 before.
__device__ __forceinline__ int entries_at(const int32_t* list, int n, int n_pos, long long p) {
  if (p >= n_pos - 1) return n;
  if (p < 0) return 0;
  const int x = (int)p + 1;
  return entries_below(list, max(0, n - (n_pos - x)), min(n, x), x);
}

// Pairs of fp16 in a word.
__device__ __forceinline__ f16x2_t halves(uint32_t w) { return __builtin_bit_cast(f16x2_t, w); }
__device__ __forceinline__ uint32_t word_of(f16x2_t h) { return __builtin_bit_cast(uint32_t, h); }
// Codes of a word as fp16 (1024 + n has its last bit at 1): pair x holds the nibbles x = 0: 0 and 4, 1: 2 and 6,
// 2: 1 and 5, 3: 3 and 7, that is the elements 0 and 2, 1 and 3, 4 and 6, 5 and 7 of a key's eight, or slots 0 and 2, 1
// and 3 of a value's dimension, then of the one 16 on.
__device__ __forceinline__ f16x2_t code_pair(uint32_t w, int x) {
  const uint32_t n = (w >> (x == 0 ? 0 : x == 1 ? 8 : x == 2 ? 4 : 12)) & 0x000F000Fu;
  return halves(n | 0x64006400u) - halves(0x64086408u);
}

// The same pairs as 16 + code + 8 (its last bit at 1 / 64): times a scale of 8
// bits or fewer, less 24 scales (24 has 2 bits, fp16 11), is exact.
__device__ __forceinline__ f16x2_t raised_pair(uint32_t w, int x) {
  const uint32_t n = (x == 0 ? w << 6 : x == 1 ? w >> 2 : x == 2 ? w << 2 : w >> 6) & 0x03C003C0u;
  return halves(n | 0x4C004C00u);
}
// A key's 8 codes times a scale pair.
__device__ __forceinline__ uint4 key_part(uint32_t w, f16x2_t s) {
  const f16x2_t s24 = s * (f16x2_t){(_Float16)-24.0f, (_Float16)-24.0f};
  auto pair = [&](int x) { return word_of(__builtin_elementwise_fma(raised_pair(w, x), s, s24)); };
  return make_uint4(pair(0), pair(1), pair(2), pair(3));
}

// Codes and scales of one thread's share of a LOW page: quarter q of slot t's
// key (NG words of 8 elements, slot t's NG scales), or 4 slots of NG pairs of
// dimensions (e + 32 i, + 16) of the values (4 slots' NG scales).
template <int D>
struct LowPart {
  static constexpr int NG = PageLayout<D>::NG;
  uint32_t code[NG];
  uint32_t scale[2 * NG];                          // keys: the first NG / 2
};
// A scale above this (fp16 bits of 2728) is wide: it is taken at 1 / 32, which
// is exact there, so that 24 scales, and 7, are below the largest fp16.  The
// other scales stay as they are (at 1 / 32 the small ones would lose bits), so
// wide groups have products of their own, between a factor of 1 / 32 and one of
// 32 on the sums.  That is slow, and rare: 8,192 queries over as many int4 tokens,
// every scale wide, take 3,600 us where others take 827, 64 drafts 432 and 138.
constexpr uint32_t kWideScale = 0x6954u;
constexpr float kWide = 32.0f;
// Of a word's two scales those that are wide, as a mask.
__device__ __forceinline__ uint32_t wide_mask(uint32_t scales) {
  return ((uint32_t)((int)(kWideScale - (scales & 0xFFFFu)) >> 31) & 0xFFFFu) |
         ((uint32_t)((int)(kWideScale - (scales >> 16)) >> 31) << 16);
}
__device__ __forceinline__ uint32_t at_1_32(uint32_t scales) {
  return word_of(halves(scales) * (f16x2_t){(_Float16)(1.0f / kWide), (_Float16)(1.0f / kWide)});
}
// The scales that one of a wide page's two products takes: the wide ones' or the others', 0 for the rest.
__device__ __forceinline__ uint32_t scales_of(bool wide, uint32_t scales) {
  const uint32_t m = wide_mask(scales);
  return wide ? at_1_32(scales) & m : scales & ~m;
}

// O += P V key by key over 32 keys (values of pages at v0 and v1), where a value
// that some query does not see is infinite or NaN (a weight of 0 times it is
// not 0): only what a query sees is added.  Lane (g, n) holds the weights of
// query n for half of the keys, and which of them are hidden; lane (1 - g, n)
// the others'.
template <int VT>
__device__ __forceinline__ void add_seen_values(const uint8_t* v0, const uint8_t* v1, f32x16_t s, uint32_t hidden,
                                                f32x16_t (&o)[VT], int g, int n) {
#pragma unroll 1
  for (int x = 0; x < 16; ++x) {
    asm volatile("" : "+v"(g));                    // no code: keeps this rare path's addresses out of the loops around it
    const float mine = s[0];
#pragma unroll
    for (int r = 0; r < 15; ++r) s[r] = s[r + 1];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const float p = __shfl(mine, n + 32 * w);
      const bool skip = (__shfl(hidden, n + 32 * w) >> x & 1u) != 0u;
      const int t = 8 * (x >> 2) + 4 * w + (x & 3);
      if (skip) continue;
#pragma unroll
      for (int m = 0; m < VT; ++m)
#pragma unroll
        for (int r = 0; r < 16; ++r) {             // element 32 m + d
          const int d = 8 * (r >> 2) + 4 * g + (r & 3);
          const uint8_t* at = (t & 16 ? v1 : v0) + m * 1024 + ((t & 15) >> 2) * 256 + (d & 15) * 16 + (d >> 4) * 8 + (t & 3) * 2;
          o[m][r] += p * bf16_lo(*reinterpret_cast<const uint16_t*>(at));
        }
    }
  }
}

// A row's queries as operands: lane (g, n) holds the chunks 2 i + g of row n.
// Scores are scaled by |scale|; its sign goes to the queries, so that a score's
// maximum is a scaled one's.  For LOW keys they are fp16, in code_pair's order,
// the row's largest at 2^14 .. and `scale` taken along.
template <bool kLow, int KI>
__device__ __forceinline__ void load_queries(const PromptArgs& a, size_t q_row, bool in, int g, uint4 (&qf)[KI], float& scale) {
  const uint32_t flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;
  const uint16_t* qrow = a.q + q_row * (16 * KI) + 8 * g;
  uint32_t most = 0u;
#pragma unroll
  for (int i = 0; i < KI; ++i) {
    qf[i] = in ? *reinterpret_cast<const uint4*>(qrow + 16 * i) : make_uint4(0u, 0u, 0u, 0u);
    if (kLow) most = max(most, abs_max_bits8(qf[i]));
    qf[i] = make_uint4(qf[i].x ^ flip, qf[i].y ^ flip, qf[i].z ^ flip, qf[i].w ^ flip);
  }
  scale = fmaxf(fabsf(a.scale_log2), FLT_MIN);     // above 0, so that a hidden score of -inf stays that
  if constexpr (kLow) {
    most = max(most, (uint32_t)__shfl_xor((int)most, 32));
    const int up = 14 - ((int)(most >> 7) - 127);
    auto two = [&](float x, float y) { return pack_half2(ldexpf(x, up), ldexpf(y, up)); };
#pragma unroll
    for (int i = 0; i < KI; ++i) {
      const uint4 q = qf[i];
      qf[i] = make_uint4(two(bf16_lo(q.x), bf16_lo(q.y)), two(bf16_hi(q.x), bf16_hi(q.y)),
                         two(bf16_lo(q.z), bf16_lo(q.w)), two(bf16_hi(q.z), bf16_hi(q.w)));
    }
    scale = fmaxf(ldexpf(scale, -up), FLT_MIN);
  }
}
// Weights of a page's 16 slots as an operand; for LOW values in code_pair's order.
template <bool kLow>
__device__ __forceinline__ uint4 packed_weights(const f32x16_t& s, int h) {
  const int r = 8 * h;
  if constexpr (kLow)
    return make_uint4(pack_half2(s[r], s[r + 2]), pack_half2(s[r + 1], s[r + 3]), pack_half2(s[r + 4], s[r + 6]),
                      pack_half2(s[r + 5], s[r + 7]));
  return make_uint4(pack_bf16x2(s[r], s[r + 1]), pack_bf16x2(s[r + 2], s[r + 3]), pack_bf16x2(s[r + 4], s[r + 5]),
                    pack_bf16x2(s[r + 6], s[r + 7]));
}
// What packed_weights<false>' rounding left (p: its result), as an operand too: of a weight 2^-16 is lost with both.
__device__ __forceinline__ uint4 weights_rest(const f32x16_t& s, int h, uint4 p) {
  const int r = 8 * h;
  auto two = [&](int x, uint32_t w) { return pack_bf16x2(s[x] - bf16_lo(w), s[x + 1] - bf16_hi(w)); };
  return make_uint4(two(r, p.x), two(r + 2, p.y), two(r + 4, p.z), two(r + 6, p.w));
}
typedef __attribute__((address_space(3))) uint32_t lds_u32;
__device__ __forceinline__ uint32_t read_lds4(uint32_t lds) { return *(const lds_u32*)(uintptr_t)lds; }
// N words of LDS, aligned to all of them up to 16 bytes.
template <int N>
__device__ __forceinline__ void read_words(uint32_t lds, uint32_t (&x)[N]) {
  if constexpr (N == 1) {
    x[0] = read_lds4(lds);
  } else if constexpr (N == 2) {
    const u32x2_t v = *(const lds_u32x2*)(uintptr_t)lds;
    x[0] = v[0];
    x[1] = v[1];
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const uint4 v = read_lds16(lds + 4 * i);
      x[i] = v.x;
      x[i + 1] = v.y;
      x[i + 2] = v.z;
      x[i + 3] = v.w;
    }
  }
}
// Copies into LDS: all but the last N that the wave issued have arrived.
template <int N>
__device__ __forceinline__ void wait_copies() {
  static_assert(N < 64, "vmcnt has 6 bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
  asm volatile("" ::: "memory");
}
// The wave's reads of LDS so far are done.
__device__ __forceinline__ void lds_barrier_wave() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);              // lgkmcnt(0)
  asm volatile("" ::: "memory");
}

// A workgroup of W waves takes 32 W rows of one KV head, row x being head x % G
// of the group's G at query token x / G, through the keys that the tile sees,
// 64 at a step, 32 at a time:
//   scores  S^T = K Q^T on v_mfma_f32_32x32x16_bf16: a lane holds scores of one
//           row, so its softmax needs one exchange (with the lane 32 on);
//   weights online softmax in base 2, rounded once to the type of the values
//           (bf16: half a step, 2^-8 of a weight; a second product of what that
//           leaves takes 8,192 bf16 tokens from 538 us to 710); sums are kept of
//           the unrounded weights;
//   values  O^T += V^T P^T.
// Pages lie in the order of 16-row operands; the operands of 32 rows are the
// same 16-byte chunks of two pages (keys), and 8-byte halves of them (values:
// the scores' lane layout is the operand layout of P up to the order of the 16
// slots of a page, which two halves 512 bytes apart follow).  So HIGH pages go
// to LDS as they lie, and every operand read is contiguous.
// LOW pages are widened to fp16 on the way, once for all rows of the workgroup,
// by packed products.  A key is code * (s8 + s3), the scale's upper 8 bits and
// its last 3: two exact fp16, whose scores take twice the products (half as many
// again in all); a value is rounded once (half a step, 2^-11) and meets weights
// of fp16.  The queries become fp16 too, each row at the power of two that takes
// its largest element below 2^15 (exact for elements down to 2^-28 of it).  Keys
// of one bf16 made the outputs of int4 histories 3.4e-3 of their size wrong and
// lse 3e-5; outputs of bf16 pages are 2.1e-3 wrong, most of it their own rounding.
// The scores of the next 32 keys are computed beside the weights of the current
// ones; two steps are on their way into a ring of three LDS buffers meanwhile.
// The keys that a row sees are, in each store, those up to a place of its list;
// in the window, a ring, those whose position is not behind the row's.
template <int D, int G, int W>
__global__ __launch_bounds__(64 * W, W / 4) void prompt_kernel(PromptArgs a) {
  using L = PageLayout<D>;
  constexpr int kRows = 32 * W, VT = D / 32, KI = D / 16, NG = L::NG;
  // A page in LDS: keys, the rest of LOW keys, values.
  constexpr int kPart = L::kHiV, kValues = 2 * kPart, kTile = 3 * kPart, kStep = kStepPages * kTile;
  __shared__ __align__(1024) uint8_t s_kv[3][kStep];
  // LOW parts (keys, values of a page) with a wide scale; of those, which slots' scale is, for each group.
  __shared__ __align__(16) uint32_t s_wide[3 * 2 * kStepPages], s_wide_slots[3 * 2 * kStepPages][NG];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int g = lane >> 5, n = lane & 31;
  // Workgroups go to the 8 XCDs in turn: neighbours are different KV heads.  The
  // last tiles of all sequences first, then the ones before them, so that the
  // tiles that end the call see the fewest keys (4 chunks of 1,123-4,096 queries
  // behind 2,258-8,192 tokens: 2,227 us with the tiles of highest number first,
  // whichever sequence they are of, 1,677 so).
  int rest = (int)blockIdx.x;
  const int head = rest % a.cv.n_kv_heads;
  rest /= a.cv.n_kv_heads;
  const int piece = rest % a.pieces;
  rest /= a.pieces;
  const int b = by_length(a, rest % a.batch), nq = a.n_q ? min(max(a.n_q[b], 0), a.max_q) : a.max_q, n_rows = nq * G;
  const int tile0 = ((n_rows + kRows - 1) / kRows - 1 - rest / a.batch) * kRows;
  if (tile0 < 0) return;
  const Keys keys = keys_of(a.cv, b, a.layer);
  const long long first = a.first ? (long long)a.first[b] : (long long)keys.n_pos - nq;
  const int row0 = tile0 + wave * 32, row = row0 + n;
  const bool in = row < n_rows;
  // Entries of each list that the tile's last row sees and the wave's first, 16
  // lanes for each of the four; and, one per lane, the positions of the next 32
  // of both lists: the wave's rows see at most its tokens' number more.
  const long long tile_at = first + (min(tile0 + kRows, n_rows) - 1) / G, wave_at = first + row0 / G;
  const long long wave_end = first + (min(row0 + 32, n_rows) - 1) / G;
  const int seen = entries_at(lane < 32 ? keys.list[0] : keys.list[1], lane < 32 ? keys.n[0] : keys.n[1], keys.n_pos,
                              lane & 16 ? wave_at : tile_at);
  const int n_see[2] = {__builtin_amdgcn_readlane(seen, 0), __builtin_amdgcn_readlane(seen, 32)};
  const int first_of[2] = {__builtin_amdgcn_readlane(seen, 16), __builtin_amdgcn_readlane(seen, 48)};
  const int near_at = (g ? first_of[1] : first_of[0]) + n;
  const bool is_near = row0 < n_rows && near_at < (g ? n_see[1] : n_see[0]);
  const int near = is_near ? (g ? keys.list[1] : keys.list[0])[near_at] : 0;
  auto more_at = [&](long long p) { return __ballot(is_near && (long long)near <= p); };   // LOW entries below, HIGH above
  const unsigned long long last = more_at(wave_end);
  const int first_sees[2] = {row0 < n_rows ? first_of[0] : 0, row0 < n_rows ? first_of[1] : 0};
  const int last_sees[2] = {first_sees[0] + (int)__popc((uint32_t)last), first_sees[1] + (int)__popc((uint32_t)(last >> 32))};
  const bool ring_seen = keys.ring_slots > 0 && tile_at >= (long long)keys.n_pos - keys.ring_slots;
  const int low_steps = (n_see[kLowPages] + kStepKeys - 1) / kStepKeys;
  const int high_steps = (n_see[kHighPages] + kStepKeys - 1) / kStepKeys;
  const int ring_steps = ring_seen ? (keys.ring_slots + kStepKeys - 1) / kStepKeys : 0;
  const int steps = low_steps + high_steps + ring_steps;
  const int j_begin = (int)((long long)steps * piece / a.pieces), j_end = (int)((long long)steps * (piece + 1) / a.pieces);

  uint4 qf[KI];
  float scale = 0.0f;                              // of the lane's row, as its queries are held
  const size_t q_row = (((size_t)b * a.max_q + (in ? row / G : 0)) * a.n_q_heads + (size_t)head * G + (in ? row % G : 0));

  // The kind of the tile's step j and its first page.
  auto kind_of = [&](int j) { return j < low_steps ? kLowPages : j < low_steps + high_steps ? kHighPages : kWindowPages; };
  auto page0_of = [&](int j, int kind) {
    return kStepPages * (j - (kind == kLowPages ? 0 : kind == kHighPages ? low_steps : low_steps + high_steps));
  };
  // Where the head's part of a step's pages starts, 16 steps at a time, one page
  // per lane; pages behind the last one, and steps behind the last one, repeat it.
  uint32_t from_lo = 0, from_hi = 0;
  int from_of = -1;                                // which 16 steps
  auto look_up = [&](int j) __attribute__((always_inline)) {
    if ((j >> 4) == from_of) return;
    from_of = j >> 4;
    const int jl = min((j & ~15) + (lane >> 2), j_end - 1), kind = kind_of(jl), p = page0_of(jl, kind) + (lane & 3);
    const int page = kind == kWindowPages ? keys.ring_page + min(p, a.cv.ring_pp - 1)
                     : kind == kLowPages  ? keys.table[0][min(p, (n_see[0] - 1) >> 4)]
                                          : keys.table[1][min(p, (n_see[1] - 1) >> 4)];
    const uint32_t hs = ((uint32_t)head + (uint32_t)page) % (uint32_t)a.cv.n_kv_heads;
    const uint64_t at = kind == kLowPages ? (uint64_t)a.cv.lo_pool + (uint64_t)page * a.cv.lo_page_bytes + hs * (uint32_t)L::kLoHead
                                          : (uint64_t)a.cv.hi_pool + (uint64_t)page * a.cv.hi_page_bytes + hs * (uint32_t)L::kHiHead;
    from_lo = (uint32_t)at;
    from_hi = (uint32_t)(at >> 32);
  };
  auto page_at = [&](int j, int k) {               // page k of step j, looked up
    const int l = (j & 15) * kStepPages + k;
    return reinterpret_cast<const uint8_t*>((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)from_hi, l) << 32 |
                                            (uint32_t)__builtin_amdgcn_readlane((int)from_lo, l));
  };
  // Copies of a HIGH or window step into LDS: instruction x of kCopies of this wave.
  constexpr int kInstr = L::kHiHead / 1024, kCopies = (kStepPages * kInstr + W - 1) / W;   // 1 KiB each; of a page
  auto copy = [&](int j, int k) __attribute__((always_inline)) {
    const int x = wave + k * W, y = x % kInstr;
    copy_to_lds<false>(page_at(j, x / kInstr), (uint32_t)(y * 1024 + lane * 16),
                lds_address(s_kv[0]) + j % 3 * kStep + (x / kInstr) * kTile + y * 1024 + (y < kInstr / 2 ? 0 : kValues - kPart));
  };
  // A LOW step's parts of this wave: part x is the keys (x even) or values of page x / 2.
  constexpr int kParts = (2 * kStepPages + W - 1) / W;
  LowPart<D> low[kParts];
  auto fetch = [&](auto low_too, int j) __attribute__((always_inline)) {
    if (j >= j_end) return;
    look_up(j);
    if (decltype(low_too)::value && kind_of(j) == kLowPages) {
#pragma unroll
      for (int k = 0; k < kParts; ++k) {
        const int x = wave + k * W;
        const uint8_t* src = page_at(j, x >> 1);
        const bool values = (x & 1) != 0;
        const uint32_t* code = reinterpret_cast<const uint32_t*>(src + (values ? L::kLoVC : 0)) + lane * NG;
        const uint32_t* scale_at = reinterpret_cast<const uint32_t*>(src + (values ? L::kLoVS : L::kLoKS));
        scale_at += values ? (lane >> 4) * 2 * NG : (lane & 15) * (NG / 2);
#pragma unroll
        for (int i = 0; i < NG; ++i) low[k].code[i] = code[i];
#pragma unroll
        for (int i = 0; i < 2 * NG; ++i)
          if (i < NG / 2 || values) low[k].scale[i] = scale_at[i];
      }
      return;
    }
#pragma unroll
    for (int k = 0; k < kCopies; ++k) copy(j, k);
  };
  // A LOW step's arrived parts into its buffer, widened; slots behind the last entry as 0.
  auto land = [&](int j) __attribute__((always_inline)) {
    if (j >= j_end || kind_of(j) != kLowPages) return;
    const uint32_t dst = lds_address(s_kv[j % 3]);
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      const int x = wave + k * W, p = x >> 1;
      const bool values = (x & 1) != 0;
      const int slots = keys.n[kLowPages] - (page0_of(j, kLowPages) + p) * kPage;   // of the page in use
      uint32_t (&sc)[2 * NG] = low[k].scale;
      if (slots < kPage) {
#pragma unroll
        for (int c = 0; c < 2 * NG; ++c)
          if ((values ? (lane >> 4) * 4 + c / (NG / 2) : lane & 15) >= slots) sc[c] = 0u;
      }
      typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
      u16x2_t most = __builtin_bit_cast(u16x2_t, sc[0]);
#pragma unroll
      for (int c = 1; c < 2 * NG; ++c)
        if (c < NG / 2 || values) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2_t, sc[c]));
      const bool wide = __ballot(max(most[0], most[1]) > kWideScale) != 0ull;
      if (__builtin_expect(wide, 0)) {
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          uint32_t of = 0u;                        // of the lane's slots those wide in group i, one bit each
#pragma unroll
          for (int t = 0; t < 4; ++t)
            if (t == 0 || values) of |= wide_mask(sc[t * (NG / 2) + i / 2]) >> (16 * (i & 1)) & 1u << t;
          if (values) {                            // lane 16 y's slots 4 y ..
            of <<= lane >> 4 << 2;
            of |= (uint32_t)__shfl_xor((int)of, 16);
            of |= (uint32_t)__shfl_xor((int)of, 32);
          } else {                                 // lane t's slot t
            of = (uint32_t)__ballot(of != 0u) & 0xFFFFu;
          }
          if (lane == 0) s_wide_slots[2 * kStepPages * (j % 3) + x][i] = of;
        }
#pragma unroll
        for (int c = 0; c < 2 * NG; ++c) {
          const uint32_t m = wide_mask(sc[c]);
          sc[c] = (at_1_32(sc[c]) & m) | (sc[c] & ~m);
        }
      }
      if (lane == 0) s_wide[2 * kStepPages * (j % 3) + x] = wide;
      const uint32_t at = dst + p * kTile + (values ? kValues : 0) + lane * 16;
      if (values) {
#pragma unroll
        for (int i = 0; i < NG; ++i) {             // half i of slot t's NG: of words (NG / 2) t + i / 2
          const uint32_t pick = i & 1 ? 0x07060302u : 0x05040100u;
          auto scales = [&](int t) {               // of slots t and t + 2
            return halves(__builtin_amdgcn_perm(sc[(t + 2) * (NG / 2) + i / 2], sc[t * (NG / 2) + i / 2], pick));
          };
          const uint32_t w = low[k].code[i];
          write_lds16(at + i * 1024, make_uint4(word_of(code_pair(w, 0) * scales(0)), word_of(code_pair(w, 1) * scales(1)),
                                                word_of(code_pair(w, 2) * scales(0)), word_of(code_pair(w, 3) * scales(1))));
        }
      } else {
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          const uint32_t pick = i & 1 ? 0x03020302u : 0x01000100u;
          const uint32_t both = __builtin_amdgcn_perm(sc[i / 2], sc[i / 2], pick), upper = both & 0xFFF8FFF8u;
          const f16x2_t s8 = halves(upper), s3 = halves(both) - s8;
          const uint32_t w = low[k].code[i];
          write_lds16(at + i * 1024, key_part(w, s8));
          write_lds16(at + kPart + i * 1024, key_part(w, s3));
        }
      }
    }
  };

  f32x16_t o[VT];
#pragma unroll
  for (int m = 0; m < VT; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[m][r] = 0.0f;
  float mx = -INFINITY, sum = 0.0f;                // the reference (of scaled scores), the weights' sum
  // Operand addresses in a unit of two pages: keys' chunk (2 i + g) of slot n, i < KI, at 512 i; values' halves of
  // page h and dimensions 32 m .. at h * kTile + 1024 m, and 512 behind.
  const uint32_t k_at = (uint32_t)((n >> 4) * kTile + g * 256 + (n & 15) * 16);
  const uint32_t v_at = (uint32_t)(kValues + g * 256 + (n & 15) * 16 + (n >> 4) * 8);
  int slot = j_begin % 3;                          // buffer of the current unit's step
  auto after = [](int s) { return s == 2 ? 0 : s + 1; };
  auto unit_at = [&](int s, int i) { return lds_address(s_kv[0]) + s * kStep + (i & 1) * 2 * kTile; };
  // Two reads of 8 bytes, as 4.1 cycles, where one instruction of both (ds_read2st64_b64) takes 8.1.
  auto value_operand = [&](uint32_t vs, uint32_t vs2, int h, int m) {
    const u32x2_t x = *(const lds_u32x2*)(uintptr_t)(vs + h * kTile + m * 1024);
    const u32x2_t y = *(const lds_u32x2*)(uintptr_t)(vs2 + h * kTile + m * 1024);
    return make_uint4(x[0], x[1], y[0], y[1]);
  };
  // Operand k of a unit's scores: with LOW keys each part of the queries meets both of the key.
  auto key_operand = [&](auto is_low, uint32_t ks, int k) {
    return read_lds16(decltype(is_low)::value ? ks + 512 * (k >> 1) + (k & 1) * kPart : ks + 512 * k);
  };
  auto query_operand = [&](auto is_low, int k) { return qf[decltype(is_low)::value ? k >> 1 : k]; };
  auto add_product = [&](auto is_low, uint4 v, uint4 p, f32x16_t c) {
    return decltype(is_low)::value ? mfma_half(v, p, c) : mfma(v, p, c);
  };
  auto scores = [&](auto is_low, int i) __attribute__((always_inline)) {
    constexpr int kProducts = decltype(is_low)::value ? 2 * KI : KI;
    f32x16_t s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.0f;
    const uint32_t ks = fresh(unit_at(slot, i) + k_at);
    uint4 ring[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) ring[k] = key_operand(is_low, ks, k);
#pragma unroll
    for (int k = 0; k < kProducts; ++k) {
      s = add_product(is_low, ring[k % kAhead], query_operand(is_low, k), s);
      if (k + kAhead < kProducts) ring[k % kAhead] = key_operand(is_low, ks, k + kAhead);
      __builtin_amdgcn_sched_barrier(0);
    }
    return s;
  };
  // The same of LOW keys with wide groups: the other groups' products, then theirs at 1 / 32.
  auto wide_scores = [&](int i) __attribute__((always_inline)) {
    f32x16_t s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.0f;
#pragma unroll 1
    for (int wide = 0; wide < 2; ++wide) {
      const int l = fresh(lane);                   // the part: keys of the page of the lane's slot
      const int part = 2 * kStepPages * slot + 4 * (i & 1) + 2 * (l >> 4 & 1);
      const uint32_t ks = fresh(unit_at(slot, i) + k_at), some = s_wide[part] ? 1u << (l & 15) : 0u;
      const uint32_t* slots_of = s_wide_slots[part];
#pragma unroll
      for (int k = 0; k < 2 * KI; ++k) {
        const uint32_t take = ((slots_of[k / 4] & some) != 0u) == (wide != 0) ? ~0u : 0u;
        const uint4 x = key_operand(std::true_type{}, ks, k);
        s = mfma_half(make_uint4(x.x & take, x.y & take, x.z & take, x.w & take), qf[k >> 1], s);
        __builtin_amdgcn_sched_barrier(0);
      }
      s *= wide ? kWide : 1.0f / kWide;
    }
    return s;
  };
  auto highest = [&](const f32x16_t& s) {          // of the lane's part of its row, scaled
    float top = fmaxf(s[0], s[1]);
#pragma unroll
    for (int r = 2; r < 16; ++r) top = fmaxf(top, s[r]);
    return top == -INFINITY ? top : top * scale;
  };
  auto exceeds = [&](float top) { return __ballot(top > mx + kHeadroom) != 0ull; };
  auto refer = [&](float top) __attribute__((always_inline)) {   // the reference follows a maximum that exceeds it
    top = fmaxf(top, __shfl_xor(top, 32));
    const float ref = top > mx + kHeadroom ? top - kBelow : mx;
    const float alpha = ref == mx ? 1.0f : __builtin_amdgcn_exp2f(mx - ref);
    sum *= alpha;
#pragma unroll
    for (int m = 0; m < VT; ++m) o[m] *= alpha;
    mx = ref;
  };
  // The weights' base: 0 while every score was -Inf (their weights are 0, and -Inf - -Inf is not).
  auto base_of_weights = [&] { return mx == -INFINITY ? 0.0f : mx; };
  auto any_wide = [&](int s) {
    const uint4* parts = reinterpret_cast<const uint4*>(s_wide + 2 * kStepPages * s);
    const uint4 x = parts[0], y = parts[1];
    return __builtin_amdgcn_readfirstlane((int)(x.x | x.y | x.z | x.w | y.x | y.y | y.z | y.w)) != 0;
  };

  // Units of 32 keys.  After a step's first unit the workgroup meets: the next
  // step has arrived (a LOW one is widened into its buffer), and the buffer of
  // the step before is free for the step after next.
  auto meet = [&](auto is_low, int j) __attribute__((always_inline)) {
    wait_loads();
    if (decltype(is_low)::value) land(j + 1);      // LOW steps come first
    __syncthreads();
  };
  if (j_begin < j_end) {
    fetch(std::true_type{}, j_begin);
    wait_loads();
    land(j_begin);
    __syncthreads();
    fetch(std::true_type{}, j_begin + 1);
  }
  // Unit i's scores s become weights and add its values, beside the scores of unit i + 1.
  float base = 0.0f, odd_sum = 0.0f, top = -INFINITY;
  auto turn = [&](auto is_low, auto is_odd, int j_next, f32x16_t& s, f32x16_t& next) __attribute__((always_inline)) {
    constexpr int kProducts = decltype(is_low)::value ? 2 * KI : KI, kAll = kProducts + 2 * VT;
    constexpr bool kOdd = decltype(is_odd)::value;
    const uint32_t ks = fresh(unit_at(kOdd ? after(slot) : slot, kOdd ? 0 : 1) + k_at);
    const uint32_t vs = fresh(unit_at(slot, kOdd ? 1 : 0) + v_at), vs2 = fresh(vs + 512);
    auto operand = [&](int x) {
      return x < kProducts ? key_operand(is_low, ks, x) : value_operand(vs, vs2, (x - kProducts) / VT, (x - kProducts) % VT);
    };
#pragma unroll
    for (int r = 0; r < 16; ++r) next[r] = 0.0f;
    uint4 ring[kAhead], p = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int x = 0; x < kAhead; ++x) ring[x] = operand(x);
    // Pinned order: a product, the read of an operand to come, a part of the weights.
#pragma unroll
    for (int x = 0; x < kAll; ++x) {
      if (x >= kProducts && (x - kProducts) % VT == 0) p = packed_weights<decltype(is_low)::value>(s, (x - kProducts) / VT);
      if (x < kProducts) {
        next = add_product(is_low, ring[x % kAhead], query_operand(is_low, x), next);
      } else {
        const int m = (x - kProducts) % VT;
        o[m] = add_product(is_low, ring[x % kAhead], p, o[m]);
      }
      if (x + kAhead < kAll) ring[x % kAhead] = operand(x + kAhead);
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (r * (kProducts + VT - 1) / 16 == x) {  // the first 8 before the first values, all before the second's
          s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], scale, -base));
          if (r & 1) odd_sum += s[r];
          else sum += s[r];
        }
      if (x == kProducts + VT) top = highest(next);
      // The step after next, in the odd unit, its copies between the products: issued together behind the barrier they
      // and their addresses took a fifth of the call.
      if (kOdd && !decltype(is_low)::value && x % 3 == 1 && x / 3 < kCopies) copy(j_next, x / 3);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  int i = 2 * j_begin;
  // The units of one kind up to u1; u0: its first.  fs, ls: entries that the wave's first and last row see; used: of its
  // slots.
  auto segment = [&](auto is_low, bool ring, int u0, int u1, int fs, int ls, int used) __attribute__((always_inline)) {
    const long long at = first + (in ? row / G : 0);
    int sees = fs;                                 // entries that the lane's row sees
    if (ls > fs) {
#pragma unroll 1
      for (int x = 0; x < 32 / G; ++x) {
        const unsigned long long c = more_at(wave_at + x);
        if (at == wave_at + x) sees = fs + (int)__popc((uint32_t)(decltype(is_low)::value ? c : c >> 32));
      }
    }
    if (!in) sees = 0;
    const int whole = min(u1, u0 + fs / 32);       // the units that all rows of the wave see whole
    while (i < u1) {
      f32x16_t s;
      // Steps whose units are whole, up to a wide page.
      if (!(i & 1) && i + 1 < whole && !(decltype(is_low)::value && any_wide(slot))) {
        f32x16_t t;
        s = scores(is_low, i);
        refer(highest(s));
        base = base_of_weights();
        auto follow = [&] {                        // rarely: the reference behind the next scores' maximum
          if (!exceeds(top)) return;
          sum += odd_sum;
          odd_sum = 0.0f;
          refer(top);
          base = base_of_weights();
        };
        bool more;
        do {                                       // (one way out: a second one costs copies of the sums)
          const int j_next = (i >> 1) + 2;
          turn(is_low, std::false_type{}, j_next, s, t);
          meet(is_low, i >> 1);
          follow();
          if (decltype(is_low)::value) fetch(is_low, j_next);
          else look_up(j_next);
          turn(is_low, std::true_type{}, j_next, t, s);
          i += 2;
          slot = after(slot);
          more = i + 1 < whole && !(decltype(is_low)::value && any_wide(slot));
          if (!more) top = -INFINITY;              // the scores in s are of no use
          follow();
        } while (more);
        sum += odd_sum;
        odd_sum = 0.0f;
        if (i >= u1) break;
      }
      // One unit by itself, as at the edge: some row of the wave does not see all its keys.
      const int slot0 = 32 * (i - u0);
      if (row0 < n_rows && (ring || ls > slot0)) {
        const bool edge = ring || fs < slot0 + 32;
        auto hides = [&](int r) {                  // the lane's row, the unit's slot of score r
          const int k = slot0 + 8 * (r >> 2) + 4 * g + (r & 3);
          return ring ? !in || ring_position(keys, a.cv.window, k) > at : k >= sees;
        };
        const uint32_t* wide_parts = &s_wide[2 * kStepPages * slot + 4 * (i & 1)];   // keys, values of the unit's two pages
        const bool wide_keys = decltype(is_low)::value && __builtin_amdgcn_readfirstlane((int)(wide_parts[0] | wide_parts[2]));
        if (__builtin_expect(wide_keys, 0)) s = wide_scores(i);
        else s = scores(is_low, i);
        if (edge)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = hides(r) ? -INFINITY : s[r];
        top = highest(s);
        if (exceeds(top)) refer(top);
        base = base_of_weights();
#pragma unroll
        for (int r = 0; r < 16; ++r) {             // 0 for what is hidden
          s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], scale, -base));
          sum += s[r];
        }
        const uint32_t vs = fresh(unit_at(slot, i) + v_at), vs2 = fresh(vs + 512);
        if constexpr (decltype(is_low)::value) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint4 p = packed_weights<decltype(is_low)::value>(s, h);
            if (!__builtin_amdgcn_readfirstlane((int)wide_parts[2 * h + 1])) {
#pragma unroll
              for (int m = 0; m < VT; ++m) o[m] = add_product(is_low, value_operand(vs, vs2, h, m), p, o[m]);
              continue;
            }
#pragma unroll 1
            for (int wide = 0; wide < 2; ++wide) {
              const uint32_t at0 = fresh(vs), at1 = fresh(vs + 512);
              const uint32_t* slots_of = s_wide_slots[fresh(2 * kStepPages * slot + 4 * (i & 1) + 2 * h + 1)];
              const int t = fresh(4 * g);
#pragma unroll
              for (int m = 0; m < VT; ++m) {       // dimensions of group m: the weights of the slots that are wide there, or not
                const uint32_t of = (slots_of[m] ^ (wide ? 0u : ~0u)) >> t;
                auto both = [&](int x) { return (of >> x & 1u ? 0xFFFFu : 0u) | (of >> (x + 2) & 1u ? 0xFFFF0000u : 0u); };
                const uint4 q = make_uint4(p.x & both(0), p.y & both(1), p.z & both(8), p.w & both(9));
                o[m] = add_product(is_low, value_operand(at0, at1, h, m), q, o[m]);
                o[m] *= wide ? kWide : 1.0f / kWide;
                __builtin_amdgcn_sched_barrier(0);
              }
            }
          }
        } else {
          // Slots behind the last entry hold what was there before: taken as 0.
          const int valid = used - slot0;
          uint4 mask[2] = {make_uint4(~0u, ~0u, ~0u, ~0u), make_uint4(~0u, ~0u, ~0u, ~0u)};
          if (valid < 32) {
            auto both = [&](int t) { return (t < valid ? 0xFFFFu : 0u) | (t + 1 < valid ? 0xFFFF0000u : 0u); };
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int t = 16 * h + 4 * g;
              mask[h] = make_uint4(both(t), both(t + 2), both(t + 8), both(t + 10));
            }
          }
          auto operand = [&](int h, int m) {
            const uint4 x = value_operand(vs, vs2, h, m);
            return make_uint4(x.x & mask[h].x, x.y & mask[h].y, x.z & mask[h].z, x.w & mask[h].w);
          };
          bool wild = false;                       // some value is infinite or NaN
          if (edge)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int m = 0; m < VT; ++m) wild |= abs_max_bits8(operand(h, m)) >= 0x7F80u;
          __builtin_amdgcn_sched_barrier(0);
          if (__ballot(wild)) {
            const uint8_t* v0 = s_kv[slot] + (i & 1) * 2 * kTile + kValues;
            uint32_t hidden = 0u;
#pragma unroll
            for (int r = 0; r < 16; ++r) hidden |= (uint32_t)hides(r) << r;
            add_seen_values<VT>(v0, v0 + kTile, s, hidden, o, g, n);
          } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint4 p = packed_weights<false>(s, h);
#pragma unroll
              for (int m = 0; m < VT; ++m) o[m] = mfma(operand(h, m), p, o[m]);
            }
          }
        }
      }
      if (!(i & 1)) {
        meet(is_low, i >> 1);
        fetch(is_low, (i >> 1) + 2);
      } else {
        slot = after(slot);
      }
      ++i;
    }
  };
  const int u_low = 2 * low_steps, u_high = 2 * (low_steps + high_steps), u_end = 2 * j_end;
  if (i < min(u_low, u_end)) {
    load_queries<true, KI>(a, q_row, in, g, qf, scale);
    segment(std::true_type{}, false, 0, min(u_low, u_end), first_sees[0], last_sees[0], keys.n[0]);
  }
  if (i < u_end) load_queries<false, KI>(a, q_row, in, g, qf, scale);
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {                    // HIGH entries, then the window's
    const int to = k ? u_end : min(u_high, u_end);
    if (i >= to) continue;
    segment(std::false_type{}, k == 1, k ? u_high : u_low, to, k ? 0 : first_sees[1], k ? 0 : last_sees[1],
            k ? keys.ring_slots : keys.n[1]);
  }
  wait_loads();                                    // copies that repeat the last step: none is left behind
  sum += __shfl_xor(sum, 32);
  if (!in) return;
  if (a.pieces > 1) {
    const size_t at = (((size_t)b * a.cv.n_kv_heads + head) * a.pieces + piece) * ((size_t)a.max_q * G) + row;
#pragma unroll
    for (int m = 0; m < VT; ++m)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<float4*>(a.ws_o + at * D + 32 * m + 2 * r + 4 * g) =
            make_float4(o[m][r], o[m][r + 1], o[m][r + 2], o[m][r + 3]);
    if (g == 0) *reinterpret_cast<float2*>(a.ws_ml + 2 * at) = make_float2(mx, sum);
    return;
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
  for (int m = 0; m < VT; ++m)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *reinterpret_cast<uint2*>(a.out + q_row * D + 32 * m + 2 * r + 4 * g) =
          make_uint2(pack_bf16x2(o[m][r] * inv, o[m][r + 1] * inv), pack_bf16x2(o[m][r + 2] * inv, o[m][r + 3] * inv));
  if (a.lse && g == 0) a.lse[q_row] = sum == 0.0f ? -INFINITY : (mx + __builtin_amdgcn_logf(sum)) * kLn2;
}

// The same for few rows, where reading the pages is the work: 32 rows of one KV
// head, the units of their keys cut over the pieces of the call and the kFewWaves
// waves of a workgroup, which join their sums in LDS.  A wave copies pages as they
// lie into LDS of its own and waits for no other: HIGH units in two halves, the
// next unit's keys asked for once this one's are read, its values likewise; LOW
// units in two batches, one taken while the other comes.  Eight waves a compute
// unit (two workgroups) keep up to 128 KiB on its way.  LOW pages are widened in
// registers.  Numerics are those of prompt_kernel, but that weights of bf16 values
// count with 16 bits, as in the decode call that follows a verified draft: a
// second product, most of it beside the reading (64 drafts behind bf16 histories
// 227 us without it and with it; behind mixed ones 127 and 129).
constexpr int kFewWaves = 4, kFewRows = 32;
template <int D, int G>
__global__ __launch_bounds__(64 * kFewWaves, 2) void prompt_few_kernel(PromptArgs a) {
  using L = PageLayout<D>;
  constexpr int VT = D / 32, KI = D / 16, NG = L::NG, kPart = L::kHiV;   // kPart: bytes of a HIGH page's keys, or values
  constexpr int kHalf = 2 * kPart / 1024;          // copies of a HIGH unit's keys, or values
  constexpr int kLowBatch = 256 / D, kRoom = 4 * kLowBatch * L::kLoHead;   // units; bytes of a wave's LDS
  static_assert(4 * kPart <= kRoom && kFewRows * D * 4 <= kRoom, "a wave's part of LDS");
  __shared__ __align__(1024) uint8_t s_room[kFewWaves][kRoom];
  __shared__ float2 s_ml[kFewWaves][kFewRows];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int g = lane >> 5, n = lane & 31;
  int rest = (int)blockIdx.x;
  const int head = rest % a.cv.n_kv_heads;
  rest /= a.cv.n_kv_heads;
  const int piece = rest % a.pieces;
  rest /= a.pieces;
  const int b = by_length(a, rest), nq = a.n_q ? min(max(a.n_q[b], 0), a.max_q) : a.max_q, n_rows = nq * G;
  if (n_rows == 0) return;
  const bool in = n < n_rows;
  const Keys keys = keys_of(a.cv, b, a.layer);
  const long long first = a.first ? (long long)a.first[b] : (long long)keys.n_pos - nq;
  // Entries of each list that the first row sees, and the last: 16 lanes for each of the four.
  const long long wave_at = first, wave_end = first + nq - 1;
  const int seen = entries_at(lane < 32 ? keys.list[0] : keys.list[1], lane < 32 ? keys.n[0] : keys.n[1], keys.n_pos,
                              lane & 16 ? wave_end : wave_at);
  const int first_sees[2] = {__builtin_amdgcn_readlane(seen, 0), __builtin_amdgcn_readlane(seen, 32)};
  const int last_sees[2] = {__builtin_amdgcn_readlane(seen, 16), __builtin_amdgcn_readlane(seen, 48)};
  const bool ring_seen = keys.ring_slots > 0 && wave_end >= (long long)keys.n_pos - keys.ring_slots;
  const int u_low = (last_sees[0] + 31) / 32, u_high = u_low + (last_sees[1] + 31) / 32;
  const int units = u_high + (ring_seen ? (keys.ring_slots + 31) / 32 : 0);
  const int part = piece * kFewWaves + wave, parts = a.pieces * kFewWaves;
  const int begin = (int)((long long)units * part / parts), end = (int)((long long)units * (part + 1) / parts);
  // The lane's row of the queries, and its position: made where they are used, which is rarely.
  auto q_row = [&] {
    const int x = fresh(in ? n : 0);
    return ((size_t)b * a.max_q + x / G) * a.n_q_heads + (size_t)head * G + x % G;
  };
  auto row_at = [&] { return first + fresh(in ? n : 0) / G; };

  // Where the head's part of the pages starts, 64 pages at a time, one per lane.
  auto kind_of = [&](int u) { return u < u_low ? kLowPages : u < u_high ? kHighPages : kWindowPages; };
  uint32_t from_lo = 0, from_hi = 0;
  int from_of = -1;
  auto page_at = [&](int page) __attribute__((always_inline)) {   // of the wave's pages, 2 a unit
    if (page >> 6 != from_of) {
      from_of = page >> 6;
      const int x = min((page & ~63) + lane, 2 * (end - begin) - 1), u = begin + (x >> 1), kind = kind_of(u);
      const int p = 2 * (u - (kind == kLowPages ? 0 : kind == kHighPages ? u_low : u_high)) + (x & 1);
      const int id = kind == kWindowPages ? keys.ring_page + min(p, a.cv.ring_pp - 1)
                     : kind == kLowPages  ? keys.table[0][min(p, (last_sees[0] - 1) >> 4)]
                                          : keys.table[1][min(p, (last_sees[1] - 1) >> 4)];
      const uint32_t hs = ((uint32_t)head + (uint32_t)id) % (uint32_t)a.cv.n_kv_heads;
      const uint64_t at = kind == kLowPages
                              ? (uint64_t)a.cv.lo_pool + (uint64_t)id * a.cv.lo_page_bytes + hs * (uint32_t)L::kLoHead
                              : (uint64_t)a.cv.hi_pool + (uint64_t)id * a.cv.hi_page_bytes + hs * (uint32_t)L::kHiHead;
      from_lo = (uint32_t)at;
      from_hi = (uint32_t)(at >> 32);
    }
    return reinterpret_cast<const uint8_t*>((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)from_hi, page & 63) << 32 |
                                            (uint32_t)__builtin_amdgcn_readlane((int)from_lo, page & 63));
  };

  uint4 qf[KI];
  float scale = 0.0f;                              // of the lane's row, as its queries are held
  f32x16_t o[VT];
#pragma unroll
  for (int m = 0; m < VT; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[m][r] = 0.0f;
  float mx = -INFINITY, sum = 0.0f;
  const uint32_t room = lds_address(s_room[wave]);
  const int t16 = n & 15, own = n >> 4;            // slot of a page, and which of a unit's two; of values: dimension, parity
  int u = begin;
  // The wave's units of one kind up to `to`; u0: the kind's first.
  auto segment = [&](auto is_low, bool ring, int u0, int to, int fs, int ls, const int32_t* list, int used)
      __attribute__((always_inline)) {
    constexpr bool kLow = decltype(is_low)::value;
    // Copies of page x of the wave's: its bytes `from` .. `from` + kBytes to LDS address `to_lds`.
    auto copy_page = [&](int x, int from, auto bytes, uint32_t to_lds) __attribute__((always_inline)) {
      constexpr int kBytes = decltype(bytes)::value;
      const uint8_t* src = page_at(x) + from;
#pragma unroll
      for (int y = 0; y < kBytes; y += 1024)
        if (y + 1024 <= kBytes || lane * 16 < kBytes - y) copy_to_lds<true>(src, (uint32_t)(y + lane * 16), to_lds + y);
    };
    // HIGH: the keys or values of unit v; LOW: the batch of units that starts at v, in half `slot` of the room.
    auto copy_half = [&](int v, int half) __attribute__((always_inline)) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        copy_page(2 * (v - begin) + h, half * kPart, std::integral_constant<int, kPart>{}, room + (2 * half + h) * kPart);
    };
    auto copy_batch = [&](int v, int slot) __attribute__((always_inline)) {
      for (int x = 0; x < 2 * min(kLowBatch, to - v); ++x)
        copy_page(2 * (v - begin) + x, 0, std::integral_constant<int, L::kLoHead>{}, room + slot * (kRoom / 2) + x * L::kLoHead);
    };
    if constexpr (kLow) {
      copy_batch(u, 0);
    } else {
      copy_half(u, 0);
      copy_half(u, 1);
    }
    load_queries<kLow, KI>(a, q_row(), in, g, qf, scale);
    // What each row sees: the entries between what the first and the last row see are fewer than the tile's tokens.
    int sees = fs;
    if (ls > fs) {
      const int pos = lane < ls - fs ? list[fs + lane] : INT32_MAX;
      const long long at = row_at();
#pragma unroll 1
      for (int x = 0; x < kFewRows / G; ++x) {
        const int c = __popcll(__ballot(lane < ls - fs && (long long)pos <= wave_at + x));
        if (at == wave_at + x) sees = fs + c;
      }
    }
    if (!in) sees = 0;
    int slot = 0;
#pragma unroll 1
    while (u < to) {
      const int batch = kLow ? min(kLowBatch, to - u) : 1, next = u + batch;
      // What is to be read has arrived; what was asked for behind it may be on its way.
      if constexpr (kLow) {
        if (next < to) copy_batch(next, slot ^ 1);
        if (next + kLowBatch <= to) wait_copies<2 * kLowBatch * ((L::kLoHead + 1023) / 1024)>();
        else wait_copies<0>();
      } else {
        wait_copies<kHalf>();
      }
#pragma unroll 1
      for (int x = 0; x < batch; ++x, ++u) {
        const int slot0 = 32 * (u - u0);           // the unit's first slot of its store
        f32x16_t s;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 0.0f;
        const int valid = used - slot0;            // of the unit's slots; what was there before is behind them
        bool wide_keys = false, wide_values = false;   // some of the unit's scales are
        const uint32_t low0 = room + slot * (kRoom / 2) + 2 * x * L::kLoHead;
        if constexpr (kLow) {
          // A page's scales are 8 NG words, NG / 2 a slot.
          const int h = lane / (8 * NG), word = lane % (8 * NG);
          if (h < 2 && 16 * h + word / (NG / 2) < valid) {
            const uint32_t ks = read_lds4(low0 + h * L::kLoHead + L::kLoKS + 4 * word);
            const uint32_t vs = read_lds4(low0 + h * L::kLoHead + L::kLoVS + 4 * word);
            wide_keys = max(ks & 0xFFFFu, ks >> 16) > kWideScale;
            wide_values = max(vs & 0xFFFFu, vs >> 16) > kWideScale;
          }
          wide_keys = __ballot(wide_keys) != 0ull;
          wide_values = __ballot(wide_values) != 0ull;
          const uint32_t k0 = low0 + own * L::kLoHead;
          uint32_t ks[NG / 2], word0[NG], word1[NG];
          read_words(k0 + L::kLoKS + t16 * 2 * NG, ks);
          read_words(k0 + (g * 16 + t16) * 4 * NG, word0);
          read_words(k0 + ((g + 2) * 16 + t16) * 4 * NG, word1);
          if (16 * own + t16 >= valid)
#pragma unroll
            for (int c = 0; c < NG / 2; ++c) ks[c] = 0u;
          if (wide_keys)
#pragma unroll
            for (int c = 0; c < NG / 2; ++c) ks[c] = scales_of(false, ks[c]);
          auto add_group = [&](int i, uint32_t sc, uint32_t w0, uint32_t w1) __attribute__((always_inline)) {
            const uint32_t both = __builtin_amdgcn_perm(sc, sc, i & 1 ? 0x03020302u : 0x01000100u);
            const f16x2_t s8 = halves(both & 0xFFF8FFF8u), s3 = halves(both) - s8;
#pragma unroll
            for (int w = 0; w < 2; ++w) {          // quarters g and g + 2: chunks 2 (2 i + w) + g
              const uint32_t word = w ? w1 : w0;
              s = mfma_half(key_part(word, s8), qf[2 * i + w], s);
              s = mfma_half(key_part(word, s3), qf[2 * i + w], s);
            }
          };
#pragma unroll
          for (int i = 0; i < NG; ++i) add_group(i, ks[i / 2], word0[i], word1[i]);
          if (wide_keys) {
            s *= 1.0f / kWide;
            const int l = fresh(lane), t = l & 15;
            const uint32_t at = low0 + (l >> 4 & 1) * L::kLoHead;
#pragma unroll
            for (int i = 0; i < NG; ++i) {
              const uint32_t sc = (l & 31) < valid ? scales_of(true, read_lds4(at + L::kLoKS + t * 2 * NG + 4 * (i / 2))) : 0u;
              const uint32_t word = at + ((l >> 5) * 16 + t) * 4 * NG + 4 * i;
              add_group(i, sc, read_lds4(word), read_lds4(word + 128 * NG));
              __builtin_amdgcn_sched_barrier(0);
            }
            s *= kWide;
          }
        } else {
          const uint32_t k0 = fresh(room + own * kPart + g * 256 + t16 * 16);
#pragma unroll
          for (int k = 0; k < KI; ++k) s = mfma(read_lds16(k0 + 512 * k), qf[k], s);
          lds_barrier_wave();                      // the keys have been read: the next unit's may come
          if (next < to) copy_half(next, 0);
        }
        // The value operands of a HIGH page h.
        const uint32_t v0 = fresh(room + 2 * kPart + g * 256 + t16 * 16 + own * 8), v1 = fresh(v0 + 512);
        auto high_value = [&](int h, int m) {
          const u32x2_t y = *(const lds_u32x2*)(uintptr_t)(v0 + h * kPart + m * 1024);
          const u32x2_t z = *(const lds_u32x2*)(uintptr_t)(v1 + h * kPart + m * 1024);
          return make_uint4(y[0], y[1], z[0], z[1]);
        };
        const bool edge = ring || fs < slot0 + 32;
        uint32_t hidden = 0u;
        if (edge) {
          const long long at = row_at();
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int k = slot0 + 8 * (r >> 2) + 4 * g + (r & 3);
            const bool hid = ring ? !in || ring_position(keys, a.cv.window, k) > at : k >= sees;
            hidden |= (uint32_t)hid << r;
            s[r] = hid ? -INFINITY : s[r];
          }
        }
        float top = fmaxf(s[0], s[1]);
#pragma unroll
        for (int r = 2; r < 16; ++r) top = fmaxf(top, s[r]);
        top = fmaxf(top, __shfl_xor(top, 32));
        top = top == -INFINITY ? top : top * scale;
        if (__ballot(top > mx + kHeadroom)) {      // the reference follows a maximum that exceeds it
          const float ref = top > mx + kHeadroom ? top - kBelow : mx;
          const float alpha = ref == mx ? 1.0f : __builtin_amdgcn_exp2f(mx - ref);
          sum *= alpha;
#pragma unroll
          for (int m = 0; m < VT; ++m) o[m] *= alpha;
          mx = ref;
        }
        const float base = mx == -INFINITY ? 0.0f : mx;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], scale, -base));
          if (!edge) sum += s[r];
        }
        if (edge) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            s[r] = hidden >> r & 1u ? 0.0f : s[r];
            sum += s[r];
          }
        }
        if constexpr (kLow) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t v[VT][4];
#pragma unroll
            for (int w = 0; w < 2; ++w) {          // slots 4 g .. and 4 g + 8 .., the parity's nibbles
              uint32_t vs[2 * NG], code[NG];
              read_words(low0 + h * L::kLoHead + L::kLoVS + (g + 2 * w) * 8 * NG, vs);
              read_words(low0 + h * L::kLoHead + L::kLoVC + ((g + 2 * w) * 16 + t16) * 4 * NG, code);
              if (valid < 32)
#pragma unroll
                for (int c = 0; c < 2 * NG; ++c)
                  if (16 * h + 4 * (g + 2 * w) + c / (NG / 2) >= valid) vs[c] = 0u;
              if (wide_values)
#pragma unroll
                for (int c = 0; c < 2 * NG; ++c) vs[c] = scales_of(false, vs[c]);
#pragma unroll
              for (int m = 0; m < VT; ++m) {
                const uint32_t pick = m & 1 ? 0x07060302u : 0x05040100u;
#pragma unroll
                for (int t = 0; t < 2; ++t)
                  v[m][2 * w + t] = word_of(code_pair(code[m] >> (4 * own), t) *
                                            halves(__builtin_amdgcn_perm(vs[(t + 2) * (NG / 2) + m / 2], vs[t * (NG / 2) + m / 2], pick)));
              }
            }
            const uint4 p = packed_weights<true>(s, h);
#pragma unroll
            for (int m = 0; m < VT; ++m) o[m] = mfma_half(make_uint4(v[m][0], v[m][1], v[m][2], v[m][3]), p, o[m]);
          }
          if (wide_values) {
            const uint4 p0 = packed_weights<true>(s, 0), p1 = packed_weights<true>(s, 1);
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
              const int l = fresh(lane), first_slot = 16 * h + 4 * (l >> 5);
              const uint4 p = make_uint4(h ? p1.x : p0.x, h ? p1.y : p0.y, h ? p1.z : p0.z, h ? p1.w : p0.w);
              const uint32_t scales = low0 + h * L::kLoHead + L::kLoVS + (l >> 5) * 8 * NG;
              const uint32_t codes = low0 + h * L::kLoHead + L::kLoVC + ((l >> 5) * 16 + (l & 15)) * 4 * NG;
#pragma unroll
              for (int m = 0; m < VT; ++m) {
                uint32_t v[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) {      // slots t and t + 2 of four
                  const int w = y >> 1, t = y & 1;
                  auto scale_at = [&](int z) {
                    const uint32_t sc = read_lds4(scales + 16 * w * NG + z * 2 * NG + 4 * (m / 2));
                    return first_slot + 8 * w + z < valid ? scales_of(true, sc) : 0u;
                  };
                  v[y] = word_of(code_pair(read_lds4(codes + w * 128 * NG + 4 * m) >> (l >> 2 & 4), t) *
                                 halves(__builtin_amdgcn_perm(scale_at(t + 2), scale_at(t), m & 1 ? 0x07060302u : 0x05040100u)));
                }
                if (h == 0) o[m] *= 1.0f / kWide;
                o[m] = mfma_half(make_uint4(v[0], v[1], v[2], v[3]), p, o[m]);
                if (h == 1) o[m] *= kWide;
                __builtin_amdgcn_sched_barrier(0);
              }
            }
          }
        } else {
          if (next < to) wait_copies<kHalf>();
          else wait_copies<0>();
          bool wild = false;                       // at the edge, some value is infinite or NaN
          if (edge) {
            // Slots behind the last entry hold what was there before: made 0 in LDS, where 16 bytes hold 4 slots twice.
            const uint32_t values = room + 2 * kPart + lane * 16;
#pragma unroll 1
            for (int c = 0; c < kHalf; ++c) {
              const int t = 16 * (c / (kHalf / 2)) + 4 * (lane >> 4);
              const uint32_t lo = (t < valid ? 0xFFFFu : 0u) | (t + 1 < valid ? 0xFFFF0000u : 0u);
              const uint32_t hi = (t + 2 < valid ? 0xFFFFu : 0u) | (t + 3 < valid ? 0xFFFF0000u : 0u);
              uint4 v = read_lds16(values + c * 1024);
              v = make_uint4(v.x & lo, v.y & hi, v.z & lo, v.w & hi);
              if (valid < 32) write_lds16(values + c * 1024, v);
              wild |= abs_max_bits8(v) >= 0x7F80u;
            }
          }
          if (__ballot(wild)) {                    // key by key, which leaves nothing for the products
            const uint8_t* values = s_room[wave] + 2 * kPart;
            add_seen_values<VT>(values, values + kPart, s, hidden, o, g, n);
            lds_barrier_wave();
#pragma unroll 1
            for (int c = 0; c < kHalf; ++c) write_lds16(room + 2 * kPart + lane * 16 + c * 1024, make_uint4(0u, 0u, 0u, 0u));
          }
          // Operands read four ahead, in pinned order: two reads that the compiler merges cost more than one after the other.
          uint4 v[kAhead], p = make_uint4(0u, 0u, 0u, 0u), rest = p;
#pragma unroll
          for (int x = 0; x < kAhead; ++x) {
            v[x] = high_value(x / VT, x % VT);
            __builtin_amdgcn_sched_barrier(0);
          }
#pragma unroll
          for (int x = 0; x < 2 * VT; ++x) {
            if (x % VT == 0) {
              p = packed_weights<false>(s, x / VT);
              rest = weights_rest(s, x / VT, p);
            }
            o[x % VT] = mfma(v[x % kAhead], p, o[x % VT]);
            o[x % VT] = mfma(v[x % kAhead], rest, o[x % VT]);
            if (x + kAhead < 2 * VT) v[x % kAhead] = high_value((x + kAhead) / VT, (x + kAhead) % VT);
            __builtin_amdgcn_sched_barrier(0);
          }
          lds_barrier_wave();
          if (next < to) copy_half(next, 1);
        }
      }
      slot ^= 1;
      lds_barrier_wave();                          // the batch has been read
    }
  };
  if (u < min(u_low, end)) segment(std::true_type{}, false, 0, min(u_low, end), first_sees[0], last_sees[0], keys.list[0], keys.n[0]);
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {                    // HIGH entries, then the window's
    const int to = k ? end : min(u_high, end);
    if (u >= to) continue;
    segment(std::false_type{}, k == 1, k ? u_high : u_low, to, k ? 0 : first_sees[1], k ? 0 : last_sees[1], keys.list[1],
            k ? keys.ring_slots : keys.n[1]);
  }
  sum += __shfl_xor(sum, 32);

  // The waves' sums joined: row x's output d at float (d + 4 x) mod D of its row, so that the stores of 32 rows do not
  // meet on the same banks.
  lds_barrier();
  float* mine = reinterpret_cast<float*>(s_room[wave]) + n * D;
#pragma unroll
  for (int m = 0; m < VT; ++m)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *reinterpret_cast<float4*>(mine + ((32 * m + 2 * r + 4 * g + 4 * n) & (D - 1))) =
          make_float4(o[m][r], o[m][r + 1], o[m][r + 2], o[m][r + 3]);
  if (g == 0) s_ml[wave][n] = make_float2(mx, sum);
  __syncthreads();
  constexpr int kEach = kFewRows * D / (64 * kFewWaves);     // outputs of a thread: 16 or 8 of one row
  const int x = (int)threadIdx.x * kEach / D, d0 = (int)threadIdx.x * kEach % D;
  float ref = -INFINITY, total = 0.0f, acc[kEach];
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) ref = fmaxf(ref, s_ml[w][x].x);
#pragma unroll
  for (int d = 0; d < kEach; ++d) acc[d] = 0.0f;
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) {
    const float2 ml = s_ml[w][x];
    if (ml.y == 0.0f) continue;
    const float f = __builtin_amdgcn_exp2f(ml.x - ref);
    total = fmaf(ml.y, f, total);
#pragma unroll
    for (int d = 0; d < kEach; d += 4) {
      const float4 v = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(s_room[w]) + x * D +
                                                        ((d0 + d + 4 * x) & (D - 1)));
      acc[d] = fmaf(v.x, f, acc[d]);
      acc[d + 1] = fmaf(v.y, f, acc[d + 1]);
      acc[d + 2] = fmaf(v.z, f, acc[d + 2]);
      acc[d + 3] = fmaf(v.w, f, acc[d + 3]);
    }
  }
  const int to = x;
  if (to >= n_rows) return;
  if (a.pieces > 1) {
    const size_t w = (((size_t)b * a.cv.n_kv_heads + head) * a.pieces + piece) * ((size_t)a.max_q * G) + to;
#pragma unroll
    for (int d = 0; d < kEach; d += 4)
      *reinterpret_cast<float4*>(a.ws_o + w * D + d0 + d) = make_float4(acc[d], acc[d + 1], acc[d + 2], acc[d + 3]);
    if (d0 == 0) *reinterpret_cast<float2*>(a.ws_ml + 2 * w) = make_float2(ref, total);
    return;
  }
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
  const size_t w = ((size_t)b * a.max_q + to / G) * a.n_q_heads + (size_t)head * G + to % G;
#pragma unroll
  for (int d = 0; d < kEach; d += 4)
    *reinterpret_cast<uint2*>(a.out + w * D + d0 + d) =
        make_uint2(pack_bf16x2(acc[d] * inv, acc[d + 1] * inv), pack_bf16x2(acc[d + 2] * inv, acc[d + 3] * inv));
  if (a.lse && d0 == 0) a.lse[w] = total == 0.0f ? -INFINITY : (ref + __builtin_amdgcn_logf(total)) * kLn2;
}

// Joins the pieces of a row: the parts' sums and outputs, taken to the largest
// of their references.  kWaves waves take every kWaves-th piece of a row; a
// workgroup takes 4 / kWaves rows.
template <int D, int G, int kWaves>
__global__ __launch_bounds__(256) void prompt_merge_kernel(PromptArgs a) {
  __shared__ float s_o[4][D];
  __shared__ float2 s_ml[4];
  constexpr int E = D / 64;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int64_t x = (int64_t)blockIdx.x * (4 / kWaves) + wave / kWaves, rows = (int64_t)a.max_q * G;
  const int64_t bh = x / rows;
  const int row = (int)(x - bh * rows), b = (int)(bh / a.cv.n_kv_heads), head = (int)(bh % a.cv.n_kv_heads);
  const bool live = b < a.batch && row < (a.n_q ? min(a.n_q[b], a.max_q) : a.max_q) * G;
  const size_t first = (size_t)bh * a.pieces * rows + row;
  float top = -INFINITY, sum = 0.0f, o[E];
#pragma unroll
  for (int d = 0; d < E; ++d) o[d] = 0.0f;
  if (live) {
    // 64 pieces at a time, references and sums one per lane.
    for (int p0 = wave % kWaves; p0 < a.pieces; p0 += 64 * kWaves) {
      const int mine = p0 + lane * kWaves, n = min(64, (a.pieces - p0 + kWaves - 1) / kWaves);
      const float2 ml = lane < n ? *reinterpret_cast<const float2*>(a.ws_ml + 2 * (first + (size_t)mine * rows))
                                 : make_float2(-INFINITY, 0.0f);
      float ref = ml.x;
#pragma unroll
      for (int s = 1; s < 64; s *= 2) ref = fmaxf(ref, __shfl_xor(ref, s));
      ref = fmaxf(ref, top);
      const float keep = top == ref ? 1.0f : __builtin_amdgcn_exp2f(top - ref);
      const float w = ml.y == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(ml.x - ref);   // 0: the row sees nothing of the piece
      float part = ml.y == 0.0f ? 0.0f : ml.y * w;
#pragma unroll
      for (int s = 1; s < 64; s *= 2) part += __shfl_xor(part, s);
      sum = fmaf(sum, keep, part);
#pragma unroll
      for (int d = 0; d < E; ++d) o[d] *= keep;
      top = ref;
      for (int p = 0; p < n; p += 8) {             // 8 at a time: their loads together, those behind the last one its own
        float f[8], v[8][E];
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const int at = min(p + y, n - 1);
          f[y] = p + y < n ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), at)) : 0.0f;
          const float* from = a.ws_o + (first + (size_t)(p0 + at * kWaves) * rows) * D + lane * E;
#pragma unroll
          for (int d = 0; d < E; ++d) v[y][d] = from[d];
        }
#pragma unroll
        for (int y = 0; y < 8; ++y)
#pragma unroll
          for (int d = 0; d < E; ++d) o[d] = f[y] == 0.0f ? o[d] : fmaf(v[y][d], f[y], o[d]);
      }
    }
  }
  if (kWaves > 1) {
#pragma unroll
    for (int d = 0; d < E; ++d) s_o[wave][lane * E + d] = o[d];
    if (lane == 0) s_ml[wave] = make_float2(top, sum);
    __syncthreads();
    if (wave) return;
    float ref = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) ref = fmaxf(ref, s_ml[w].x);
    sum = 0.0f;
#pragma unroll
    for (int d = 0; d < E; ++d) o[d] = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (s_ml[w].y == 0.0f) continue;
      const float f = __builtin_amdgcn_exp2f(s_ml[w].x - ref);
      sum = fmaf(s_ml[w].y, f, sum);
#pragma unroll
      for (int d = 0; d < E; ++d) o[d] = fmaf(s_o[w][lane * E + d], f, o[d]);
    }
    top = ref;
  }
  if (!live) return;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  const size_t to = ((size_t)b * a.max_q + row / G) * a.n_q_heads + (size_t)head * G + row % G;
  if constexpr (D == 128) {
    *reinterpret_cast<uint32_t*>(a.out + to * D + 2 * lane) = pack_bf16x2(o[0] * inv, o[1] * inv);
  } else {
    a.out[to * D + lane] = f32_to_bf16_rne_dev(o[0] * inv);
  }
  if (a.lse && lane == 0) a.lse[to] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <int D, int G>
void launch_group(const PromptArgs& a, const PromptCut& c, hipStream_t s) {
  const dim3 blocks((unsigned)prompt_blocks(a, c));
  if (c.rows == kFewRows) prompt_few_kernel<D, G><<<blocks, dim3(64 * kFewWaves), 0, s>>>(a);
  else prompt_kernel<D, G, 8><<<blocks, dim3(512), 0, s>>>(a);
  if (a.pieces > 1) {
    const int64_t rows = (int64_t)a.batch * a.cv.n_kv_heads * a.max_q * G;
    if (a.pieces > 8) prompt_merge_kernel<D, G, 4><<<dim3((unsigned)rows), dim3(256), 0, s>>>(a);
    else prompt_merge_kernel<D, G, 1><<<dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s>>>(a);
  }
}

template <int D>
void launch_dim(const PromptArgs& a, const PromptCut& c, hipStream_t s) {
  switch (a.n_q_heads / a.cv.n_kv_heads) {
    case 1: launch_group<D, 1>(a, c, s); break;
    case 2: launch_group<D, 2>(a, c, s); break;
    case 4: launch_group<D, 4>(a, c, s); break;
    default: launch_group<D, 8>(a, c, s); break;
  }
}

}  // namespace

// Tiles of 256 rows, whose eight waves share every page through LDS, or of 32,
// whose waves share the rows, where no sequence has more (32 sequences of 1,000-
// 8,000 tokens, 32 rows of each: 79 us so, 145 in tiles of 256; 48 rows, in a build
// before, in two tiles of 32: 153, in one of 256: 155).  The keys are cut into
// pieces where the tiles leave compute units idle: for 32 rows by the workgroups the
// card holds (8 KV heads; with 1, 2 and 4 pieces 128 sequences of 500-4,096 tokens
// take 131, 142, 155 us, 64 of 1,024-8,192 124, 130, 140, 32 of 1,000-8,000 94, 78,
// 78; one of 32,005 tokens with 32, 64 and 128 pieces 29, 27, 41).  For tiles of 256
// rows by what a call takes with each number of pieces, in microseconds: as many
// turns of the 256 compute units as the workgroups need, each a piece's steps at
// 2.5 (64 keys: 2.1 of bf16 pages, 3.2 of int4 ones) and 10 to begin and end, and
// the joining, 6 and its traffic (88 tiles of 32,333 tokens, most of them int4:
// 509 us with 2 pieces, 428 with the number of this rule).
PromptCut prompt_cut(int32_t batch, int32_t max_q, int32_t group, int32_t n_kv_heads, int32_t head_dim,
                     int32_t max_ctx_hint) {
  PromptCut c;
  const int64_t rows = (int64_t)max_q * group;
  c.rows = rows <= kFewRows ? kFewRows : 256;
  c.pieces = 1;
  const int64_t tiles = (rows + c.rows - 1) / c.rows * batch * n_kv_heads;
  if (c.rows == kFewRows) {                        // of 4 waves each, with a unit or more for each wave
    const int64_t want = tiles < 128 ? 512 : 1024;
    c.pieces = (int32_t)std::max<int64_t>(1, std::min<int64_t>((want + tiles - 1) / tiles, (max_ctx_hint + 127) / 128));
    return c;
  }
  const double steps = (max_ctx_hint + kStepKeys - 1) / kStepKeys, traffic = 2.0 * 4 * head_dim * c.rows * 1e-6 / 4.0;
  double least = 0.0;
  for (int32_t p = 1; p == 1 || (p <= 32 && p * tiles <= 1024 && 4 * p <= steps); ++p) {
    double t = (double)((tiles * p + 255) / 256) * (2.5 * steps / p + 10.0);
    if (p > 1) t += 6.0 + traffic * (double)(tiles * p);
    if (p > 1 && t >= least) continue;
    least = t;
    c.pieces = p;
  }
  return c;
}

int64_t prompt_blocks(const PromptArgs& a, const PromptCut& c) {
  const int64_t rows = (int64_t)a.max_q * (a.n_q_heads / a.cv.n_kv_heads);
  return (rows + c.rows - 1) / c.rows * a.batch * a.cv.n_kv_heads * a.pieces;
}

hipError_t launch_prompt(const PromptArgs& a, const PromptCut& c, hipStream_t s) {
  if (a.cv.head_dim == 64) launch_dim<64>(a, c, s);
  else launch_dim<128>(a, c, s);
  return hipGetLastError();
}

}  // namespace pask
