// gfx950 kernels of the absorbed latent attention: one query per sequence and
// head over the persisted latents of a layer.
//
//   latent_attn   a workgroup takes a contiguous range of the list of tiles
//                 (32 slots of one store) of all sequences, all heads at once,
//                 so every latent is read from memory once and serves as key
//                 and as value from the same LDS tile.
//   latent_merge  joins the partial results of sequences that several
//                 workgroups share.
#include <hip/hip_runtime.h>

#include <math.h>

#include <algorithm>
#include <type_traits>

#include "pask_latent_device.h"

namespace pask {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = 4;           // of the merge
constexpr int kTile = 32;                          // slots per tile: two pages of one store
constexpr float kLn2 = 0.6931471805599453f;

// D[16x16] += A[16x32] B[32x16]: lane l holds A[l % 16][8 (l / 16) ..], B[8 (l / 16) ..][l % 16],
// D[4 (l / 16) ..][l % 16].
__device__ __forceinline__ f32x4_t mfma(uint4 a, uint4 b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0,
                                                 0, 0);
}

// ---------------------------------------------------------------------------
// the list of tiles
// ---------------------------------------------------------------------------
// Sequence b has ceil(n_hi / 32) + ceil(n_lo / 32) tiles, or one if it holds
// nothing (its worker writes the empty result).  Worker w of W takes tiles
// [w u, w u + u), u = ceil(total / W).
__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }
struct Counts {
  int n_hi, n_lo;
};
__device__ __forceinline__ Counts counts_at(const LatentAttnArgs& a, int b) {
  const int32_t* c = counters_of(a.cv, min(b, a.batch - 1), a.layer);
  return Counts{c[kCntHi], c[kCntLo]};
}
__device__ __forceinline__ int tiles_of(const Counts& c) {
  return max(1, (c.n_hi + kTile - 1) / kTile + (c.n_lo + kTile - 1) / kTile);
}

// Over the whole workgroup of T threads (thread t counts sequences [t B / T,
// (t + 1) B / T)): the tiles of all sequences, and the sequence that holds tile
// at(total) with the tile its list starts at.
struct ListPlace {
  long long total, start;
  int b;
};
template <int T, typename At>
__device__ __forceinline__ ListPlace find_in_list(const LatentAttnArgs& a, long long* s_scan, At at) {
  constexpr int kWaves = T / 64;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto tiles = [&](int b) { return tiles_of(counts_at(a, b)); };
  long long mine = 0;
  const int first = (int)((long long)a.batch * tid / T), last = (int)((long long)a.batch * (tid + 1) / T);
  for (int b = first; b < last; ++b) mine += tiles(b);
  long long incl = mine;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const long long y = __shfl_up(incl, off);
    if (lane >= off) incl += y;
  }
  if (lane == 63) s_scan[wave] = incl;
  __syncthreads();
  long long before = incl - mine, total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += s_scan[w];
    total += s_scan[w];
  }
  const long long x = at(total);
  if (x >= before && x < before + mine) {          // one thread at most
    int b = first;
    long long start = before;
    for (int nt; start + (nt = tiles(b)) <= x; ++b) start += nt;
    s_scan[kWaves] = start;
    s_scan[kWaves + 1] = b;
  }
  __syncthreads();
  return ListPlace{total, s_scan[kWaves], uni((int)s_scan[kWaves + 1])};
}

// Tiles each worker takes.  More workers finish their tiles sooner but leave
// more partial results, whose writing and merging costs about 1/150 of a tile's
// time for 16 heads when the whole chip shares it: with W workers the tiles take
// total / W tiles' times and the partials W head_tiles / 150, least at
// W = sqrt(150 total / head_tiles).  Rank 512, this rule / all workers / 1/76:
// one sequence of 8,000 tokens, 64 heads 28.6 / 41.5 / 29.3 us; four of 16,000,
// 128 heads 66.3 / 76.7 / 86.6; one of 64,001, 128 heads 69.5 / 66.7 / 81.7.
__device__ __forceinline__ long long tiles_per_worker(long long total, int workers, int head_tiles) {
  const int best = (int)sqrtf(150.0f * (float)total / (float)head_tiles) + 1;
  const int n = min(workers, best);
  return (total + n - 1) / n;
}

// The next 64 tiles of a worker, looked up by one wave at once (a chain of two
// loads for all of them: page ids loaded tile by tile came, in the loads' order,
// behind the copies of the tiles before).
struct Item {
  int b, what, p0, p1;                             // sequence; slots | flags; pages (p1 negative: none)
  __device__ __forceinline__ int slots() const { return what & 63; }   // 0: the tile of an empty sequence
  __device__ __forceinline__ bool high() const { return (what & 64) != 0; }    // of the HIGH store
  __device__ __forceinline__ bool first() const { return (what & 128) != 0; }  // of its sequence
  __device__ __forceinline__ bool last() const { return (what & 256) != 0; }
};
// Lane k: tile `at` + k of the list, whose tile `start` is the first of
// sequence b (start <= at, and at is not behind the sequence).  The place to go
// on from for tile at + 64 goes to b and start.
__device__ __forceinline__ Item look_up(const LatentAttnArgs& a, long long at, int& b, long long& start) {
  const int lane = fresh((int)threadIdx.x & 63);
  const Counts c = counts_at(a, b + lane);         // 64 sequences have 64 tiles or more
  const int nt = tiles_of(c);
  int incl = nt;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int y = __shfl_up(incl, off);
    if (lane >= off) incl = min(incl + y, 1 << 30);
  }
  const int x = (int)(at - start) + lane;          // the lane's tile from `start` on
  int lo = 0;                                      // the sequence that holds it: the first with incl > x
#pragma unroll
  for (int step = 32; step > 0; step >>= 1)
    if (__shfl(incl, lo + step - 1) <= x) lo += step;
  const int behind = __shfl(incl, lo), n = __shfl(nt, lo), j = x - (behind - n);
  const Counts s{__shfl(c.n_hi, lo), __shfl(c.n_lo, lo)};
  Item it;
  it.b = b + lo;
  const int nt_hi = (s.n_hi + kTile - 1) / kTile;
  const bool high = j < nt_hi;
  const int k = high ? j : j - nt_hi, m = max(0, min(kTile, (high ? s.n_hi : s.n_lo) - k * kTile));
  it.what = m | (high ? 64 : 0) | (j == 0 ? 128 : 0) | (j + 1 == n ? 256 : 0);
  it.p0 = 0;
  it.p1 = -1;
  if (it.b < a.batch && m > 0) {                   // tiles behind the list's last are not used
    const int32_t* bt = block_table_of(a.cv, it.b, a.layer, high ? kHi : kLo) + 2 * k;
    it.p0 = bt[0];
    if (m > kPage) it.p1 = bt[1];
  }
  const bool ended = j + 1 == n;
  b = __builtin_amdgcn_readlane(ended ? it.b + 1 : it.b, 63);
  start += __builtin_amdgcn_readlane(ended ? behind : behind - n, 63);
  return it;
}

// ---------------------------------------------------------------------------
// one tile into LDS
// ---------------------------------------------------------------------------
// Pages are copied as they lie, without passing through registers.  Those of a
// LOW tile go to the end of the tile's buffer, from where the tile is widened
// in place once they have arrived (widen_low).
template <int R, int P, int T>
struct Tile {
  using PG = LatentPage<R, P>;
  static constexpr int kWaves = T / 64;
  static constexpr int kBytes = 2 * PG::kHiBytes, kRaw = kBytes - 2 * PG::kLoBytes;
  static constexpr int kLoChunks = PG::kLoBytes / 16;

  // The copy of a tile's pages, in pieces of 64 chunks (1 KiB).
  struct Copy {
    const uint8_t *b0, *b1;                        // chunk c of the two pages: at (c < split ? b0 : b1) + 16 c
    int split, chunks;
    uint8_t* to;
  };
  __device__ __forceinline__ static Copy no_copy() { return Copy{nullptr, nullptr, 0, 0, nullptr}; }
  __device__ __forceinline__ static Copy copy_of(const CacheView& cv, const Item& x, uint8_t* tile) {
    const uint8_t* pool = x.high() ? cv.hi_pool : cv.lo_pool;
    const int n = x.high() ? PG::kHiChunks : kLoChunks;
    return Copy{pool + (size_t)x.p0 * (16 * n), pool + ((long long)x.p1 - 1) * (16 * n), n,
                x.slots() == 0 ? 0 : x.p1 < 0 ? n : 2 * n, tile + (x.high() ? 0 : kRaw)};
  }
  __device__ __forceinline__ static void copy_piece(const Copy& y, int piece) {
    const int c = piece * 64 + (fresh((int)threadIdx.x) & 63);
    if (c < y.chunks) load_to_lds<true>((c < y.split ? y.b0 : y.b1) + c * 16, y.to + piece * 1024);
  }
  // Slots from n on as zeros: what lies there is not an entry (any bytes, NaN
  // among them), and a weight of 0 does not make a NaN value harmless.
  __device__ __forceinline__ static void clear_from(uint8_t* tile_buf, int n) {
    const uint32_t tile = lds_address(tile_buf);
    for (int c = fresh((int)threadIdx.x); c < 2 * PG::kHiChunks; c += T) {
      const int page = c < PG::kHiChunks ? 0 : 1, d = c - page * PG::kHiChunks;
      if (page * kPage + latent_swap((d >> 4) & 3, d & 15) >= n)
        write_lds16(tile + c * 16, make_uint4(0u, 0u, 0u, 0u));
    }
  }
  // The tile of n slots from the pages' bytes at its end, by the whole
  // workgroup: all of them are read before the first value is written.
  __device__ __forceinline__ static void widen_low(uint8_t* tile_buf, int n) {
    const uint32_t tile = lds_address(tile_buf), raw = tile + kRaw;
    const int tid = fresh((int)threadIdx.x);
    constexpr int NC = (2 * PG::kGroups + T - 1) / T;          // code groups per thread
    static_assert(2 * PG::kRopeChunks <= T, "a rotary piece per thread");
    uint4 codes[NC], rope = make_uint4(0u, 0u, 0u, 0u);
    float scale[NC];
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int g = tid + T * k, page = g < PG::kGroups ? 0 : 1, h = g - page * PG::kGroups;
      if (g < 2 * PG::kGroups) {
        codes[k] = read_lds16(raw + page * PG::kLoBytes + h * 16);
        scale[k] = half_value(
            *reinterpret_cast<const uint16_t*>(tile_buf + kRaw + page * PG::kLoBytes + PG::kScales + 2 * h));
      }
    }
    const int c = tid, rp = c < PG::kRopeChunks ? 0 : 1, rd = c - rp * PG::kRopeChunks;
    if (c < 2 * PG::kRopeChunks)
      rope = read_lds16(raw + rp * PG::kLoBytes + PG::kRopeAt + rd * 16);
    lds_barrier();
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int g = tid + T * k, page = g < PG::kGroups ? 0 : 1, h = g - page * PG::kGroups;
      if (g < 2 * PG::kGroups) {
        const int t = h & 15;
        const bool in = page * kPage + t < n;
        const uint32_t w[4] = {codes[k].x, codes[k].y, codes[k].z, codes[k].w};
        const uint32_t dst = tile + page * PG::kHiBytes + (h >> 4) * 1024;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint4 v = low_values(w[q], scale[k]);
          write_lds16(dst + (16 * q + latent_swap(q, t)) * 16, in ? v : make_uint4(0u, 0u, 0u, 0u));
        }
      }
    }
    if (c < 2 * PG::kRopeChunks) {
      const int slot = rp * kPage + latent_swap((rd >> 4) & 3, rd & 15);
      write_lds16(tile + rp * PG::kHiBytes + PG::RI * 1024 + rd * 16, slot < n ? rope : make_uint4(0u, 0u, 0u, 0u));
    }
    lds_barrier();
  }
};

// ---------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------
// Per tile (32 slots, all heads; NHT tiles of 16 heads):
//   scores  S^T = C Q^T on v_mfma_f32_16x16x32_bf16, a wave per head tile (per
//           page of a head tile, up to 32 heads): lane (q, n) holds head n's
//           scores of slots 4q .. 4q + 3 of a page; queries stay in registers.
//   weights online softmax in base 2.  Weights are rounded once to bf16 (half a
//           step, 2^-8 of a weight), their sum is kept of the unrounded ones in
//           fp32.  The rounding adds about as much to the output's error as the
//           output's own: 2.2e-3 relative to the 64-bit result (64 sequences,
//           16 heads), 1.7e-3 with weights of 32 bits.  The grouped-query kernel
//           splits a HIGH page's weights in two; here that would double the
//           value products and the weights' way through LDS.  A head's
//           reference moves only when a score exceeds it by more than kHeadroom:
//           weights up to 2^16 are as precise as those below 1, and the sums of
//           values, which fill the registers, are left alone in the loop.
//   values  O^T += C^T P^T: wave w of W owns output elements [w R / W, (w + 1) R
//           / W) of every head, so a value is read from LDS once per workgroup;
//           weights pass through LDS in the operand order (a score lane holds
//           exactly one operand lane's weights).
// The next tiles, also across sequences, are on their way into the other LDS
// buffers meanwhile, and the page ids of the one behind them into registers.
// Up to 32 heads two workgroups of four waves share a compute unit, each with
// one tile under way; more heads take eight waves' registers, and the one
// workgroup keeps two tiles under way.  Few heads wait for their copies: 64
// sequences of 1,000-8,192 tokens, 16 heads, rank 512 are 192 MB in 54 us, 3.6
// TB/s where a plain read reaches 7.1, with 72 KiB under way per compute unit and
// 6 us before the first product.  Many wait in the chain copies - scores - values
// of a tile, the matrix cores being busy 35% of the time (128 of 1,024-8,192, 128
// heads: 157 GFLOP in 225 us, and 20 us for the merge of 100 MB of partial
// results); a LOW tile's widening is a link of that chain of its own.
// Scores of 32 heads by two waves that halve the dimensions and exchange sums
// halve the reads of keys from LDS and took 24 us more.
constexpr int latent_waves(int head_tiles) { return head_tiles >= 4 ? 8 : 4; }
constexpr int latent_ahead(int head_tiles) { return head_tiles >= 4 ? 2 : 1; }
constexpr float kHeadroom = 16.0f;

template <int R, int P, int NHT>
__global__ __launch_bounds__(64 * latent_waves(NHT), 2) void latent_attn_kernel(LatentAttnArgs a) {
  using PG = LatentPage<R, P>;
  constexpr int NW = latent_waves(NHT), T = 64 * NW;
  constexpr int KI = PG::KI, DT = R / (16 * NW);   // score steps; 16-element output tiles of a wave
  constexpr int JP = 2 * NHT <= NW ? 1 : 2;        // pages per scoring wave
  constexpr int D = latent_ahead(NHT);             // tiles under way
  constexpr int kQl = R >= 512 && NHT >= 8 ? 4 : 0;            // score steps whose queries stay in LDS: registers are full
  constexpr int QW = NHT * 2 / JP;                 // scoring waves
  static_assert(QW <= NW, "a wave per score job");
  __shared__ __align__(16) struct {
    uint8_t tile[D + 1][2 * PG::kHiBytes];
    uint8_t p[NHT * 1024];
    uint8_t q[kQl > 0 ? NHT * kQl * 1024 : 16];
    long long scan[NW + 2];
    uint8_t item[128 * 16];
    float top[QW * 16], sum[QW * 16], alpha[NHT * 16];
    int grown[QW];
  } sm;
  const CacheView& cv = a.cv;
  const int lane = (int)threadIdx.x & 63, wave = uni((int)threadIdx.x >> 6);
  const int q4 = lane >> 4, n = lane & 15;
  const int ht = JP == 1 ? wave >> 1 : wave, page0 = JP == 1 ? wave & 1 : 0;   // a scoring wave's job
  const bool scores = wave < QW;
  long long units = 1;
  const ListPlace place = find_in_list<T>(a, sm.scan, [&](long long total) {
    units = tiles_per_worker(total, a.workers, NHT);
    return (long long)blockIdx.x * units;
  });
  const long long u0 = (long long)blockIdx.x * units, u1 = u0 + units < place.total ? u0 + units : place.total;
  if (u0 >= place.total) return;
  const int e = (n & 3) >> 1;                      // value operand: quarter, slot and half of a lane's 8 bytes
  const int v_at = (e * 16 + latent_swap(e, 4 * q4 + (n >> 2))) * 16 + 8 * (n & 1) + wave * DT * 512;
  const int k_at = (16 * q4 + latent_swap(q4, n)) * 16 + page0 * PG::kHiBytes;

  // The table of the worker's tiles, 64 at a time: entry (tile - u0) mod 128.
  int walk_b = place.b;
  long long walk_start = place.start;
  auto fill = [&](long long at) {                  // tiles at .. at + 63
    if (wave == 0) {
      const Item x = look_up(a, at, walk_b, walk_start);
      write_lds16(lds_address(sm.item) + (((int)(at - u0) & 64) + fresh(lane)) * 16,
                  make_uint4((uint32_t)x.b, (uint32_t)x.what, (uint32_t)x.p0, (uint32_t)x.p1));
    }
    lds_barrier();
  };
  auto item = [&](long long u) {
    const uint4 x = read_lds16(lds_address(sm.item) + ((int)(u - u0) & 127) * 16);
    return Item{uni((int)x.x), uni((int)x.y), uni((int)x.z), uni((int)x.w)};
  };
  using TL = Tile<R, P, T>;
  // With two tiles under way the copy of a tile is issued piece by piece,
  // between the score steps: at once, each wave waited about 900 cycles for room
  // in the queue (128 heads: 288 us, 250 so).  With one under way it is issued
  // at once: the sooner the better (16 heads, 64 sequences: 53 us, 56 between
  // the steps).
  constexpr bool kBetween = D == 2;
  static_assert(!kBetween || QW == NW, "every wave scores");
  constexpr int NP = (2 * KI + NW - 1) / NW;       // pieces of a wave
  bool long_wait = true;                           // the newest copies are not a full HIGH tile's
  typename TL::Copy copy = TL::no_copy();
  auto issue = [&](int k) { TL::copy_piece(copy, wave + k * NW); };
  auto fetch = [&](const Item& x, uint8_t* tile) {
    copy = TL::copy_of(cv, x, tile);
    long_wait = !x.high() || x.p1 < 0;
  };
  uint4 qf[KI - kQl];
  const uint32_t q_at = lds_address(sm.q) + (ht * kQl * 64 + lane) * 16;
  auto load_queries = [&](int b) {
    const int l = fresh(lane), head = ht * 16 + (l & 15);
    const uint16_t* src = a.q + ((size_t)b * a.heads + head) * (R + P) + 8 * (l >> 4);
#pragma unroll
    for (int i = 0; i < KI; ++i) {
      const uint4 x =
          scores && head < a.heads ? *reinterpret_cast<const uint4*>(src + 32 * i) : make_uint4(0u, 0u, 0u, 0u);
      if (i < KI - kQl) qf[i] = x;
      else if (scores) write_lds16(fresh(q_at) + (i - KI + kQl) * 1024, x);
    }
  };
  f32x4_t acc[NHT][DT];
  float x[4 * JP], mx, sum, part = 0.0f, top = -INFINITY;      // scaled scores of the tile, reference, sums
  auto restart = [&]() {
#pragma unroll
    for (int h = 0; h < NHT; ++h)
#pragma unroll
      for (int m = 0; m < DT; ++m) acc[h][m] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    mx = -INFINITY;
    sum = 0.0f;
  };
  auto weigh = [&]() {                             // weights of x into LDS
    const float base = mx == -INFINITY ? 0.0f : mx;
    float w[4 * JP];
    part = 0.0f;
    const uint32_t p_at = lds_address(sm.p) + (ht * 64 + fresh(lane)) * 16 + page0 * 8;
#pragma unroll
    for (int r = 0; r < 4 * JP; ++r) {
      w[r] = __builtin_amdgcn_exp2f(x[r] - base);
      part += w[r];
    }
#pragma unroll
    for (int jp = 0; jp < JP; ++jp)
      write_lds8(p_at + jp * 8,
                 make_uint2(pack_bf16x2(w[4 * jp], w[4 * jp + 1]), pack_bf16x2(w[4 * jp + 2], w[4 * jp + 3])));
  };
  // Scores and weights of a tile in LDS, and the copies of the tile ahead; true for every wave if some head's
  // reference has to move first (move_reference).
  auto score = [&](const Item& at, uint8_t* tile) {
    const int m = at.slots();
    if (!at.high() && m > 0) {
      TL::widen_low(tile, m);
    } else if (m < kTile) {                        // a HIGH store's last tile, or an empty sequence's
      TL::clear_from(tile, m);
      lds_barrier();
    }
    if (scores) {
      // Two sums at a time (the two pages, or even and odd steps of one), the
      // operands of kAhead steps read in advance: in pinned order, as left to
      // itself the compiler saves registers and waits for every read.
      constexpr int kAhead = JP == 1 ? 6 : (NHT >= 8 ? 2 : 3);
      // Addresses are formed here: kept in registers, they would push others out.
      const uint32_t kb = lds_address(tile) + fresh(k_at), qb = fresh(q_at);
      auto operand = [&](int i, int jp) { return read_lds16(kb + jp * PG::kHiBytes + i * 1024); };
      f32x4_t s[2] = {f32x4_t{0.0f, 0.0f, 0.0f, 0.0f}, f32x4_t{0.0f, 0.0f, 0.0f, 0.0f}};
      // Steps whose queries are in LDS come last.
      auto queries = [&](int i) { return i < KI - kQl ? qf[i] : read_lds16(qb + (i - KI + kQl) * 1024); };
      uint4 kf[kAhead][JP], ql[2];
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
#pragma unroll
        for (int jp = 0; jp < JP; ++jp) kf[i][jp] = operand(i, jp);
#pragma unroll
      for (int i = 0; i < KI; ++i) {
        const uint4 qi = i < KI - kQl ? qf[i] : ql[i & 1];
#pragma unroll
        for (int jp = 0; jp < JP; ++jp) {
          f32x4_t& to = s[JP == 1 ? i & 1 : jp];
          to = mfma(kf[i % kAhead][jp], qi, to);
          if (i + kAhead < KI) kf[i % kAhead][jp] = operand(i + kAhead, jp);
        }
        if (kQl > 0 && i + 2 >= KI - kQl && i + 2 < KI) ql[i & 1] = queries(i + 2);
        if (kBetween && i * NP / KI != (i + 1) * NP / KI) issue(i * NP / KI);
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (JP == 1) s[0] += s[1];
      top = -INFINITY;
      const int left = m - page0 * kPage - 4 * (fresh(lane) >> 4);
#pragma unroll
      for (int r = 0; r < 4 * JP; ++r) {
        x[r] = (r >> 2) * kPage + (r & 3) < left ? s[r >> 2][r & 3] * a.scale_log2 : -INFINITY;
        top = fmaxf(top, x[r]);
      }
      weigh();
      const bool grown = __ballot(top > mx + kHeadroom) != 0ull;
      if (lane == 0) sm.grown[wave] = grown;
    }
    lds_barrier();
    int grown = 0;
#pragma unroll
    for (int w = 0; w < QW; ++w) grown |= sm.grown[w];
    return uni(grown) != 0;
  };
  auto move_reference = [&]() {
    if (scores) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      if (q4 == 0) sm.top[wave * 16 + n] = top;
    }
    lds_barrier();
    if (scores) {
      if constexpr (JP == 1) top = fmaxf(top, sm.top[(wave ^ 1) * 16 + n]);
      const float ref = top > mx + kHeadroom ? top : mx;
      const float alpha = ref == mx ? 1.0f : __builtin_amdgcn_exp2f(mx - ref);
      mx = ref;
      sum *= alpha;
      weigh();
      if (q4 == 0 && page0 == 0) sm.alpha[ht * 16 + n] = alpha;
    }
    lds_barrier();
#pragma unroll
    for (int h = 0; h < NHT; ++h) {
      const float alpha = sm.alpha[h * 16 + n];
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[h][d] *= alpha;
    }
  };
  auto add_values = [&](const uint8_t* tile) {
    const uint32_t vs = lds_address(tile) + fresh(v_at), ps = lds_address(sm.p) + fresh(lane) * 16;
    constexpr int kW = NHT < 4 ? NHT : 4;          // weights read in advance
    uint4 w[kW], v[DT > 4 ? 8 : 4];
#pragma unroll
    for (int h = 0; h < kW; ++h) w[h] = read_lds16(ps + h * 1024);
    if constexpr (DT > 4) {
      read_transposed8<PG::kHiBytes>(vs, v);
    } else {
      constexpr int k1 = DT > 1 ? 512 : 0, k2 = DT > 2 ? 1024 : 0, k3 = DT > 3 ? 1536 : 0;
      read_transposed<0, k1, k2, k3, PG::kHiBytes>(vs, vs, vs, vs, v);
    }
#pragma unroll
    for (int h = 0; h < NHT; ++h) {
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[h][d] = mfma(v[d], w[h % kW], acc[h][d]);
      if (h + kW < NHT) w[h % kW] = read_lds16(ps + (h + kW) * 1024);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  long long u = u0, seq_u = u0;                    // the current tile; the first here of its sequence
  int buf = 0;                                     // its buffer
  auto buffer = [&](int k) {
    const int x = buf + k;
    return sm.tile[x > D ? x - D - 1 : x];
  };
  fill(u0);
  Item cur = item(u0);
  load_queries(cur.b);
  restart();
#pragma unroll
  for (int k = 0; k < D; ++k)
    if (u + k < u1) {
      fetch(item(u + k), buffer(k));
      for (int j = 0; j < NP; ++j) issue(j);
    }
  wait_loads();
  __syncthreads();
  // With every wave done with the tile before: the tile that goes into its buffer.
  auto look_ahead = [&]() {
    copy = TL::no_copy();
    if (u + D >= u1) return;
    if (((u + D - u0) & 63) == 0) fill(u + D);
    fetch(item(u + D), buffer(D));
    if (!kBetween) {
#pragma unroll
      for (int k = 0; k < NP; ++k) issue(k);
    }
  };
  auto advance = [&]() {
    ++u;
    buf = buf == D ? 0 : buf + 1;
    // The next tile has arrived when only the newest one's copies are under way.
    constexpr int kNewest = 2 * PG::KI / NW;       // at least, of each wave
    static_assert(kNewest < 16, "in the counter's low bits");
    if (D == 1 || long_wait || u + D > u1) wait_loads();
    else __builtin_amdgcn_s_waitcnt(0x0F70 | kNewest);
    lds_barrier();
    cur = item(u);
  };
  look_ahead();
  bool grown = score(cur, sm.tile[0]);
  bool later = false, begun = cur.first();         // not the worker's first sequence; the sequence's first tile was here
  for (;;) {
    if (grown) move_reference();
    bool ends;
    for (;;) {                                     // tiles of one sequence, until a reference has to move
      sum += part;
      add_values(sm.tile[buf]);
      ends = cur.last() || u + 1 == u1;            // the worker's last tile of this sequence
      if (ends) break;
      advance();
      look_ahead();
      grown = score(cur, sm.tile[buf]);
      if (grown) break;
    }
    if (!ends) continue;

    // Results: the whole history, or a part of it in slot 2w (the worker's
    // first sequence) or 2w + 1 of the partials.
    const int b = cur.b;
    const bool whole = begun && cur.last();
    const int slot = 2 * (int)blockIdx.x + (later ? 1 : 0);
    if (threadIdx.x == 0 && begun) {
      int parts = 0;
      if (!whole) {                                // it goes on to u1 and further
        const Counts c = counts_at(a, b);
        const long long rest = tiles_of(c) - (u + 1 - seq_u);
        parts = 1 + (int)((rest + units - 1) / units);
      }
      a.ws_seq[2 * b] = slot;
      a.ws_seq[2 * b + 1] = parts;
    }
    if (scores) {
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (q4 == 0) sm.sum[wave * 16 + n] = sum;
    }
    lds_barrier();
    if (scores && page0 == 0 && q4 == 0) {
      if constexpr (JP == 1) sum += sm.sum[(wave + 1) * 16 + n];
      const int head = ht * 16 + n;
      sm.alpha[head] = sum == 0.0f ? 0.0f : 1.0f / sum;
      if (whole) {
        if (a.lse && head < a.heads)
          a.lse[(size_t)b * a.heads + head] = sum == 0.0f ? -INFINITY : (mx + __builtin_amdgcn_logf(sum)) * kLn2;
      } else {
        float* ml = a.ws_ml + ((size_t)slot * NHT * 16 + head) * 2;
        ml[0] = mx;
        ml[1] = sum;
      }
    }
    const bool more = u + 1 < u1;
    if (more) load_queries(item(u + 1).b);
    lds_barrier();
    const int l = fresh(lane);
#pragma unroll
    for (int h = 0; h < NHT; ++h) {
      const int head = h * 16 + (l & 15);
      if (head < a.heads) {
        const float inv = sm.alpha[head];
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const int dim = 16 * (wave * DT + d) + 4 * (l >> 4);
          const f32x4_t o = acc[h][d];
          if (whole) {
            *reinterpret_cast<uint2*>(a.out + ((size_t)b * a.heads + head) * R + dim) =
                make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
          } else {
            *reinterpret_cast<f32x4_t*>(a.ws_o + ((size_t)slot * NHT * 16 + head) * R + dim) = o;
          }
        }
      }
    }
    if (!more) return;
    restart();
    long_wait = true;                              // results have been stored since
    advance();
    later = true;
    begun = true;
    seq_u = u;
    look_ahead();
    grown = score(cur, sm.tile[buf]);
  }
}

// ---------------------------------------------------------------------------
// merge
// ---------------------------------------------------------------------------
// The partials of a head: maxima and sums give each one's weight, then the
// weighted values are added in order of the partials (slot of the first, then
// the first slots of the workers after it).  Up to 8 partials: a wave per head.
// More: a workgroup per slice of a head, R / (8 slices) lanes to a partial, as
// many partials at a time as fit, added up through LDS.  With few heads in the
// call a head is cut into slices, down to 64 elements (376 partials of 20 heads:
// 17 us whole, 8.5 in 8 slices); with enough to fill the chip it is not (64
// sequences of 16 heads: 6.6 us whole, 12 in slices, each of which finds the
// maximum again).
template <int R>
__global__ __launch_bounds__(kThreads) void latent_merge_kernel(LatentAttnArgs a, int tile_heads, int log_slices) {
  constexpr int E = R / 64;                        // elements per lane of a wave's head
  __shared__ f32x4_t s_o[2][kThreads];
  __shared__ float s_w[kThreads / 8];
  const int b = blockIdx.y, lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  const int first = a.ws_seq[2 * b], n = a.ws_seq[2 * b + 1];
  if (n == 0) return;
  auto slot = [&](int k) { return k == 0 ? first : 2 * (first / 2 + k); };
  auto maxima = [&](int h) {
    float top = -INFINITY;
    for (int k = lane; k < n; k += 64) top = fmaxf(top, a.ws_ml[((size_t)slot(k) * tile_heads + h) * 2]);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
    return top;
  };
  if (n <= 8) {
    for (int h = (int)blockIdx.x * kWaves + wave; h < a.heads; h += (int)gridDim.x * kWaves) {
      const float top = maxima(h), base = top == -INFINITY ? 0.0f : top;
      float o[E] = {}, total = 0.0f;
#pragma unroll 4
      for (int k = 0; k < n; ++k) {
        const size_t at = (size_t)slot(k) * tile_heads + h;
        const float2 ml = *reinterpret_cast<const float2*>(a.ws_ml + at * 2);
        const float* src = a.ws_o + at * R + lane * E;
        const float w = __builtin_amdgcn_exp2f(ml.x - base);
        total += w * ml.y;
#pragma unroll
        for (int u = 0; u < E; ++u) o[u] += w * src[u];
      }
      const float inv = total == 0.0f ? 0.0f : 1.0f / total;
      const size_t at = (size_t)b * a.heads + h;
      uint32_t* dst = reinterpret_cast<uint32_t*>(a.out + at * R + lane * E);
#pragma unroll
      for (int u = 0; u < E / 2; ++u) dst[u] = pack_bf16x2(o[2 * u] * inv, o[2 * u + 1] * inv);
      if (lane == 0 && a.lse) a.lse[at] = total == 0.0f ? -INFINITY : (base + __builtin_amdgcn_logf(total)) * kLn2;
    }
    return;
  }
  const int lanes = (R / 8) >> log_slices, groups = kThreads / lanes;
  const int g = (int)threadIdx.x / lanes, l = (int)threadIdx.x - g * lanes;
  for (int x = blockIdx.x; x < a.heads << log_slices; x += gridDim.x) {
    const int h = x >> log_slices, part = x - (h << log_slices), e = (part * lanes + l) * 8;
    const float top = maxima(h), base = top == -INFINITY ? 0.0f : top;
    f32x4_t o[2] = {f32x4_t{0.0f, 0.0f, 0.0f, 0.0f}, f32x4_t{0.0f, 0.0f, 0.0f, 0.0f}};
    float total = 0.0f;
#pragma unroll 4
    for (int k = g; k < n; k += groups) {
      const size_t at = (size_t)slot(k) * tile_heads + h;
      const float2 ml = *reinterpret_cast<const float2*>(a.ws_ml + at * 2);
      const f32x4_t* v = reinterpret_cast<const f32x4_t*>(a.ws_o + at * R + e);
      const float w = __builtin_amdgcn_exp2f(ml.x - base);
      total += w * ml.y;
      o[0] += v[0] * w;
      o[1] += v[1] * w;
    }
    __syncthreads();                               // the sums before have been read
    s_o[0][threadIdx.x] = o[0];
    s_o[1][threadIdx.x] = o[1];
    if (l == 0) s_w[g] = total;
    __syncthreads();
    if (g > 0) continue;
    for (int i = 1; i < groups; ++i) {
      o[0] += s_o[0][i * lanes + l];
      o[1] += s_o[1][i * lanes + l];
      total += s_w[i];
    }
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    const size_t at = (size_t)b * a.heads + h;
    *reinterpret_cast<uint4*>(a.out + at * R + e) =
        make_uint4(pack_bf16x2(o[0][0] * inv, o[0][1] * inv), pack_bf16x2(o[0][2] * inv, o[0][3] * inv),
                   pack_bf16x2(o[1][0] * inv, o[1][1] * inv), pack_bf16x2(o[1][2] * inv, o[1][3] * inv));
    if (e == 0 && a.lse) a.lse[at] = total == 0.0f ? -INFINITY : (base + __builtin_amdgcn_logf(total)) * kLn2;
  }
}

template <int R, int P>
void launch_heads(const LatentAttnArgs& a, hipStream_t s) {
  const dim3 grid(a.workers), block(64 * latent_waves(latent_head_tiles(a.heads)));
  switch (latent_head_tiles(a.heads)) {
    case 1: latent_attn_kernel<R, P, 1><<<grid, block, 0, s>>>(a); break;
    case 2: latent_attn_kernel<R, P, 2><<<grid, block, 0, s>>>(a); break;
    case 4: latent_attn_kernel<R, P, 4><<<grid, block, 0, s>>>(a); break;
    default: latent_attn_kernel<R, P, 8><<<grid, block, 0, s>>>(a); break;
  }
}

}  // namespace

int latent_workers(int heads, int64_t tiles) {
  const int resident = latent_head_tiles(heads) >= 4 ? 256 : 512;
  return (int)std::max<int64_t>(1, std::min<int64_t>(resident, tiles));
}

hipError_t launch_latent_attention(const LatentAttnArgs& a, hipStream_t s) {
  if (a.rope == 32) {
    if (a.rank == 128) launch_heads<128, 32>(a, s);
    else if (a.rank == 256) launch_heads<256, 32>(a, s);
    else launch_heads<512, 32>(a, s);
  } else {
    if (a.rank == 128) launch_heads<128, 64>(a, s);
    else if (a.rank == 256) launch_heads<256, 64>(a, s);
    else launch_heads<512, 64>(a, s);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.workers == 1) return hipSuccess;           // nothing is shared
  const int heads = 16 * latent_head_tiles(a.heads);
  constexpr int kBlocks = 1024;
  int log_slices = 0;
  while ((a.rank / 64) >> (log_slices + 1) && ((int64_t)a.batch * a.heads << (log_slices + 1)) <= kBlocks) ++log_slices;
  const dim3 grid(std::max(1, std::min(a.heads << log_slices, kBlocks / a.batch)), a.batch);
  if (a.rank == 128) latent_merge_kernel<128><<<grid, dim3(kThreads), 0, s>>>(a, heads, log_slices);
  else if (a.rank == 256) latent_merge_kernel<256><<<grid, dim3(kThreads), 0, s>>>(a, heads, log_slices);
  else latent_merge_kernel<512><<<grid, dim3(kThreads), 0, s>>>(a, heads, log_slices);
  return hipGetLastError();
}

}  // namespace pask
