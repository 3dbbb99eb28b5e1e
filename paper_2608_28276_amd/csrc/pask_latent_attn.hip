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
struct Seq {
  int b, n_hi, n_lo, nt_hi, nt;
  // Slots of tile j (0 or less: the tile of an empty sequence).
  __device__ __forceinline__ int slots(int j) const {
    return j < nt_hi ? min(kTile, n_hi - j * kTile) : min(kTile, n_lo - (j - nt_hi) * kTile);
  }
};
__device__ __forceinline__ Seq seq_at(const LatentAttnArgs& a, int b) {
  const int32_t* c = counters_of(a.cv, b, a.layer);
  Seq s;
  s.b = b;
  s.n_hi = c[kCntHi];
  s.n_lo = c[kCntLo];
  s.nt_hi = (s.n_hi + kTile - 1) / kTile;
  s.nt = max(1, s.nt_hi + (s.n_lo + kTile - 1) / kTile);
  return s;
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
  long long mine = 0;
  const int first = (int)((long long)a.batch * tid / T), last = (int)((long long)a.batch * (tid + 1) / T);
  for (int b = first; b < last; ++b) mine += seq_at(a, b).nt;
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
    for (int nt; start + (nt = seq_at(a, b).nt) <= x; ++b) start += nt;
    s_scan[kWaves] = start;
    s_scan[kWaves + 1] = b;
  }
  __syncthreads();
  return ListPlace{total, s_scan[kWaves], (int)s_scan[kWaves + 1]};
}

// ---------------------------------------------------------------------------
// one tile into LDS
// ---------------------------------------------------------------------------
// A HIGH tile is the two pages as they lie, copied without passing through
// registers.  A LOW tile's codes, scales and rotary keys pass through registers
// (loaded while the tile before is attended) and are widened on their way.
template <int R, int P, int T>
struct Tile {
  using PG = LatentPage<R, P>;
  static constexpr int NC = (2 * PG::kGroups + T - 1) / T;     // code groups per thread of two LOW pages
  uint4 codes[NC], rope;
  uint16_t scale[NC];

  // p0, p1: the two pages (p1 negative: none).  kWaves waves share the 1 KiB pieces.
  __device__ __forceinline__ static void copy_high(const uint8_t* pool, int p0, int p1, uint8_t* tile, int wave,
                                                   int lane) {
    const uint8_t* b0 = pool + (size_t)p0 * PG::kHiBytes;
    const uint8_t* b1 = pool + (size_t)p1 * PG::kHiBytes - PG::kHiBytes;
    const int n = p1 < 0 ? PG::KI : 2 * PG::KI;
#pragma unroll
    for (int k = 0; k < (2 * PG::KI + T / 64 - 1) / (T / 64); ++k) {
      const int x = wave + k * (T / 64);
      if (x < n) load_to_lds<true>((x < PG::KI ? b0 : b1) + x * 1024 + lane * 16, tile + x * 1024);
    }
  }
  // Slots from n on as zeros: what lies there is not an entry (any bytes, NaN
  // among them), and a weight of 0 does not make a NaN value harmless.
  __device__ __forceinline__ static void clear_from(uint8_t* tile, int n) {
    for (int c = (int)threadIdx.x; c < 2 * PG::kHiChunks; c += T) {
      const int page = c < PG::kHiChunks ? 0 : 1, d = c - page * PG::kHiChunks;
      if (page * kPage + latent_swap((d >> 4) & 3, d & 15) >= n)
        reinterpret_cast<uint4*>(tile)[c] = make_uint4(0u, 0u, 0u, 0u);
    }
  }
  __device__ __forceinline__ void load_low(const uint8_t* pool, int p0, int p1) {
    const uint8_t* b0 = pool + (size_t)p0 * PG::kLoBytes;
    const uint8_t* b1 = pool + (size_t)(p1 < 0 ? p0 : p1) * PG::kLoBytes;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int g = (int)threadIdx.x + T * k, h = g < PG::kGroups ? g : g - PG::kGroups;
      const uint8_t* pg = g < PG::kGroups ? b0 : b1;
      if (g < 2 * PG::kGroups) {
        codes[k] = stream_load16(pg + h * 16);
        scale[k] = *reinterpret_cast<const uint16_t*>(pg + PG::kScales + 2 * h);
      }
    }
    const int c = (int)threadIdx.x, d = c < PG::kRopeChunks ? c : c - PG::kRopeChunks;
    static_assert(2 * PG::kRopeChunks <= T, "a rotary piece per thread");
    if (c < 2 * PG::kRopeChunks) rope = stream_load16((c < PG::kRopeChunks ? b0 : b1) + PG::kRopeAt + d * 16);
  }
  __device__ __forceinline__ void store_low(uint8_t* tile, int n) const {
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int g = (int)threadIdx.x + T * k, page = g < PG::kGroups ? 0 : 1, h = g - page * PG::kGroups;
      if (g < 2 * PG::kGroups) {
        const int t = h & 15;
        const bool in = page * kPage + t < n;
        const float s = half_value(scale[k]);
        const uint32_t w[4] = {codes[k].x, codes[k].y, codes[k].z, codes[k].w};
        uint8_t* dst = tile + page * PG::kHiBytes + (h >> 4) * 1024;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint4 v = low_values(w[q], s);
          *reinterpret_cast<uint4*>(dst + (16 * q + latent_swap(q, t)) * 16) = in ? v : make_uint4(0u, 0u, 0u, 0u);
        }
      }
    }
    const int c = (int)threadIdx.x, page = c < PG::kRopeChunks ? 0 : 1, d = c - page * PG::kRopeChunks;
    if (c < 2 * PG::kRopeChunks) {
      const int slot = page * kPage + latent_swap((d >> 4) & 3, d & 15);
      *reinterpret_cast<uint4*>(tile + page * PG::kHiBytes + PG::RI * 1024 + d * 16) =
          slot < n ? rope : make_uint4(0u, 0u, 0u, 0u);
    }
  }
};

// ---------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------
// Per tile (32 slots, all heads; NHT tiles of 16 heads):
//   scores  S^T = C Q^T on v_mfma_f32_16x16x32_bf16, a wave per head tile:
//           lane (q, n) holds head n's scores of slots 4q .. 4q + 3 of both
//           pages; queries stay in registers.
//   weights online softmax in base 2; the reference m of a head moves only
//           when a tile's maximum exceeds it by more than 8, so weights stay
//           below 2^8 and the sums are rarely rescaled.  Weights are rounded
//           to bf16 (half a step, 2^-8 of a weight; independent over slots, so
//           it averages out below the output's own rounding); their sum is
//           kept of the unrounded ones in fp32.
//   values  O^T += C^T P^T: wave w of W owns output elements [w R / W, (w + 1) R
//           / W) of every head, so a value is read from LDS once per workgroup;
//           weights pass through LDS in the operand order (a score lane holds
//           exactly one operand lane's 8 weights).
// The next tile, also across sequences, is on its way into the other LDS
// buffer meanwhile.
constexpr int latent_waves(int head_tiles) { return head_tiles >= 8 ? 8 : 4; }

template <int R, int P, int NHT>
__global__ __launch_bounds__(64 * latent_waves(NHT), 2) void latent_attn_kernel(LatentAttnArgs a) {
  using PG = LatentPage<R, P>;
  constexpr int NW = latent_waves(NHT), T = 64 * NW;
  constexpr int KI = PG::KI, DT = R / (16 * NW);   // score steps; 16-element output tiles of a wave
  __shared__ __align__(16) struct {
    uint8_t tile[2][2 * PG::kHiBytes];
    uint4 p[NHT * 64];
    long long scan[NW + 2];
    float alpha[NHT * 16];
    int grown[NHT];
  } sm;
  const CacheView& cv = a.cv;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int q4 = lane >> 4, n = lane & 15;
  long long units = 1;
  const ListPlace place = find_in_list<T>(a, sm.scan, [&](long long total) {
    units = (total + a.workers - 1) / a.workers;
    return (long long)blockIdx.x * units;
  });
  const long long u0 = (long long)blockIdx.x * units, u1 = u0 + units < place.total ? u0 + units : place.total;
  if (u0 >= place.total) return;
  const int e = (n & 3) >> 1;                      // value operand: quarter, slot and half of a lane's 8 bytes
  const int v_at = (e * 16 + ((4 * q4 + (n >> 2)) ^ (8 * e))) * 16 + 8 * (n & 1) + wave * DT * 512;
  const int k_at = (16 * q4 + latent_swap(q4, n)) * 16;
  Tile<R, P, T> low;
  auto fetch = [&](const Seq& s, int j, uint8_t* tile) {
    const int m = s.slots(j);
    if (m <= 0) return;
    const bool high = j < s.nt_hi;
    const int32_t* bt = block_table_of(cv, s.b, a.layer, high ? kHi : kLo) + 2 * (high ? j : j - s.nt_hi);
    const int p0 = bt[0], p1 = m > kPage ? bt[1] : -1;
    if (high) Tile<R, P, T>::copy_high(cv.hi_pool, p0, p1, tile, wave, lane);
    else low.load_low(cv.lo_pool, p0, p1);
  };
  uint4 qf[KI];
  auto load_queries = [&](int b) {
    const int head = wave * 16 + n;
    const uint16_t* src = a.q + ((size_t)b * a.heads + head) * (R + P) + 8 * q4;
#pragma unroll
    for (int i = 0; i < KI; ++i)
      qf[i] = wave < NHT && head < a.heads ? *reinterpret_cast<const uint4*>(src + 32 * i) : make_uint4(0u, 0u, 0u, 0u);
  };
  f32x4_t acc[NHT][DT];
  float mx = -INFINITY, sum = 0.0f;
  auto restart = [&]() {
#pragma unroll
    for (int h = 0; h < NHT; ++h)
#pragma unroll
      for (int m = 0; m < DT; ++m) acc[h][m] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    mx = -INFINITY;
    sum = 0.0f;
  };
  restart();

  Seq s = seq_at(a, place.b);
  long long start = place.start;                   // the list's tile 0 of sequence s
  int j = (int)(u0 - start), buf = 0;
  load_queries(s.b);
  fetch(s, j, sm.tile[0]);
  if (j >= s.nt_hi && s.slots(j) > 0) low.store_low(sm.tile[0], s.slots(j));
  wait_loads();
  __syncthreads();
  for (long long u = u0; u < u1; ++u) {
    uint8_t* tile = sm.tile[buf];
    uint8_t* other = sm.tile[buf ^ 1];
    const int m = s.slots(j);
    const bool ends = j + 1 == s.nt || u + 1 == u1;             // the worker's last tile of this sequence
    Seq next = s;
    int nj = j + 1;
    if (j + 1 == s.nt && u + 1 < u1) {
      next = seq_at(a, s.b + 1);
      nj = 0;
    }
    if (u + 1 < u1) fetch(next, nj, other);
    if (m < kTile && (j < s.nt_hi || m <= 0)) {    // a HIGH store's last tile, or an empty sequence's
      Tile<R, P, T>::clear_from(tile, m);
      lds_barrier();
    }
    if (wave < NHT) {
      f32x4_t s0 = {0.0f, 0.0f, 0.0f, 0.0f}, s1 = s0;
#pragma unroll
      for (int i = 0; i < KI; ++i) {
        s0 = mfma(*reinterpret_cast<const uint4*>(tile + i * 1024 + k_at), qf[i], s0);
        s1 = mfma(*reinterpret_cast<const uint4*>(tile + PG::kHiBytes + i * 1024 + k_at), qf[i], s1);
      }
      float x[8], top = -INFINITY;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const int slot = (r < 4 ? 0 : kPage) + 4 * q4 + (r & 3);
        x[r] = slot < m ? (r < 4 ? s0[r & 3] : s1[r & 3]) * a.scale_log2 : -INFINITY;
        top = fmaxf(top, x[r]);
      }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float ref = top > mx + 8.0f ? top : mx;
      const float alpha = ref == mx ? 1.0f : __builtin_amdgcn_exp2f(mx - ref);
      mx = ref;
      const float base = ref == -INFINITY ? 0.0f : ref;
      float part = 0.0f;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        x[r] = __builtin_amdgcn_exp2f(x[r] - base);
        part += x[r];
      }
      sum = sum * alpha + part;
      sm.p[wave * 64 + lane] = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                                         pack_bf16x2(x[6], x[7]));
      if (q4 == 0) sm.alpha[wave * 16 + n] = alpha;
      const bool grown = __ballot(alpha != 1.0f) != 0ull;
      if (lane == 0) sm.grown[wave] = grown;
    }
    lds_barrier();
    int grown = 0;
#pragma unroll
    for (int h = 0; h < NHT; ++h) grown |= sm.grown[h];
    if (__builtin_amdgcn_readfirstlane(grown)) {
#pragma unroll
      for (int h = 0; h < NHT; ++h) {
        const float alpha = sm.alpha[h * 16 + n];
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[h][d] *= alpha;
      }
    }
    uint4 pf[NHT];
#pragma unroll
    for (int h = 0; h < NHT; ++h) pf[h] = sm.p[h * 64 + lane];
    const uint32_t vs = lds_address(tile) + v_at;
    auto add_values = [&](auto first) {            // output tiles first .. + 3 (those below DT)
      constexpr int d0 = decltype(first)::value, k = d0 * 512;
      constexpr int k1 = DT > d0 + 1 ? k + 512 : k, k2 = DT > d0 + 2 ? k + 1024 : k, k3 = DT > d0 + 3 ? k + 1536 : k;
      uint4 v[4];
      read_transposed<k, k1, k2, k3, PG::kHiBytes>(vs, vs, vs, vs, v);
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int h = 0; h < NHT; ++h)
          if (d0 + d < DT) acc[h][d0 + d] = mfma(v[d], pf[h], acc[h][d0 + d]);
    };
    add_values(std::integral_constant<int, 0>{});
    if constexpr (DT > 4) add_values(std::integral_constant<int, 4>{});
    if (u + 1 < u1 && nj >= next.nt_hi && next.slots(nj) > 0) low.store_low(other, next.slots(nj));

    if (ends) {
      // Results: the whole history, or a part of it in slot 2w (the worker's
      // first sequence) or 2w + 1 of the partials.
      const bool whole = start >= u0 && start + s.nt <= u1;
      const int part = 2 * (int)blockIdx.x + (start > u0 ? 1 : 0);
      if (threadIdx.x == 0 && start >= u0) {
        a.ws_seq[2 * s.b] = part;
        a.ws_seq[2 * s.b + 1] = whole ? 0 : (int)((start + s.nt - 1) / units) - (int)blockIdx.x + 1;
      }
      lds_barrier();                               // the scale factors have been read
      if (wave < NHT) {
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        const int head = wave * 16 + n;
        if (q4 == 0) {
          sm.alpha[head] = sum == 0.0f ? 0.0f : 1.0f / sum;
          if (whole) {
            if (a.lse && head < a.heads)
              a.lse[(size_t)s.b * a.heads + head] =
                  sum == 0.0f ? -INFINITY : (mx + __builtin_amdgcn_logf(sum)) * kLn2;
          } else {
            float* ml = a.ws_ml + ((size_t)part * NHT * 16 + head) * 2;
            ml[0] = mx;
            ml[1] = sum;
          }
        }
      }
      if (u + 1 < u1) load_queries(next.b);
      lds_barrier();
#pragma unroll
      for (int h = 0; h < NHT; ++h) {
        const int head = h * 16 + n;
        if (head < a.heads) {
          const float inv = sm.alpha[head];
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const int dim = 16 * (wave * DT + d) + 4 * q4;
            const f32x4_t o = acc[h][d];
            if (whole) {
              *reinterpret_cast<uint2*>(a.out + ((size_t)s.b * a.heads + head) * R + dim) =
                  make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
            } else {
              *reinterpret_cast<f32x4_t*>(a.ws_o + ((size_t)part * NHT * 16 + head) * R + dim) = o;
            }
          }
        }
      }
      restart();
      if (nj == 0) start += s.nt;
    }
    s = next;
    j = nj;
    buf ^= 1;
    wait_loads();
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// merge
// ---------------------------------------------------------------------------
// A wave per head: the partials' maxima and sums give each one's weight, then
// the sums of values are added in order of the partials (slot of the first,
// then the first slots of the workers after it).
template <int R>
__global__ __launch_bounds__(kThreads) void latent_merge_kernel(LatentAttnArgs a, int tile_heads) {
  const int b = blockIdx.y, lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
  const int first = a.ws_seq[2 * b], n = a.ws_seq[2 * b + 1];
  if (n == 0) return;
  constexpr int E = R / 64;                        // elements per lane
  auto slot = [&](int k) { return k == 0 ? first : 2 * (first / 2 + k); };
  for (int h = (int)blockIdx.x * kWaves + wave; h < a.heads; h += (int)gridDim.x * kWaves) {
    float top = -INFINITY;
    for (int k = lane; k < n; k += 64) top = fmaxf(top, a.ws_ml[((size_t)slot(k) * tile_heads + h) * 2]);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
    const float base = top == -INFINITY ? 0.0f : top;
    float o[E] = {}, total = 0.0f;
    for (int k = 0; k < n; ++k) {
      const size_t at = (size_t)slot(k) * tile_heads + h;
      const float w = __builtin_amdgcn_exp2f(a.ws_ml[at * 2] - base);
      total += w * a.ws_ml[at * 2 + 1];
      const float* src = a.ws_o + at * R + lane * E;
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

int latent_workers(int rank, int rope, int heads, int64_t tiles) {
  (void)rank;
  (void)rope;
  const int resident = latent_head_tiles(heads) >= 8 ? 256 : 512;
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
  const dim3 grid(std::max(1, std::min((a.heads + kWaves - 1) / kWaves, 1024 / a.batch)), a.batch);
  if (a.rank == 128) latent_merge_kernel<128><<<grid, dim3(kThreads), 0, s>>>(a, heads);
  else if (a.rank == 256) latent_merge_kernel<256><<<grid, dim3(kThreads), 0, s>>>(a, heads);
  else latent_merge_kernel<512><<<grid, dim3(kThreads), 0, s>>>(a, heads);
  return hipGetLastError();
}

}  // namespace pask
