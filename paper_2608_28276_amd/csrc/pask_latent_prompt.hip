// gfx950 kernel of the expanded latent attention: causal attention of packed,
// ragged prompts, with keys (per-head part, shared rotary key) and values per
// head.
#include <hip/hip_runtime.h>

#include <math.h>

#include <algorithm>
#include <type_traits>

#include "pask_latent_device.h"

namespace pask {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kKeys = 64;                          // keys of a step
// The reference of a query's weights moves only when a score exceeds it by more
// than this (in base 2).  Weights up to 2^16 and their sums are as precise as
// weights below 1 (bf16 and fp32 have the same exponents); the sums stay below the
// largest fp32 for values that sum to less than 2^112, the bound the header
// gives.  (A reference 2^16 higher would trade that for entries lost at 2^-110 of
// the largest weight in place of 2^-126.)  A reference that follows every maximum
// costs a multiplication of all sums in the loop, which the compiler answers with
// copies of them.
constexpr float kHeadroom = 16.0f;
constexpr int kAhead = 4;                          // score operands read ahead of their product
constexpr float kLn2 = 0.6931471805599453f;

// D[32x32] += A[32x16] B[16x32]: lane l holds A[l % 32][8 (l / 32) ..], B[8 (l / 32) ..][l % 32], and
// D[8 (r / 4) + 4 (l / 32) + r % 4][l % 32], r < 16.
__device__ __forceinline__ f32x16_t mfma(uint4 a, uint4 b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0,
                                                 0, 0);
}
// Rows of C 16-byte chunks in LDS, row t's chunk d at t * C + swap(t, d): the
// operand reads, 8 neighbouring rows' chunk d at once, fall on all banks
// (256 / (16 C) rows share the 64 banks).
template <int C>
__device__ __forceinline__ int key_swap(int t, int d) { return d ^ ((C >= 16 ? t : t / (16 / C)) & (C - 1)); }
// The same for values, which the transposing reads take 4 rows x 4 chunks at a time.
template <int C>
__device__ __forceinline__ int value_swap(int t, int d) { return d ^ ((t / (16 / C) & (C / 4 - 1)) << 2); }

// O += P V key by key over 32 keys (values at s_v), where a value that some
// query does not see is infinite or NaN (a weight of 0 times it is not 0): only
// keys up to `see` are added.  Lane (g, n) holds the weights of query n for half
// of the keys, lane (1 - g, n) the others'; the weights move down one register
// a turn.
template <int VT, int VC>
__device__ __forceinline__ void add_seen_values(const uint8_t* s_v, f32x16_t s, f32x16_t (&o)[VT], int see, int g, int n) {
#pragma unroll 1
  for (int x = 0; x < 16; ++x) {
    asm volatile("" : "+v"(g));                    // no code: keeps this rare path's addresses out of the loops around it
    const float mine = s[0];
#pragma unroll
    for (int r = 0; r < 15; ++r) s[r] = s[r + 1];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const float p = __shfl(mine, n + 32 * w);
      const int t = 8 * (x >> 2) + 4 * w + (x & 3);
      if (t > see) continue;
#pragma unroll
      for (int m = 0; m < VT; ++m)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {          // elements 32 m + 2 r + 4 g ..
          const int d = 4 * m + (r >> 2);
          const uint2 v = *reinterpret_cast<const uint2*>(s_v + (t * VC + value_swap<VC>(t, d)) * 16 + 8 * g);
          o[m][r] += p * bf16_lo(v.x);
          o[m][r + 1] += p * bf16_hi(v.x);
          o[m][r + 2] += p * bf16_lo(v.y);
          o[m][r + 3] += p * bf16_hi(v.y);
        }
    }
  }
}

// A workgroup of W waves takes 32 W queries of one head (32 per wave) through
// the keys they see, 64 at a step, 32 at a time:
//   scores  S^T = K Q^T on v_mfma_f32_32x32x16_bf16: a lane holds scores of one
//           query, so its softmax needs one exchange (with the lane 32 on);
//   weights online softmax in base 2, rounded once to bf16 (half a step, 2^-8
//           of a weight; 2.1e-3 relative to the 64-bit result for the call
//           below, 1.6e-3 with weights of 32 bits); sums are kept of the
//           unrounded weights;
//   values  O^T += V^T P^T: the scores' lane layout is the operand layout of P
//           up to the order of the 16 keys of a product, which the value operand
//           follows (two transposing reads of 4 keys).
// The scores of the next 32 keys are computed beside the weights of the current
// ones, so that the matrix and the vector units work at once; two steps of keys
// and values are on their way into a ring of three LDS buffers meanwhile.
// Rows past the sequence repeat its last one: no query sees them.
// The keys a query sees are the first ones of its sequence, as many as its place
// from the end allows or, where the keys come with positions, as lie at its
// position or before (8,192 queries and keys of 32 heads: 699 us by place, 710
// by position).
// 8,192 queries and keys, 32 heads of 128 + 64 and values of 128 take 688-743 us
// from card to card (687 GFLOP, 925-999 TFLOP/s); this loop's products alone take
// 516.  Of what is between, most is the operands' reads from LDS, 1.45
// instructions a product since each serves 32 queries of one wave: with operands
// made in registers 583 us in place of 700.  Without exponentials it is 670.
template <int N, int P, int V, int W>
__global__ __launch_bounds__(64 * W, 2) void latent_prompt_kernel(LatentPromptArgs a, int q_tiles) {
  constexpr int T = 64 * W, kRows = 32 * W;
  constexpr int NC = N / 8, PC = P / 8, VC = V / 8, VT = V / 32;   // 16-byte chunks of a row; output tiles
  constexpr int NI = N / 16, KI = (N + P) / 16;                    // score steps
  constexpr int kKn = kKeys * NC * 16, kKr = kKeys * PC * 16, kV = kKeys * VC * 16, kStep = kKn + kKr + kV;
  __shared__ __align__(1024) uint8_t s_kv[3][kStep];
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int g = lane >> 5, n = lane & 31;
  // Workgroups go to the 8 XCDs in turn.  With a multiple of 8 heads each XCD gets neighbouring heads.
  int head = (int)blockIdx.x % a.heads;
  int rest = (int)blockIdx.x / a.heads;
  if (a.heads % 8 == 0) head = head % 8 * (a.heads / 8) + head / 8;
  auto q_at = [&](int b) { return min(max(a.cu_q[b], 0), a.total_q); };
  auto k_at = [&](int b) { return min(max(a.cu_k[b], 0), a.total_k); };
  // The longest tiles first: the last of every sequence before the ones before
  // it, or by the keys they see where there are few enough to rank in a wave's
  // lanes (with more the rest evens out; 8 chunks of 266-1,024 queries with up
  // to 2,306 keys before them, 20 heads: 208 us by the first, 168 so).  With
  // positions too these are the keys by the place from the end, the fewest they
  // can be: the order only has to be good.
  const int items = q_tiles * a.batch;
  if (items <= 64) {
    const int b = lane % a.batch, tile = q_tiles - 1 - lane / a.batch;
    int keys = -1;                                 // of lane's item; an empty tile is the last
    if (lane < items) {
      const int nq = min(q_at(b + 1) - q_at(b), a.max_q), last = min(tile * kRows + kRows, nq) - 1;
      if (tile * kRows < nq) keys = max(0, k_at(b + 1) - k_at(b) - (q_at(b + 1) - q_at(b)) + last + 1);
    }
    int before = 0;
    for (int y = 0; y < items; ++y) {
      const int other = __builtin_amdgcn_readlane(keys, y);
      before += other > keys || (other == keys && y < lane);
    }
    rest = __builtin_amdgcn_readfirstlane((int)__ffsll((unsigned long long)__ballot(lane < items && before == rest)) - 1);
  }
  const int b = rest % a.batch, tile = q_tiles - 1 - rest / a.batch;
  const int q0 = q_at(b), q1 = q_at(b + 1), k0 = k_at(b), k1 = k_at(b + 1);
  const int nq = q1 - q0, nk = max(k1 - k0, 0), nq_in = min(nq, a.max_q);
  if (tile * kRows >= nq_in) return;
  const int row0 = tile * kRows + wave * 32, row = row0 + n;   // this lane's query
  const int past = nk - nq;
  // Keys that the tile's last query, the wave's first and its last see: by their place from the end, or those at their
  // position and before, found by 16 lanes each.
  const int tile_last = min(tile * kRows + kRows, nq_in) - 1, wave_last = min(row0 + 31, nq_in - 1);
  auto by_place = [&](int i) { return min(max(i + past + 1, 0), nk); };
  auto position = [&](int i) { return (long long)a.q_first[b] + i; };
  int n_see = by_place(tile_last), first_sees = by_place(row0), last_sees = by_place(wave_last);
  if (a.pos) {
    const long long at = position(lane < 16 ? tile_last : lane < 32 ? row0 : wave_last);
    const int seen = at >= INT32_MAX ? nk : entries_below(a.pos + k0, 0, nk, (int)at + 1);
    n_see = __builtin_amdgcn_readlane(seen, 0);
    first_sees = __builtin_amdgcn_readlane(seen, 16);
    last_sees = __builtin_amdgcn_readlane(seen, 32);
  }
  if (row0 >= nq_in) first_sees = last_sees = 0;
  const int steps = (n_see + kKeys - 1) / kKeys;

  // Scores are scaled by |scale|; its sign goes to the queries, so that a score's maximum is a scaled one's.
  uint4 qf[KI];
  const bool in = row < nq_in;
  const uint32_t flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;
  const float scale = fabsf(a.scale_log2);
  const uint16_t* qrow = a.q + ((size_t)(q0 + (in ? row : 0)) * a.heads + head) * (N + P) + 8 * g;
#pragma unroll
  for (int i = 0; i < KI; ++i) {
    qf[i] = in ? *reinterpret_cast<const uint4*>(qrow + 16 * i) : make_uint4(0u, 0u, 0u, 0u);
    qf[i] = make_uint4(qf[i].x ^ flip, qf[i].y ^ flip, qf[i].z ^ flip, qf[i].w ^ flip);
  }
  const size_t kv_row = (size_t)a.heads * (N + V);
  const uint16_t* kv = a.kv + ((size_t)k0 * a.heads + head) * (N + V);
  const uint16_t* rk = a.r + (size_t)k0 * P;
  // Rows of C chunks, `stride` elements apart, of keys 64 j .. into LDS, a wave taking every W-th KiB; the offset from
  // the step's first row is the lane's own for the whole call.
  auto fetch_rows = [&](auto chunks, auto swap, const uint16_t* src, uint32_t stride, int j, uint8_t* dst) {
    constexpr int C = decltype(chunks)::value;
    src += (size_t)j * kKeys * stride;
    const int most = nk - 1 - j * kKeys;
#pragma unroll
    for (int k = 0; k < (C + W - 1) / W; ++k) {
      const int x = wave + k * W, c = x * 64 + lane, t = c / C;
      if ((k + 1) * W > C && x >= C) continue;
      const uint32_t at = (uint32_t)(most < kKeys - 1 ? min(t, most) : t) * stride + 8 * swap(t, c % C);
      load_to_lds<false>(src + at, dst + x * 1024);
    }
  };
  auto fetch = [&](int j) {
    if (j >= steps) return;
    uint8_t* dst = s_kv[j % 3];
    fetch_rows(std::integral_constant<int, NC>{}, [](int t, int d) { return key_swap<NC>(t, d); }, kv, (uint32_t)kv_row, j,
               dst);
    fetch_rows(std::integral_constant<int, PC>{}, [](int t, int d) { return key_swap<PC>(t, d); }, rk, P, j, dst + kKn);
    fetch_rows(std::integral_constant<int, VC>{}, [](int t, int d) { return value_swap<VC>(t, d); }, kv + N,
               (uint32_t)kv_row, j, dst + kKn + kKr);
  };
  f32x16_t o[VT];
#pragma unroll
  for (int m = 0; m < VT; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[m][r] = 0.0f;
  float mx = -INFINITY, sum = 0.0f;                // the reference (of scaled scores), the weights' sum
  // Operand addresses.  The swaps XOR a chunk's index with bits of its row, so chunk d + x of a lane's row, x and d
  // having no bit in common, is at (the address of chunk d) ^ 16 x: one base each for the per-head keys, the rotary
  // keys and the values.
  const int l16 = lane & 15, v_row = 4 * g + (l16 >> 2);       // value operand: 4 keys x 16 elements per 16 lanes
  const uint32_t kn_at = (uint32_t)(n * NC + key_swap<NC>(n, g)) * 16;
  const uint32_t kr_at = (uint32_t)(kKn + (n * PC + key_swap<PC>(n, g)) * 16);
  const uint32_t v_at = (uint32_t)(kKn + kKr + (v_row * VC + value_swap<VC>(v_row, 2 * ((lane >> 4) & 1) + ((l16 & 3) >> 1))) * 16 +
                                   8 * (l16 & 1));
  auto scores = [&](uint32_t kvs, int u) {         // of keys 32 u .. of the step at LDS address kvs
    f32x16_t s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.0f;
    const uint32_t kn = fresh(kvs + kn_at), kr = fresh(kvs + kr_at);
#pragma unroll
    for (int i = 0; i < KI; ++i) {
      const uint32_t at = i < NI ? (kn ^ (32 * i)) + u * 32 * NC * 16 : (kr ^ (32 * (i - NI))) + u * 32 * PC * 16;
      s = mfma(read_lds16(at), qf[i], s);
    }
    return s;
  };
  auto highest = [&](const f32x16_t& s) {          // of the lane's query, scaled
    float top = fmaxf(s[0], s[1]);
#pragma unroll
    for (int r = 2; r < 16; ++r) top = fmaxf(top, s[r]);
    top = fmaxf(top, __shfl_xor(top, 32));
    return top == -INFINITY ? top : top * scale;
  };
  auto exceeds = [&](float top) { return __ballot(top > mx + kHeadroom) != 0ull; };
  auto refer = [&](float top) {                    // the reference follows a maximum that exceeds it
    const float ref = top > mx + kHeadroom ? top : mx;
    const float alpha = ref == mx ? 1.0f : __builtin_amdgcn_exp2f(mx - ref);
    sum *= alpha;
#pragma unroll
    for (int m = 0; m < VT; ++m) o[m] *= alpha;
    mx = ref;
  };
  auto weigh = [&](f32x16_t& s) {
    const float base = mx == -INFINITY ? 0.0f : mx;
    float part = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], scale, -base));
      if (r & 1) part += s[r];
      else sum += s[r];
    }
    sum += part;
  };
  auto packed = [](const f32x16_t& s, int h) {     // weights of 16 keys as an operand
    return make_uint4(pack_bf16x2(s[8 * h], s[8 * h + 1]), pack_bf16x2(s[8 * h + 2], s[8 * h + 3]),
                      pack_bf16x2(s[8 * h + 4], s[8 * h + 5]), pack_bf16x2(s[8 * h + 6], s[8 * h + 7]));
  };
  auto add_values = [&](uint32_t kvs, int u, const f32x16_t& s) {
    const uint32_t vs = fresh(kvs + v_at + u * 32 * VC * 16);
    const uint4 p[2] = {packed(s, 0), packed(s, 1)};
    uint4 v[4];
    constexpr int kRow = VC * 16, k1 = 16 * kRow;
    if constexpr (VT == 4) {
      read_transposed<0, 0, 0, 0, 8 * kRow>(vs, vs ^ 64, vs ^ 128, vs ^ 192, v);
#pragma unroll
      for (int m = 0; m < 4; ++m) o[m] = mfma(v[m], p[0], o[m]);
      read_transposed<k1, k1, k1, k1, 8 * kRow>(vs, vs ^ 64, vs ^ 128, vs ^ 192, v);
#pragma unroll
      for (int m = 0; m < 4; ++m) o[m] = mfma(v[m], p[1], o[m]);
    } else {
      read_transposed<0, 0, k1, k1, 8 * kRow>(vs, vs ^ 64, vs, vs ^ 64, v);
#pragma unroll
      for (int x = 0; x < 4; ++x) o[x & 1] = mfma(v[x], p[x >> 1], o[x & 1]);
    }
  };

  fetch(0);
  fetch(1);
  wait_loads();
  __syncthreads();
  // Units of 32 keys.  After a step's first unit the workgroup meets: the next
  // step's copies have arrived, and the buffer of the step before is free for
  // those of the step after next.
  const int units = 2 * steps;
  auto step_of = [&](int i) { return lds_address(s_kv[(i >> 1) % 3]); };
  auto meet = [&](int i) {
    if (i & 1) return;
    wait_loads();
    __syncthreads();
    fetch(i / 2 + 2);
  };
  // The units that all queries of the wave see whole: unit i's scores s become
  // weights beside the scores of unit i + 1.  The loop is left to move the
  // reference: in it the sums are only added to.
  const int whole = min(units, first_sees / 32);
  float base = 0.0f, odd_sum = 0.0f, top = -INFINITY;
  auto turn = [&](int i, f32x16_t& s, f32x16_t& next) {
    const uint32_t nkvs = step_of(i + 1), nu = (i + 1) & 1;
    const uint32_t kn = fresh(nkvs + kn_at + nu * 32 * NC * 16), kr = fresh(nkvs + kr_at + nu * 32 * PC * 16);
    const uint32_t vs = fresh(step_of(i) + v_at + (i & 1) * 32 * VC * 16);
    auto operand = [&](int k) { return read_lds16(k < NI ? kn ^ (32 * k) : kr ^ (32 * (k - NI))); };
    constexpr int kRow = VC * 16, k1 = 16 * kRow;
#pragma unroll
    for (int r = 0; r < 16; ++r) next[r] = 0.0f;
    uint4 kf[kAhead], v[4], p = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) kf[k] = operand(k);
    // Pinned order: a score product, the read of one to come, a part of the weights; from the middle on also a
    // product of values with the first 16 weights.
    constexpr int kWeigh = KI - 2, kFirst = kWeigh / 2;
#pragma unroll
    for (int k = 0; k < KI; ++k) {
      next = mfma(kf[k % kAhead], qf[k], next);
      if (k + kAhead < KI) kf[k % kAhead] = operand(k + kAhead);
#pragma unroll
      for (int r = 16 * k / kWeigh; r < min(16, 16 * (k + 1) / kWeigh); ++r) {
        s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], scale, -base));
        if (r & 1) odd_sum += s[r];
        else sum += s[r];
      }
      if (VT == 4 && k >= kFirst && k < kFirst + 4) {
        if (k == kFirst) {
          p = packed(s, 0);
          read_transposed<0, 0, 0, 0, 8 * kRow>(vs, vs ^ 64, vs ^ 128, vs ^ 192, v);
        }
        o[k - kFirst] = mfma(v[k - kFirst], p, o[k - kFirst]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (VT == 4) {
      p = packed(s, 1);
      read_transposed<k1, k1, k1, k1, 8 * kRow>(vs, vs ^ 64, vs ^ 128, vs ^ 192, v);
#pragma unroll
      for (int m = 0; m < 4; ++m) o[m] = mfma(v[m], p, o[m]);
    } else {
      read_transposed<0, 0, k1, k1, 8 * kRow>(vs, vs ^ 64, vs, vs ^ 64, v);
#pragma unroll
      for (int x = 0; x < 4; ++x) o[x & 1] = mfma(v[x], packed(s, x >> 1), o[x & 1]);
    }
    top = highest(next);
    meet(i);
    return exceeds(top);
  };
  f32x16_t s;
  int i = 0;
  if (whole > 0) {
    s = scores(step_of(0), 0);
    refer(highest(s));
  }
  while (i < whole) {
    base = mx == -INFINITY ? 0.0f : mx;
    f32x16_t t;
    bool out = false;
    while (i + 2 < whole) {                        // two turns, so that neither's scores are copied
      out = turn(i, s, t);
      ++i;
      if (out) {
        s = t;
        break;
      }
      out = turn(i, t, s);
      ++i;
      if (out) break;
    }
    if (!out && i + 1 < whole) {
      out = turn(i, s, t);
      ++i;
      s = t;
    }
    sum += odd_sum;
    odd_sum = 0.0f;
    if (out) {
      refer(top);
    } else {                                       // the last of them
      weigh(s);
      add_values(step_of(i), i & 1, s);
      meet(i);
      ++i;
    }
  }
  // Units at the edge: some query of the wave does not see all their keys.
  int sees = row + past + 1;                       // keys that this query sees
  if (a.pos) {                                     // between the wave's first and last query's
    sees = first_sees;
    for (int end = last_sees; sees < end;) {
      const int mid = (sees + end) >> 1;
      if (a.pos[k0 + mid] <= position(row)) sees = mid + 1;
      else end = mid;
    }
  }
  for (; i < units; ++i) {
    if (last_sees > 32 * i) {                      // some query of the wave sees a key
      const uint8_t* s_v = s_kv[(i >> 1) % 3] + kKn + kKr + (i & 1) * 32 * VC * 16;
      const int see = sees - 1 - 32 * i;           // this query sees the unit's keys 0 .. see
      auto hidden = [&](int r) { return 8 * (r >> 2) + 4 * g + (r & 3) > see; };
      s = scores(step_of(i), i & 1);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = hidden(r) ? -INFINITY : s[r];
      refer(highest(s));
      base = mx == -INFINITY ? 0.0f : mx;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float w = __builtin_amdgcn_exp2f(fmaf(s[r], scale, -base));
        s[r] = hidden(r) ? 0.0f : w;
        sum += s[r];
      }
      bool wild = false;                           // some value is infinite or NaN
      for (int c = lane; c < 32 * VC; c += 64) wild |= abs_max_bits8(reinterpret_cast<const uint4*>(s_v)[c]) >= 0x7F80u;
      if (__ballot(wild)) add_seen_values<VT, VC>(s_v, s, o, see, g, n);
      else add_values(step_of(i), i & 1, s);
    }
    meet(i);
  }
  if (!in) return;
  sum += __shfl_xor(sum, 32);
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  const size_t at = (size_t)(q0 + row) * a.heads + head;
#pragma unroll
  for (int m = 0; m < VT; ++m)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *reinterpret_cast<uint2*>(a.out + at * V + 32 * m + 2 * r + 4 * g) =
          make_uint2(pack_bf16x2(o[m][r] * inv, o[m][r + 1] * inv), pack_bf16x2(o[m][r + 2] * inv, o[m][r + 3] * inv));
  if (a.lse && g == 0) a.lse[at] = sum == 0.0f ? -INFINITY : (mx + __builtin_amdgcn_logf(sum)) * kLn2;
}

// Waves of a workgroup: eight share every key and value through LDS; two where
// no sequence has more queries than they take.
int prompt_waves(const LatentPromptArgs& a) { return a.max_q <= 64 ? 2 : 8; }

template <int N, int P, int V>
void launch_waves(const LatentPromptArgs& a, hipStream_t s) {
  const unsigned blocks = (unsigned)latent_prompt_blocks(a);
  if (prompt_waves(a) == 2) latent_prompt_kernel<N, P, V, 2><<<dim3(blocks), dim3(128), 0, s>>>(a, (a.max_q + 63) / 64);
  else latent_prompt_kernel<N, P, V, 8><<<dim3(blocks), dim3(512), 0, s>>>(a, (a.max_q + 255) / 256);
}

template <int N, int P>
void launch_dims(const LatentPromptArgs& a, hipStream_t s) {
  if (a.v == 64) launch_waves<N, P, 64>(a, s);
  else launch_waves<N, P, 128>(a, s);
}

}  // namespace

int64_t latent_prompt_blocks(const LatentPromptArgs& a) {
  const int rows = 32 * prompt_waves(a);
  return ((int64_t)a.max_q + rows - 1) / rows * a.batch * a.heads;
}

hipError_t launch_latent_prompt(const LatentPromptArgs& a, hipStream_t s) {
  if (a.nope == 64) {
    if (a.rope == 32) launch_dims<64, 32>(a, s);
    else launch_dims<64, 64>(a, s);
  } else {
    if (a.rope == 32) launch_dims<128, 32>(a, s);
    else launch_dims<128, 64>(a, s);
  }
  return hipGetLastError();
}

}  // namespace pask
