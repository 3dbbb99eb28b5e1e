// gfx950 kernel of the expanded latent attention: causal attention of packed,
// ragged prompts, with keys (per-head part, shared rotary key) and values per
// head.
#include <hip/hip_runtime.h>

#include <math.h>

#include <algorithm>

#include "pask_device.h"
#include "pask_latent_internal.h"

namespace pask {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256;
constexpr int kRows = 128, kKeys = 64;             // queries of a workgroup, keys of a step
constexpr float kLn2 = 0.6931471805599453f;

// D[32x32] += A[32x16] B[16x32]: lane l holds A[l % 32][8 (l / 32) ..], B[8 (l / 32) ..][l % 32], and
// D[8 (r / 4) + 4 (l / 32) + r % 4][l % 32], r < 16.
__device__ __forceinline__ f32x16_t mfma(uint4 a, uint4 b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0,
                                                 0, 0);
}
// Element i of four rows for lane i of each 16 (lanes 4r .. 4r + 3 address row r's 8-byte quarters).
__device__ __forceinline__ uint2 read_transposed(const uint8_t* lds) {
  typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;
  return __builtin_bit_cast(
      uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(__attribute__((address_space(3))) uint8_t*)lds));
}

// O += P V key by key, for a step in which a value that some query does not
// see is infinite or NaN (a weight of 0 times it is not 0): only keys up to
// `see` are added.  Lane (g, n) holds the weights of query n for half of the
// keys, lane (1 - g, n) the others'; the weights move down one register a turn.
template <int VT, int VC>
__device__ __forceinline__ void add_seen_values(const uint8_t* s_v, f32x16_t (&s)[2], f32x16_t (&o)[VT], int see, int g,
                                             int n) {
#pragma unroll 1
  for (int x = 0; x < 32; ++x) {
    const float mine = s[0][0];
#pragma unroll
    for (int r = 0; r < 31; ++r) s[r >> 4][r & 15] = s[(r + 1) >> 4][(r + 1) & 15];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const float p = __shfl(mine, n + 32 * w);
      const int t = 32 * (x >> 4) + 8 * ((x & 15) >> 2) + 4 * w + (x & 3);
      if (t > see) continue;
#pragma unroll
      for (int m = 0; m < VT; ++m)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {          // elements 32 m + 2 r + 4 g ..
          const int d = 4 * m + (r >> 2);
          const uint2 v = *reinterpret_cast<const uint2*>(s_v + (t * VC + (d ^ ((t & (VC / 2 - 1)) << 1))) * 16 + 8 * g);
          o[m][r] += p * bf16_lo(v.x);
          o[m][r + 1] += p * bf16_hi(v.x);
          o[m][r + 2] += p * bf16_lo(v.y);
          o[m][r + 3] += p * bf16_hi(v.y);
        }
    }
  }
}

// A workgroup takes 128 queries of one head (32 per wave) through the keys
// they see, 64 at a time:
//   scores  S^T = K Q^T on v_mfma_f32_32x32x16_bf16: a lane holds scores of one
//           query, so its softmax needs one exchange (with the lane 32 on);
//   weights online softmax in base 2, rounded to bf16 (2^-8 of a weight at
//           most, as the values' own); the reference maximum moves only when
//           exceeded by more than 8, sums are kept of the unrounded weights;
//   values  O^T += V^T P^T: the scores' lane layout is the operand layout of P
//           up to the order of the 16 keys of a step, which the value operand
//           follows (two transposing reads of 4 keys).
// LDS: K chunks of 8 elements, chunk d of key t at d * 64 + (t ^ d mod 16) (both
// the row-wise writes and the operand reads fall on all banks); V rows with
// their 32-byte pairs swapped by the key for the transposing reads.
template <int N, int P, int V>
__global__ __launch_bounds__(kThreads, 2) void latent_prompt_kernel(LatentPromptArgs a, int q_tiles) {
  constexpr int KD = (N + P) / 8, KI = (N + P) / 16;           // 16-byte chunks of a key, score steps
  constexpr int NC = N / 8, PC = P / 8, VC = V / 8, VT = V / 32;
  constexpr int NK = kKeys * KD / kThreads, NV = kKeys * VC / kThreads;
  static_assert(kKeys * KD % kThreads == 0 && kKeys * VC % kThreads == 0, "whole pieces per thread");
  __shared__ __align__(16) uint8_t s_k[kKeys * KD * 16];
  __shared__ __align__(16) uint8_t s_v[kKeys * VC * 16];
  __shared__ int s_wild[2];                        // steps j and j + 1: some value is infinite or NaN
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 5, n = lane & 31;
  const int head = (int)blockIdx.x % a.heads, rest = (int)blockIdx.x / a.heads;
  const int b = rest % a.batch, tile = q_tiles - 1 - rest / a.batch;   // the longest first
  const int q0 = min(max(a.cu_q[b], 0), a.total_q), q1 = min(max(a.cu_q[b + 1], 0), a.total_q);
  const int k0 = min(max(a.cu_k[b], 0), a.total_k), k1 = min(max(a.cu_k[b + 1], 0), a.total_k);
  const int nq = q1 - q0, nk = max(k1 - k0, 0), nq_in = min(nq, a.max_q);
  if (tile * kRows >= nq_in) return;
  const int row0 = tile * kRows + wave * 32, row = row0 + n;   // this lane's query
  const int past = nk - nq;
  const int last = min(tile * kRows + kRows, nq_in) - 1;       // the tile's last query
  const int n_see = min(nk, last + past + 1);                  // keys it sees; may be <= 0
  const int steps = n_see > 0 ? (n_see + kKeys - 1) / kKeys : 0;

  uint4 qf[KI];
  const bool in = row < nq_in;
  const uint16_t* qrow = a.q + ((size_t)(q0 + (in ? row : 0)) * a.heads + head) * (N + P) + 8 * g;
#pragma unroll
  for (int i = 0; i < KI; ++i)
    qf[i] = in ? *reinterpret_cast<const uint4*>(qrow + 16 * i) : make_uint4(0u, 0u, 0u, 0u);

  uint4 kx[NK], vx[NV];
  const size_t kv_row = (size_t)a.heads * (N + V);
  const uint16_t* kv = a.kv + ((size_t)k0 * a.heads + head) * (N + V);
  const uint16_t* rk = a.r + (size_t)k0 * P;
  auto fetch = [&](int j) {                        // keys 64 j .. of the sequence; zeros past the last
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      const int c = tid + kThreads * k;
      const bool rope = c >= kKeys * NC;
      const int x = rope ? c - kKeys * NC : c, t = x / (rope ? PC : NC), d = x % (rope ? PC : NC);
      const int key = j * kKeys + t;
      kx[k] = key < nk ? *reinterpret_cast<const uint4*>(rope ? rk + (size_t)key * P + 8 * d : kv + key * kv_row + 8 * d)
                       : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = tid + kThreads * k, key = j * kKeys + c / VC;
      vx[k] = key < nk ? *reinterpret_cast<const uint4*>(kv + key * kv_row + N + 8 * (c % VC))
                       : make_uint4(0u, 0u, 0u, 0u);
    }
  };
  auto store = [&](int j, bool hides) {
    bool wild = false;
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      const int c = tid + kThreads * k;
      const bool rope = c >= kKeys * NC;
      const int x = rope ? c - kKeys * NC : c, t = x / (rope ? PC : NC), d = (rope ? NC : 0) + x % (rope ? PC : NC);
      *reinterpret_cast<uint4*>(s_k + (d * kKeys + (t ^ (d & 15))) * 16) = kx[k];
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = tid + kThreads * k, t = c / VC, d = c % VC;
      *reinterpret_cast<uint4*>(s_v + (t * VC + (d ^ ((t & (VC / 2 - 1)) << 1))) * 16) = vx[k];
      if (hides) wild |= abs_max_bits8(vx[k]) >= 0x7F80u;
    }
    if (wild) s_wild[j & 1] = 1;
  };
  f32x16_t o[VT];
#pragma unroll
  for (int m = 0; m < VT; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[m][r] = 0.0f;
  float mx = -INFINITY, sum = 0.0f;
  const int l16 = lane & 15, half = (lane >> 4) & 1;           // value operand: 4 keys x 16 elements per 16 lanes
  if (tid < 2) s_wild[tid] = 0;
  if (steps > 0) fetch(0);
  __syncthreads();
  for (int j = 0; j < steps; ++j) {
    store(j, tile * kRows + past < j * kKeys + kKeys - 1);     // a query of the tile does not see every key
    __syncthreads();
    const bool wild = s_wild[j & 1] != 0;
    if (tid == 0) s_wild[(j + 1) & 1] = 0;
    if (j + 1 < steps) fetch(j + 1);
    const int see = row + past - j * kKeys;        // this query sees the step's keys 0 .. see
    if (row0 + 31 + past >= j * kKeys) {           // wave-uniform: some query of the wave sees a key
      f32x16_t s[2];
#pragma unroll
      for (int r = 0; r < 16; ++r) s[0][r] = s[1][r] = 0.0f;
#pragma unroll
      for (int i = 0; i < KI; ++i) {
        const int d = 2 * i + g;
#pragma unroll
        for (int u = 0; u < 2; ++u)
          s[u] = mfma(*reinterpret_cast<const uint4*>(s_k + (d * kKeys + ((32 * u + n) ^ (d & 15))) * 16), qf[i], s[u]);
      }
      float top = -INFINITY;
      const bool edge = row0 + past - j * kKeys < kKeys - 1;   // some query of the wave does not see them all
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = 32 * u + 8 * (r >> 2) + 4 * g + (r & 3);
          float x = s[u][r] * a.scale_log2;
          if (edge) x = key <= see ? x : -INFINITY;
          s[u][r] = x;
          top = fmaxf(top, x);
        }
      top = fmaxf(top, __shfl_xor(top, 32));
      const float ref = top > mx + 8.0f ? top : mx;
      if (__ballot(ref != mx)) {
        const float alpha = ref == mx ? 1.0f : __builtin_amdgcn_exp2f(mx - ref);
        sum *= alpha;
#pragma unroll
        for (int m = 0; m < VT; ++m) o[m] *= alpha;
        mx = ref;
      }
      const float base = mx == -INFINITY ? 0.0f : mx;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[u][r] = __builtin_amdgcn_exp2f(s[u][r] - base);
          sum += s[u][r];
        }
      if (wild && edge) {
        add_seen_values<VT, VC>(s_v, s, o, see, g, n);
      } else
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {              // 16 keys
          const uint4 p = make_uint4(pack_bf16x2(s[u][8 * h], s[u][8 * h + 1]), pack_bf16x2(s[u][8 * h + 2], s[u][8 * h + 3]),
                                     pack_bf16x2(s[u][8 * h + 4], s[u][8 * h + 5]), pack_bf16x2(s[u][8 * h + 6], s[u][8 * h + 7]));
#pragma unroll
          for (int m = 0; m < VT; ++m) {
            uint2 w[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int t = 32 * u + 16 * h + 8 * x + 4 * g + (l16 >> 2);
              const int d = 4 * m + 2 * half + ((l16 & 3) >> 1);
              w[x] = read_transposed(s_v + (t * VC + (d ^ ((t & (VC / 2 - 1)) << 1))) * 16 + 8 * (l16 & 1));
            }
            o[m] = mfma(make_uint4(w[0].x, w[0].y, w[1].x, w[1].y), p, o[m]);
          }
        }
      }
    }
    __syncthreads();
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

template <int N, int P>
void launch_dims(const LatentPromptArgs& a, unsigned blocks, int q_tiles, hipStream_t s) {
  if (a.v == 64) latent_prompt_kernel<N, P, 64><<<dim3(blocks), dim3(kThreads), 0, s>>>(a, q_tiles);
  else latent_prompt_kernel<N, P, 128><<<dim3(blocks), dim3(kThreads), 0, s>>>(a, q_tiles);
}

}  // namespace

int64_t latent_prompt_blocks(const LatentPromptArgs& a) {
  return (int64_t)((a.max_q + kRows - 1) / kRows) * a.batch * a.heads;
}

hipError_t launch_latent_prompt(const LatentPromptArgs& a, hipStream_t s) {
  const int q_tiles = (a.max_q + kRows - 1) / kRows;
  const unsigned blocks = (unsigned)latent_prompt_blocks(a);
  if (a.nope == 64) {
    if (a.rope == 32) launch_dims<64, 32>(a, blocks, q_tiles, s);
    else launch_dims<64, 64>(a, blocks, q_tiles, s);
  } else {
    if (a.rope == 32) launch_dims<128, 32>(a, blocks, q_tiles, s);
    else launch_dims<128, 64>(a, blocks, q_tiles, s);
  }
  return hipGetLastError();
}

}  // namespace pask
