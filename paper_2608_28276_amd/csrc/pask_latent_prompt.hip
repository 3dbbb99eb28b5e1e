// gfx950 kernel of the expanded latent attention: causal attention of packed,
// ragged prompts, with keys (per-head part, shared rotary key) and values per
// head.
#include <hip/hip_runtime.h>

#include <math.h>

#include <algorithm>
#include <type_traits>

#include "pask_device.h"
#include "pask_latent_internal.h"

namespace pask {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kKeys = 64;                          // keys of a step
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

// Rows of C 16-byte chunks in LDS, row t's chunk d at t * C + swap(t, d): the
// operand reads, 8 neighbouring rows' chunk d at once, fall on all banks
// (256 / (16 C) rows share the 64 banks).
template <int C>
__device__ __forceinline__ int key_swap(int t, int d) { return d ^ ((C >= 16 ? t : t / (16 / C)) & (C - 1)); }
// The same for values, which the transposing reads take in pairs of chunks of 4 rows.
template <int C>
__device__ __forceinline__ int value_swap(int t, int d) { return d ^ ((t & (C / 2 - 1)) << 1); }

// O += P V key by key, for a step in which a value that some query does not
// see is infinite or NaN (a weight of 0 times it is not 0): only keys up to
// `see` are added.  Lane (g, n) holds the weights of query n for half of the
// keys, lane (1 - g, n) the others'; the weights move down one register a turn.
template <int VT, int VC>
__device__ __forceinline__ void add_seen_values(const uint8_t* s_v, f32x16_t (&s)[2], f32x16_t (&o)[VT], int see, int g,
                                             int n) {
#pragma unroll 1
  for (int x = 0; x < 32; ++x) {
    asm volatile("" : "+v"(g));                    // no code: keeps this rare path's addresses out of the loops around it
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
          const uint2 v = *reinterpret_cast<const uint2*>(s_v + (t * VC + value_swap<VC>(t, d)) * 16 + 8 * g);
          o[m][r] += p * bf16_lo(v.x);
          o[m][r + 1] += p * bf16_hi(v.x);
          o[m][r + 2] += p * bf16_lo(v.y);
          o[m][r + 3] += p * bf16_hi(v.y);
        }
    }
  }
}

// 16 bytes per lane from memory straight into LDS: lane l's to lds + 16 l (lds is
// the same for the wave).  The caller waits (wait_loads) and synchronises.
__device__ __forceinline__ void load_to_lds(const uint16_t* src, uint8_t* lds) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)src,
                                   (__attribute__((address_space(3))) uint32_t*)lds, 16, 0, 0);
}
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }   // vmcnt(0)

// A workgroup of W waves takes 32 W queries of one head (32 per wave) through
// the keys they see, 64 at a time:
//   scores  S^T = K Q^T on v_mfma_f32_32x32x16_bf16: a lane holds scores of one
//           query, so its softmax needs one exchange (with the lane 32 on);
//   weights online softmax in base 2, rounded to bf16 (2^-8 of a weight at
//           most, as the values' own); the reference maximum moves only when
//           exceeded by more than 8, sums are kept of the unrounded weights;
//   values  O^T += V^T P^T: the scores' lane layout is the operand layout of P
//           up to the order of the 16 keys of a step, which the value operand
//           follows (two transposing reads of 4 keys).
// The next step's keys and values are on their way into the other LDS buffers
// meanwhile.  Rows past the sequence repeat its last one: no query sees them.
template <int N, int P, int V, int W>
__global__ __launch_bounds__(64 * W, 2) void latent_prompt_kernel(LatentPromptArgs a, int q_tiles) {
  constexpr int T = 64 * W, kRows = 32 * W;
  constexpr int NC = N / 8, PC = P / 8, VC = V / 8, VT = V / 32;   // 16-byte chunks of a row; output tiles
  constexpr int NI = N / 16, KI = (N + P) / 16;                    // score steps
  constexpr int kKn = kKeys * NC * 16, kKr = kKeys * PC * 16, kV = kKeys * VC * 16;
  __shared__ __align__(16) uint8_t s_kv[2][kKn + kKr + kV];
  __shared__ int s_wild;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int g = lane >> 5, n = lane & 31;
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
  auto fetch = [&](int j, uint8_t* dst) {          // keys 64 j .. of the sequence
#pragma unroll
    for (int k = 0; k < (NC + W - 1) / W; ++k) {
      const int x = wave + k * W, c = x * 64 + lane, t = c / NC;
      if (x < NC)
        load_to_lds(kv + min(j * kKeys + t, nk - 1) * kv_row + 8 * key_swap<NC>(t, c % NC), dst + x * 1024);
    }
#pragma unroll
    for (int k = 0; k < (PC + W - 1) / W; ++k) {
      const int x = wave + k * W, c = x * 64 + lane, t = c / PC;
      if (x < PC)
        load_to_lds(rk + (size_t)min(j * kKeys + t, nk - 1) * P + 8 * key_swap<PC>(t, c % PC), dst + kKn + x * 1024);
    }
#pragma unroll
    for (int k = 0; k < (VC + W - 1) / W; ++k) {
      const int x = wave + k * W, c = x * 64 + lane, t = c / VC;
      if (x < VC)
        load_to_lds(kv + min(j * kKeys + t, nk - 1) * kv_row + N + 8 * value_swap<VC>(t, c % VC),
                    dst + kKn + kKr + x * 1024);
    }
  };
  f32x16_t o[VT];
#pragma unroll
  for (int m = 0; m < VT; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[m][r] = 0.0f;
  float mx = -INFINITY, sum = 0.0f;                // the reference (of scaled scores), the weights' sum
  const int l16 = lane & 15, half = (lane >> 4) & 1;           // value operand: 4 keys x 16 elements per 16 lanes
  if (steps > 0) fetch(0, s_kv[0]);
  wait_loads();
  __syncthreads();
  // One step of the wave.  kEdge: some query of the wave does not see all its keys.
  auto attend = [&](auto edge_tag, int j, const uint8_t* s_k, bool wild) {
    constexpr bool kEdge = decltype(edge_tag)::value;
    const uint8_t* s_v = s_k + kKn + kKr;
    const int see = row + past - j * kKeys;        // this query sees the step's keys 0 .. see
    auto key_at = [&](int i, int u) {              // operand i of keys 32 u ..
      const int t = 32 * u + n;
      return *reinterpret_cast<const uint4*>(i < NI ? s_k + (t * NC + key_swap<NC>(t, 2 * i + g)) * 16
                                                    : s_k + kKn + (t * PC + key_swap<PC>(t, 2 * (i - NI) + g)) * 16);
    };
    f32x16_t s[2];
#pragma unroll
    for (int r = 0; r < 16; ++r) s[0][r] = s[1][r] = 0.0f;
    uint4 kf[2][2] = {{key_at(0, 0), key_at(0, 1)}, {key_at(1, 0), key_at(1, 1)}};
#pragma unroll
    for (int i = 0; i < KI; ++i) {
      const uint4 c0 = kf[i & 1][0], c1 = kf[i & 1][1];
      s[0] = mfma(c0, qf[i], s[0]);
      s[1] = mfma(c1, qf[i], s[1]);
      if (i + 2 < KI) {
        kf[i & 1][0] = key_at(i + 2, 0);
        kf[i & 1][1] = key_at(i + 2, 1);
      }
    }
    if constexpr (kEdge) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[u][r] = 32 * u + 8 * (r >> 2) + 4 * g + (r & 3) <= see ? s[u][r] : -INFINITY;
    }
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[u][r]);
    top = fmaxf(top, __shfl_xor(top, 32));
    top = top == -INFINITY ? top : top * scale;
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
        float w = __builtin_amdgcn_exp2f(fmaf(s[u][r], scale, -base));
        if constexpr (kEdge) w = 32 * u + 8 * (r >> 2) + 4 * g + (r & 3) <= see ? w : 0.0f;
        s[u][r] = w;
        sum += w;
      }
    if constexpr (kEdge) {
      if (wild) {
        add_seen_values<VT, VC>(s_v, s, o, see, g, n);
        return;
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {                // 16 keys
        const uint4 p =
            make_uint4(pack_bf16x2(s[u][8 * h], s[u][8 * h + 1]), pack_bf16x2(s[u][8 * h + 2], s[u][8 * h + 3]),
                       pack_bf16x2(s[u][8 * h + 4], s[u][8 * h + 5]), pack_bf16x2(s[u][8 * h + 6], s[u][8 * h + 7]));
#pragma unroll
        for (int m = 0; m < VT; ++m) {
          uint2 w[2];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int t = 32 * u + 16 * h + 8 * x + 4 * g + (l16 >> 2);
            const int d = 4 * m + 2 * half + ((l16 & 3) >> 1);
            w[x] = read_transposed(s_v + (t * VC + value_swap<VC>(t, d)) * 16 + 8 * (l16 & 1));
          }
          o[m] = mfma(make_uint4(w[0].x, w[0].y, w[1].x, w[1].y), p, o[m]);
        }
      }
  };
  // Steps that every query of the workgroup sees whole, then those at the edge.
  const int whole = min(steps, max(0, (tile * kRows + past + 1) / kKeys));
  for (int j = 0; j < whole; ++j) {
    if (j + 1 < steps) fetch(j + 1, s_kv[(j + 1) & 1]);
    attend(std::false_type{}, j, s_kv[j & 1], false);
    wait_loads();
    __syncthreads();
  }
  for (int j = whole; j < steps; ++j) {
    const uint8_t* s_k = s_kv[j & 1];
    if (j + 1 < steps) fetch(j + 1, s_kv[(j + 1) & 1]);
    // Values that are infinite or NaN, where some query may not see them.
    if (threadIdx.x == 0) s_wild = 0;
    __syncthreads();
    bool wild = false;
    for (int c = (int)threadIdx.x; c < kKeys * VC; c += T)
      wild |= abs_max_bits8(reinterpret_cast<const uint4*>(s_k + kKn + kKr)[c]) >= 0x7F80u;
    if (wild) s_wild = 1;
    __syncthreads();
    if (row0 + 31 + past >= j * kKeys) attend(std::true_type{}, j, s_k, s_wild != 0);   // some query of the wave sees a key
    wait_loads();
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
