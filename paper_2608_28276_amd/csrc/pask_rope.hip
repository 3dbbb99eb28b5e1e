// gfx950 kernel of the rotary positions: rows of queries and keys rotated at
// their positions, once over the data.
#include <hip/hip_runtime.h>

#include <math.h>

#include <algorithm>

#include "pask_device.h"
#include "pask_prompt_internal.h"

namespace pask {
namespace {

constexpr int kThreads = 256, kMaxTokens = 8;

// Sine and cosine of a position's angle: the turns, reduced in 64 bits (their
// product is off by 2^-53 of itself: 2^-24 turns at position 2^31 and a
// frequency of 1 / 4 turn, 2^-38 at 131,072), then sinpi and cospi of at most
// half a turn in 32.
__device__ __forceinline__ float2 rotation(const pask_rope& r, int64_t pos, int i) {
  const double t = (double)pos * r.turns[i];
  const float x = 2.0f * (float)(t - rint(t));
  float s, c;
  sincospif(x, &s, &c);
  return make_float2(c * r.magnitude, s * r.magnitude);
}
__device__ __forceinline__ float2 turn(float x, float y, float2 cs) {
  return make_float2(fmaf(x, cs.x, -(y * cs.y)), fmaf(x, cs.y, y * cs.x));
}

// What a thread does at a time.  Chunks: 16-byte chunks, in the half layout a
// pair of them R / 2 elements apart; a copied one alone.  Otherwise a pair of
// elements, a copied one alone.
template <bool kChunks, bool kHalf>
struct Piece {
  uint4 x, y;
  size_t at;                                       // element of the row
  int pair;                                        // first pair
  bool rotated;
  __device__ __forceinline__ void place(const pask_rope& r, int piece, int rot_pieces) {
    rotated = piece < rot_pieces;
    constexpr int step = kChunks ? (kHalf ? 8 : 4) : 1;   // pairs of a piece
    pair = rotated ? piece * step : 0;
    if (rotated) {
      at = r.rot_first + (kHalf ? pair : 2 * pair);
    } else {
      const int e = (piece - rot_pieces) * (kChunks ? 8 : 1);
      at = e < r.rot_first ? e : e + r.rot_dim;
    }
  }
  __device__ __forceinline__ void load(const pask_rope& r, const uint16_t* row) {
    const uint16_t* p = row + at;
    if constexpr (kChunks) {
      x = *reinterpret_cast<const uint4*>(p);
      if (kHalf && rotated) y = *reinterpret_cast<const uint4*>(p + r.rot_dim / 2);
    } else {
      x.x = p[0];
      if (rotated) y.x = p[kHalf ? r.rot_dim / 2 : 1];
    }
  }
  __device__ __forceinline__ void turn_pairs(const float2* cs) {
    if (!rotated) return;
    cs += pair;
    if constexpr (!kChunks) {
      const float2 z = turn(bf16_lo(x.x), bf16_lo(y.x), cs[0]);
      x.x = f32_to_bf16_rne_dev(z.x);
      y.x = f32_to_bf16_rne_dev(z.y);
    } else if constexpr (kHalf) {
      auto two = [&](uint32_t& a, uint32_t& b, float2 c0, float2 c1) {
        const float2 lo = turn(bf16_lo(a), bf16_lo(b), c0), hi = turn(bf16_hi(a), bf16_hi(b), c1);
        a = pack_bf16x2(lo.x, hi.x);
        b = pack_bf16x2(lo.y, hi.y);
      };
      two(x.x, y.x, cs[0], cs[1]);
      two(x.y, y.y, cs[2], cs[3]);
      two(x.z, y.z, cs[4], cs[5]);
      two(x.w, y.w, cs[6], cs[7]);
    } else {
      auto one = [&](uint32_t& a, float2 c) {
        const float2 z = turn(bf16_lo(a), bf16_hi(a), c);
        a = pack_bf16x2(z.x, z.y);
      };
      one(x.x, cs[0]);
      one(x.y, cs[1]);
      one(x.z, cs[2]);
      one(x.w, cs[3]);
    }
  }
  __device__ __forceinline__ void store(const pask_rope& r, uint16_t* row) const {
    uint16_t* p = row + at;
    if constexpr (kChunks) {
      *reinterpret_cast<uint4*>(p) = x;
      if (kHalf && rotated) *reinterpret_cast<uint4*>(p + r.rot_dim / 2) = y;
    } else {
      p[0] = (uint16_t)x.x;
      if (rotated) p[kHalf ? r.rot_dim / 2 : 1] = (uint16_t)y.x;
    }
  }
};

// The rows of a workgroup's turn: row0 .. , their sines and cosines in LDS for
// all heads, and which of them are to be done.
__device__ __forceinline__ void prepare_rows(const RopeArgs& a, int64_t row0, float2* s_cs, int* s_live) {
  const int pairs = a.rope.rot_dim / 2;
  const int b0 = (int)(row0 / a.max_new), i0 = (int)(row0 - (int64_t)b0 * a.max_new);
  for (int x = (int)threadIdx.x; x < a.tokens * pairs; x += kThreads) {
    const int token = x / pairs, pair = x - token * pairs;
    int b = b0, i = i0 + token;
    while (i >= a.max_new) {
      i -= a.max_new;
      ++b;
    }
    const bool live = b < a.batch && (!a.n_new || i < a.n_new[b]);
    if (pair == 0) s_live[token] = live;
    if (!live) continue;
    const int64_t pos = a.pos ? a.pos[row0 + token] : (int64_t)a.first[b * a.first_stride] + i;
    s_cs[x] = rotation(a.rope, pos, pair);
  }
  __syncthreads();
}

// A workgroup takes `tokens` rows at a turn, their pieces in the order of memory.
template <bool kChunks, bool kHalf>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a) {
  extern __shared__ float2 s_cs[];                 // [tokens][pairs]
  __shared__ int s_live[kMaxTokens];
  const int pairs = a.rope.rot_dim / 2, per_row = (a.q_heads + a.k_heads) * a.pieces;
  const int64_t rows = (int64_t)a.batch * a.max_new;
  for (int64_t row0 = (int64_t)blockIdx.x * a.tokens; row0 < rows; row0 += (int64_t)gridDim.x * a.tokens) {
    auto find = [&](int x, Piece<kChunks, kHalf>& p, const uint16_t*& from, uint16_t*& to, int& token) {
      token = x / per_row;
      const int y = x - token * per_row, head = y / a.pieces;
      const bool is_q = head < a.q_heads;
      const RopeRows& t = is_q ? a.q : a.k;
      p.place(a.rope, y - head * a.pieces, a.rot_pieces);
      const int64_t at = (int64_t)(is_q ? head : head - a.q_heads) * a.rope.head_dim;
      from = t.src + (row0 + token) * t.in + at;
      to = t.dst + (row0 + token) * t.out + at;
      return p.rotated || (is_q ? a.q_copies : a.k_copies);
    };
    prepare_rows(a, row0, s_cs, s_live);
    for (int x = (int)(blockIdx.y * kThreads + threadIdx.x); x < a.tokens * per_row; x += (int)gridDim.y * kThreads) {
      Piece<kChunks, kHalf> p;
      const uint16_t* from;
      uint16_t* to;
      int token;
      if (!find(x, p, from, to, token) || !s_live[token]) continue;
      p.load(a.rope, from);
      p.turn_pairs(s_cs + token * pairs);
      p.store(a.rope, to);
    }
    __syncthreads();
  }
}

// The same where rows and heads are whole 16-byte chunks but the rotated part is
// not: heads go through LDS, where every element finds its pair's other one.  A
// thread has a chunk of a head, a workgroup 256 / (chunks of a head) heads.
template <bool kHalf>
__global__ __launch_bounds__(kThreads) void rope_staged_kernel(RopeArgs a) {
  extern __shared__ float2 s_cs[];                 // [tokens][pairs]
  __shared__ int s_live[kMaxTokens];
  __shared__ __align__(16) uint16_t s_x[8 * kThreads];
  const pask_rope& r = a.rope;
  const int pairs = r.rot_dim / 2, heads = a.q_heads + a.k_heads, chunks = r.head_dim / 8, each = kThreads / chunks;
  const int slot = (int)threadIdx.x / chunks, e0 = ((int)threadIdx.x - slot * chunks) * 8;   // first element of the chunk
  const int64_t rows = (int64_t)a.batch * a.max_new;
  for (int64_t row0 = (int64_t)blockIdx.x * a.tokens; row0 < rows; row0 += (int64_t)gridDim.x * a.tokens) {
    prepare_rows(a, row0, s_cs, s_live);
    const int all = a.tokens * heads;
    for (int x0 = (int)blockIdx.y * each; x0 < all; x0 += (int)gridDim.y * each) {
      const int x = x0 + slot, token = x / heads, head = x - token * heads;
      const bool is_q = head < a.q_heads, mine = slot < each && x < all && s_live[min(token, a.tokens - 1)];
      const RopeRows& t = is_q ? a.q : a.k;
      const int64_t at = (int64_t)(is_q ? head : head - a.q_heads) * r.head_dim + e0;
      union {
        uint4 v;
        uint16_t e[8];
      } c;
      if (mine) {
        c.v = *reinterpret_cast<const uint4*>(t.src + (row0 + token) * t.in + at);
        *reinterpret_cast<uint4*>(s_x + 8 * (int)threadIdx.x) = c.v;
      }
      __syncthreads();
      if (mine) {
        const uint16_t* row = s_x + 8 * slot * chunks;
        const float2* cs = s_cs + token * pairs;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int i = e0 + j - r.rot_first;      // of the rotated part
          if (i < 0 || i >= r.rot_dim) continue;
          const bool second = kHalf ? i >= pairs : (i & 1) != 0;
          const int other = kHalf ? (second ? -pairs : pairs) : (second ? -1 : 1);
          const float x1 = bf16_lo(c.e[j]), y1 = bf16_lo(row[e0 + j + other]);
          const float2 z = second ? turn(y1, x1, cs[kHalf ? i - pairs : i >> 1]) : turn(x1, y1, cs[kHalf ? i : i >> 1]);
          c.e[j] = f32_to_bf16_rne_dev(second ? z.y : z.x);
        }
        *reinterpret_cast<uint4*>(t.dst + (row0 + token) * t.out + at) = c.v;
      }
      __syncthreads();
    }
  }
}

bool aligned_rows(const RopeRows& t, int heads) {
  if (heads == 0) return true;
  return ((reinterpret_cast<uintptr_t>(t.src) | reinterpret_cast<uintptr_t>(t.dst)) & 15u) == 0 && t.in % 8 == 0 &&
         t.out % 8 == 0;
}

}  // namespace

hipError_t launch_rope(const RopeArgs& args, hipStream_t s) {
  RopeArgs a = args;
  const pask_rope& r = a.rope;
  const bool half = r.layout == PASK_ROPE_HALF;
  const bool rows16 = r.head_dim % 8 == 0 && aligned_rows(a.q, a.q_heads) && aligned_rows(a.k, a.k_heads);
  // 16-byte chunks where every chunk is whole: rows, heads, the rotated part and, in the half layout, its halves.
  const bool chunks = rows16 && r.rot_first % 8 == 0 && r.rot_dim % (half ? 16 : 8) == 0;
  const int rest = r.head_dim - r.rot_dim;
  a.rot_pieces = chunks ? r.rot_dim / (half ? 16 : 8) : r.rot_dim / 2;
  a.pieces = a.rot_pieces + (chunks ? rest / 8 : rest);
  a.q_copies = a.q.src != a.q.dst;
  a.k_copies = a.k.src != a.k.dst;
  if (!(a.q_copies && a.q_heads) && !(a.k_copies && a.k_heads)) a.pieces = a.rot_pieces;   // nothing to copy
  const int heads = a.q_heads + a.k_heads;
  const int64_t rows = (int64_t)a.batch * a.max_new;
  const bool staged = rows16 && !chunks;
  // Turns of a workgroup that a row takes: with few rows they go to workgroups of their own, with many a workgroup takes
  // several rows (the angles of a row are made by 1 thread a pair).
  const int each = staged ? kThreads / (r.head_dim / 8) : kThreads;
  const int64_t per_row = ((int64_t)heads * (staged ? 1 : a.pieces) + each - 1) / each;
  a.tokens = rows >= 4096 ? (rows >= 16384 ? 8 : 4) : 1;
  const int64_t blocks = std::min<int64_t>((rows + a.tokens - 1) / a.tokens, 1 << 22);   // the rest in turn
  const int split = a.tokens > 1 ? 1 : (int)std::max<int64_t>(1, std::min(per_row, 4096 / blocks));
  const dim3 grid((unsigned)blocks, (unsigned)split), threads(kThreads);
  const size_t lds = sizeof(float2) * (size_t)a.tokens * (r.rot_dim / 2);
  if (staged) {
    if (half) rope_staged_kernel<true><<<grid, threads, lds, s>>>(a);
    else rope_staged_kernel<false><<<grid, threads, lds, s>>>(a);
  } else if (chunks) {
    if (half) rope_kernel<true, true><<<grid, threads, lds, s>>>(a);
    else rope_kernel<true, false><<<grid, threads, lds, s>>>(a);
  } else {
    if (half) rope_kernel<false, true><<<grid, threads, lds, s>>>(a);
    else rope_kernel<false, false><<<grid, threads, lds, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace pask
