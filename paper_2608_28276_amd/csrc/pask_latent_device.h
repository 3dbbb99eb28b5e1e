// Shared by the latent-attention kernels (pask_latent.hip: persisting and
// reading back; pask_latent_attn.hip: absorbed decode attention): the launch
// arguments and the page layout.
#pragma once

#include "pask_device.h"
#include "pask_latent_internal.h"

namespace pask {
namespace {

// Pages of 16 slots, laid out for the attention kernel, which copies a page
// into LDS as it lies and uses the tile both as keys and as values:
//   HIGH  16-byte chunks, chunk 64 i + 16 q + (t ^ 8 (q & 1)) holding elements
//         32 i + 8 q .. + 7 of slot t (the rotary key follows the latent), so
//         lane (q, t) of a score operand reads 1 KiB per wave contiguously, and
//         the transposing reads of the value operand, which take 4 slots x 16
//         elements per 16 lanes, fall on all banks (without the XOR the chunks
//         of two neighbouring q would share them).
//   LOW   code words (16 i + t) * 4 + q of elements 32 i + 8 q .. + 7 (k_word
//         order, offset binary): the 16 bytes and the scale of a 32-element
//         group belong to one thread, in the write and in the attention's
//         widening; fp16 scales 16 i + t; the rotary keys' chunks as in HIGH.
template <int R, int P>
struct LatentPage {
  static constexpr int kRank = R, kRope = P;
  static constexpr int RI = R / 32, PI = P / 32, KI = RI + PI;   // 32-element groups
  static constexpr int kHiBytes = 32 * (R + P), kHiChunks = 64 * KI;
  static constexpr int kGroups = 16 * RI;                        // code groups of a LOW page
  static constexpr int kScales = 16 * kGroups, kRopeAt = kScales + 2 * kGroups;
  static constexpr int kLoBytes = kRopeAt + 32 * P, kRopeChunks = 64 * PI;
  static_assert(kLoBytes % 16 == 0 && kRopeAt % 16 == 0, "16-byte pieces");
};
// Slot t and its chunk position within a row of 16 chunks of quarter q.
__host__ __device__ __forceinline__ constexpr int latent_swap(int q, int t) { return t ^ ((q & 1) << 3); }

// The bf16 values of the 8 codes of a word under scale s, as 16 bytes in
// element order: (n - 8) * s = fma(n, s, -8 s) is exact in fp32 (a code has 3
// bits, an fp16 scale 11), so the one rounding is the format's, to bf16.
__device__ __forceinline__ uint4 low_values(uint32_t w, float s) {
  const uint32_t lo = w & 0x0F0F0F0Fu, hi = (w >> 4) & 0x0F0F0F0Fu;
  const float z = -8.0f * s;
  auto v = [&](uint32_t p, int b) { return fmaf((float)((p >> (8 * b)) & 0xFFu), s, z); };
  return make_uint4(pack_bf16x2(v(lo, 0), v(lo, 1)), pack_bf16x2(v(lo, 2), v(lo, 3)),
                    pack_bf16x2(v(hi, 0), v(hi, 1)), pack_bf16x2(v(hi, 2), v(hi, 3)));
}
__device__ __forceinline__ float half_value(uint16_t h) { return (float)__builtin_bit_cast(_Float16, h); }

}  // namespace
}  // namespace pask
