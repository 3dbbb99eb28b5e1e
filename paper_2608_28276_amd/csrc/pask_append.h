// Helpers of the kernels that write pages (pask_append.hip, pask_latent.hip),
// beside those that the attention shares (pask_device.h).
#pragma once

#include "pask_device.h"
#include "pask_pages.h"

namespace pask {

hipError_t launch_append_plan(const AppendArgs& a, hipStream_t s);   // slots, pages and counters alone; no window, no states

// The offset-binary codes q + 8 of the 8 bf16 elements of x under scale s
// (inv ~ 1 / s), the rule of quant_code, with code u in the low byte of b[u]
// (bits 4..7 zero, the bits above unspecified).  y = RN(x * inv + 1.5 * 2^23
// + 8) lies in [2^23, 2^24), where floats are spaced by 1, so its low byte is
// rint(x * inv) + 8; r = x * inv - (y - M) is the part rounded away.  As in
// codes8, x * inv rounds like x / s unless x / s lies within 2^-12 of a
// half-integer, so a lane whose largest |r| comes within 1.2e-4 of 1/2 takes
// quant_code for its 8 elements.  plain: s is a normal, unsaturated fp16
// scale of the group's absmax (quant_scale_bf16), so |x / s| <= 7 (1 + 2^-11)
// for every element of the group and the code needs no clamp; a lane without
// it (s subnormal or zero, or saturated at 65504) takes quant_code too.  About
// half the vector instructions of codes8 + k_word, which the bulk pack of
// RETAIN-LOW pages, bound by its vector ALU, spends most of its time on.
__device__ __forceinline__ void code_bytes8(const uint4& x, float s, float inv, bool plain, uint32_t (&b)[8]) {
  const float f[8] = {bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y),
                      bf16_lo(x.z), bf16_hi(x.z), bf16_lo(x.w), bf16_hi(x.w)};
  constexpr float M = 12582920.0f;                 // 1.5 * 2^23 + 8
  float worst = 0.0f;
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const float y = fmaf(f[u], inv, M);
    worst = fmaxf(worst, fabsf(fmaf(f[u], inv, M - y)));
    b[u] = __float_as_uint(y);
  }
  const bool exact = !plain || worst > 0.49988f;
  if (__ballot(exact)) {
    if (exact) {
#pragma unroll
      for (int u = 0; u < 8; ++u) b[u] = (uint32_t)(quant_code(f[u], s, inv) + 8);
    }
  }
}
// Low bytes of w0..w3 as bytes 0..3 of one word.
__device__ __forceinline__ uint32_t low_bytes4(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3) {
  return __builtin_amdgcn_perm(w1, w0, 0x0c0c0400u) | __builtin_amdgcn_perm(w3, w2, 0x04000c0cu);
}

// The largest |element| of the 8 bf16 in x, as the bits of its bf16 magnitude
// (the order of non-negative floats is that of their bits): packed 16-bit
// integer maxima of the sign-cleared words.
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t abs_max_bits8(const uint4& x) {
  const uint32_t m = 0x7FFF7FFFu;
  const u16x2_t a = __builtin_bit_cast(u16x2_t, x.x & m), b = __builtin_bit_cast(u16x2_t, x.y & m);
  const u16x2_t c = __builtin_bit_cast(u16x2_t, x.z & m), d = __builtin_bit_cast(u16x2_t, x.w & m);
  const u16x2_t r = __builtin_elementwise_max(__builtin_elementwise_max(a, b), __builtin_elementwise_max(c, d));
  return r.x > r.y ? (uint32_t)r.x : (uint32_t)r.y;
}

// quant_scale of a bf16 absmax, dividing only where s is an fp16 subnormal:
// from 7 * 2^-14 up, the product with RN(1/7) rounds to the same fp16 as the
// correctly rounded quotient (an exact quotient of a bf16 by 7 has at most 8
// significant bits, an inexact one never comes within 2^-15 of an fp16
// midpoint); below it an exact quotient can be a midpoint between fp16
// subnormals, which the product may miss.  Equal to quant_scale for every
// bf16 absmax (checked over all of them on the CPU).  plain: s is a normal
// fp16 and not saturated (7 * 2^-14 <= absmax <= 7 * 65504).
__device__ __forceinline__ uint16_t quant_scale_bf16(float absmax, float& s, float& inv, bool& plain) {
  float q = absmax * (1.0f / 7.0f);
  const bool small = absmax < 7.0f * 0x1p-14f;
  if (__ballot(small)) {
    if (small) {
      float a = absmax;
      asm volatile("" : "+v"(a));                  // no code: keeps the division on this rare branch
      q = a / 7.0f;
    }
  }
  plain = !small && absmax <= 7.0f * 65504.0f;
  const _Float16 h = (_Float16)fminf(q, 65504.0f);
  s = (float)h;
  inv = __builtin_amdgcn_rcpf(s);
  return __builtin_bit_cast(uint16_t, h);
}

// Tokens that sequence b appends in this call.
__device__ __forceinline__ int clamp_n_new(const AppendArgs& a, int b, uint32_t& flags) {
  int n = a.n_new ? a.n_new[b] : a.max_new;
  if (n < 0 || n > a.max_new) {
    flags |= PASK_FLAG_BAD_COUNT;
    n = n < 0 ? 0 : a.max_new;
  }
  return n;
}

// A 16-byte piece of a page a bulk append writes once (read only by later
// attention calls): non-temporal, so the stream does not displace other lines
// (and, with whole lines written, none is read first: the batch-64 prompt
// append's counter traffic fell from 1.076x to 1.012x its algorithmic bytes).
__device__ __forceinline__ void stream_store16(uint8_t* p, const uint4& v) {
  __builtin_nontemporal_store(u32x4_t{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4_t*>(p));
}

}  // namespace pask
