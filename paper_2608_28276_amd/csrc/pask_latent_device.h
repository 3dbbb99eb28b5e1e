// Shared by the latent-attention kernels (pask_latent.hip: persisting and
// reading back; pask_latent_attn.hip: absorbed decode attention;
// pask_latent_prompt.hip: expanded attention): the page layout, the search of a
// list of positions and LDS access.
#pragma once

#include "pask_append.h"
#include "pask_latent_internal.h"

namespace pask {
namespace {

// Pages of 16 slots, laid out for the attention kernel, which copies a page
// into LDS as it lies and uses the tile both as keys and as values:
//   HIGH  16-byte chunks, chunk 64 i + 16 q + (t ^ 12 (q & 1)) holding elements
//         32 i + 8 q .. + 7 of slot t (the rotary key follows the latent).  A
//         score operand is 1 KiB per wave; its reads take lanes 0-3, 12-15,
//         20-23, 24-27 (and so on) at a time, which the XOR keeps on different
//         banks, while the transposing reads of the value operand, 4 slots x 2
//         chunks per 16 lanes, would without it find neighbouring q on the same
//         ones (cycles per instruction and compute unit, keys / values: no XOR
//         4.3 / 4, with 8 in place of 12 8.0 / 2, with 12 4.3 / 2).
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
__host__ __device__ __forceinline__ constexpr int latent_swap(int q, int t) { return t ^ ((q & 1) * 12); }

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

// Entries of an ascending list below x, known to be lo or more and hi or fewer:
// 16 lanes of a wave together, 16 entries at a time.
__device__ __forceinline__ int entries_below(const int32_t* list, int lo, int hi, int x) {
  const int lane = (int)threadIdx.x & 63, l = lane & 15;
  while (lo < hi) {
    const int step = (hi - lo + 15) >> 4, at = lo + (l + 1) * step - 1;
    const bool below = at < hi && list[at] < x;
    const int c = __popc((uint32_t)(__ballot(below) >> (lane & 48)) & 0xFFFFu);
    lo = min(lo + c * step, hi);
    hi = min(lo + step - 1, hi);
  }
  return lo;
}

// x, which the compiler takes for new (no code): what follows from it is made
// where it is used, not kept in registers through the loops around.
template <typename I>
__device__ __forceinline__ I fresh(I x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Transposing reads of LDS (ds_read_b64_tr_b16): of each 16 lanes, lanes 4r ..
// 4r + 3 address row r's four 8-byte quarters (4 rows of 16 2-byte elements),
// and lane i receives element i of the rows.  Four pairs of reads at a time,
// pair k at at[k] + kOff[k] and kStep behind it, in one asm block that waits
// for its own reads: before the builtin the compiler waits for every copy into
// LDS under way (load_to_lds), which is what the copies are there to avoid.
template <int kOff0, int kOff1, int kOff2, int kOff3, int kStep>
__device__ __forceinline__ void read_transposed(uint32_t at0, uint32_t at1, uint32_t at2, uint32_t at3, uint4 (&v)[4]) {
  uint2 a[4], b[4];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8 offset:%12\n\t"
      "ds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
      "ds_read_b64_tr_b16 %2, %9 offset:%14\n\t"
      "ds_read_b64_tr_b16 %3, %9 offset:%15\n\t"
      "ds_read_b64_tr_b16 %4, %10 offset:%16\n\t"
      "ds_read_b64_tr_b16 %5, %10 offset:%17\n\t"
      "ds_read_b64_tr_b16 %6, %11 offset:%18\n\t"
      "ds_read_b64_tr_b16 %7, %11 offset:%19\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(a[0]), "=&v"(b[0]), "=&v"(a[1]), "=&v"(b[1]), "=&v"(a[2]), "=&v"(b[2]), "=&v"(a[3]), "=&v"(b[3])
      : "v"(at0), "v"(at1), "v"(at2), "v"(at3), "n"(kOff0), "n"(kOff0 + kStep), "n"(kOff1), "n"(kOff1 + kStep),
        "n"(kOff2), "n"(kOff2 + kStep), "n"(kOff3), "n"(kOff3 + kStep)
      : "memory");
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = make_uint4(a[k].x, a[k].y, b[k].x, b[k].y);
}
// The same for eight pairs of one address, pair k at at + 512 k and kStep behind it.
template <int kStep>
__device__ __forceinline__ void read_transposed8(uint32_t at, uint4 (&v)[8]) {
  uint2 a[8], b[8];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %16\n\t"
      "ds_read_b64_tr_b16 %1, %16 offset:%17\n\t"
      "ds_read_b64_tr_b16 %2, %16 offset:512\n\t"
      "ds_read_b64_tr_b16 %3, %16 offset:%18\n\t"
      "ds_read_b64_tr_b16 %4, %16 offset:1024\n\t"
      "ds_read_b64_tr_b16 %5, %16 offset:%19\n\t"
      "ds_read_b64_tr_b16 %6, %16 offset:1536\n\t"
      "ds_read_b64_tr_b16 %7, %16 offset:%20\n\t"
      "ds_read_b64_tr_b16 %8, %16 offset:2048\n\t"
      "ds_read_b64_tr_b16 %9, %16 offset:%21\n\t"
      "ds_read_b64_tr_b16 %10, %16 offset:2560\n\t"
      "ds_read_b64_tr_b16 %11, %16 offset:%22\n\t"
      "ds_read_b64_tr_b16 %12, %16 offset:%25\n\t"
      "ds_read_b64_tr_b16 %13, %16 offset:%23\n\t"
      "ds_read_b64_tr_b16 %14, %16 offset:3584\n\t"
      "ds_read_b64_tr_b16 %15, %16 offset:%24\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(a[0]), "=&v"(b[0]), "=&v"(a[1]), "=&v"(b[1]), "=&v"(a[2]), "=&v"(b[2]), "=&v"(a[3]), "=&v"(b[3]),
        "=&v"(a[4]), "=&v"(b[4]), "=&v"(a[5]), "=&v"(b[5]), "=&v"(a[6]), "=&v"(b[6]), "=&v"(a[7]), "=&v"(b[7])
      : "v"(at), "n"(kStep), "n"(kStep + 512), "n"(kStep + 1024), "n"(kStep + 1536), "n"(kStep + 2048),
        "n"(kStep + 2560), "n"(kStep + 6 * 512), "n"(kStep + 3584), "n"(6 * 512)
      : "memory");
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = make_uint4(a[k].x, a[k].y, b[k].x, b[k].y);
}
// A barrier that LDS reads and writes of the workgroup are ordered by, and that
// copies under way do not wait for (__syncthreads waits for them).
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);              // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// 16 and 8 bytes of LDS by address, as plain vectors: before accesses of the
// struct types uint4 and uint2 the compiler waits for every copy under way.
typedef __attribute__((address_space(3))) u32x4_t lds_u32x4;
typedef __attribute__((address_space(3))) u32x2_t lds_u32x2;
__device__ __forceinline__ uint4 read_lds16(uint32_t lds) {
  const u32x4_t x = *(const lds_u32x4*)(uintptr_t)lds;
  return make_uint4(x[0], x[1], x[2], x[3]);
}
__device__ __forceinline__ void write_lds16(uint32_t lds, const uint4& v) {
  *(lds_u32x4*)(uintptr_t)lds = u32x4_t{v.x, v.y, v.z, v.w};
}
__device__ __forceinline__ void write_lds8(uint32_t lds, const uint2& v) {
  *(lds_u32x2*)(uintptr_t)lds = u32x2_t{v.x, v.y};
}
__device__ __forceinline__ uint32_t lds_address(const uint8_t* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)p;
}

// 16 bytes per lane from memory straight into LDS: lane l's to lds + 16 l (lds is
// the same for the wave).  The caller waits (wait_loads) and synchronises.
// kOnce: data read once per call (non-temporal).
template <bool kOnce>
__device__ __forceinline__ void load_to_lds(const void* src, uint8_t* lds) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)src,
                                   (__attribute__((address_space(3))) uint32_t*)lds, 16, 0, kOnce ? 2 : 0);
}
// The same from src (the same for the wave) + at, uncounted: the compiler waits
// for every load_to_lds that it knows of before the next read of LDS, that of
// another buffer too; these are waited for where the caller says so alone.  In
// asm, no register of which is written; m0, which holds the LDS address, cannot
// be declared as overwritten (the compiler reserves it, and merges the settings
// of its own copies on either side of this one), so it is given back.  Its two
// moves cost nothing that shows beside the copies of a prompt's pages (8,192
// tokens, bf16: 559 us without, 561 with; int4 811 and 815).
template <bool kOnce>
__device__ __forceinline__ void copy_to_lds(const uint8_t* src, uint32_t at, uint32_t lds) {
  lds = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds);
  uint32_t m0;
  if constexpr (kOnce)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "v"(at), "s"(src), "s"(lds) : "memory");
  else
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "v"(at), "s"(src), "s"(lds) : "memory");
}
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }   // vmcnt(0)

}  // namespace
}  // namespace pask
