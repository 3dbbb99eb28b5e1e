// Copies into LDS through the compiler's builtin on either side of ones in asm:
// what test_native_lds_copies.py compiles and follows m0 through.
#include <hip/hip_runtime.h>

#include "pask_latent_device.h"

namespace pask {
namespace {

template <bool kOnce>
__global__ void copies(const uint8_t* a, const uint8_t* b, uint4* out) {
  __shared__ __align__(1024) uint8_t s[2][1024];
  const uint32_t at = threadIdx.x * 16;
  load_to_lds<kOnce>(a + at, s[0]);
  copy_to_lds<kOnce>(b, at, lds_address(s[1]));
  load_to_lds<kOnce>(b + 4096 + at, s[0]);
  wait_loads();
  __syncthreads();
  out[threadIdx.x] = *reinterpret_cast<const uint4*>(s[0] + at);
  out[64 + threadIdx.x] = *reinterpret_cast<const uint4*>(s[1] + at);
}

template __global__ void copies<false>(const uint8_t*, const uint8_t*, uint4*);
template __global__ void copies<true>(const uint8_t*, const uint8_t*, uint4*);

}  // namespace
}  // namespace pask
