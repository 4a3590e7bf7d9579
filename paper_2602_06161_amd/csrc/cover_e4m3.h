// The e4m3 form of a row (include/cover.h): scale and codes, shared by the norm and the 8-bit cache.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cover {

// the scale of a row whose largest magnitude is `top` (a NaN there stays one)
__device__ __forceinline__ float e4m3_scale(float top) {
  const float s = top / 448.0f;
  return s < 0x1p-126f ? 0x1p-126f : s;
}

// four codes of a, b, c, d times inv, first in the lowest byte.  The instruction rounds to nearest,
// ties to even; |x * inv| <= 448 (1 + 2^-22), which rounds to 448 at most.
__device__ __forceinline__ uint32_t e4m3_pack(float a, float b, float c, float d, float inv) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, r, true);
}

// magnitude with an order in which NaN is the largest
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

}  // namespace cover
