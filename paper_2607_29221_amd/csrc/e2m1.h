// Eight elements in 4 bits: a dword of e2m1 codes and a scale byte
// (include/mosaic_cache.h). gfx950 converts two codes at a time, with the scale
// as the exponent of a float32: to nearest, even codes between two, 6 beyond.
#pragma once

#include "cache.h"

namespace mosaic {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float e2m1_scale(uint32_t e) { return __uint_as_float(e << 23); }

// The codes of x, and their scale as the function's value.
__device__ __forceinline__ uint32_t e2m1_encode(const float* x, uint32_t* codes) {
  uint32_t top = 0;                              // the largest magnitude's bits; NaN is above infinity
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  // 2^e times 3.5 (not) to 7 (with): in eighths of a power of two, 1.75 is the border
  const int fit = (int)(top >> 23) - 2 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  const uint32_t e = top >= 0x7F800000u ? 255u : (uint32_t)min(max(fit, 1), 252);
  const float s = e2m1_scale(e);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
  *codes = e == 255u ? 0u : c;
  return e;
}

// What codes stand for under a scale, exactly: bf16 has room for all of them,
// two to a dword.
__device__ __forceinline__ void e2m1_decode(uint32_t codes, float s, uint32_t* x) {
  x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0));
  x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1));
  x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2));
  x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3));
}

}  // namespace
}  // namespace mosaic
