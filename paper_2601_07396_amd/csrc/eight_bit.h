// Values in e4m3 with scales that are powers of two: what the kernels that make them and the ones that read them share.
#pragma once
#include "eight_bit_sizes.h"
#include "svdc_device.h"

namespace svdc {

// 16 bytes aligned to the smallest element: global memory takes wide accesses at any such address
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

// The scale of a block as its stored byte: 2^(byte - 127) for the least power of two with amax <= 448 * 2^e, e in -126 .. 126.
// With amax = 1.m * 2^(x - 127) and 448 = 1.75 * 2^8 that is e = x - 135, and one more where 1.m > 1.75.  An infinity counts as the
// largest float32; amax is never a NaN (the maximum of a NaN and a number is the number).
__device__ __forceinline__ int scale_byte(float amax) {
  const uint32_t u = __float_as_uint(fminf(amax, 3.402823466e38f));
  const int byte = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return u == 0 ? 127 : (byte < 1 ? 1 : byte);
}
__device__ __forceinline__ float inverse_scale(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }

// four values to e4m3, rounded to nearest even; |v| <= 448 or not finite (then NaN)
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// maximum over the 16 lanes of a DPP row (lanes 16 i .. 16 i + 15), in all of them
__device__ __forceinline__ float row16_max(float v) {
#define SVDC_ROR_MAX(n) \
  v = fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + n, 0xf, 0xf, false)))
  SVDC_ROR_MAX(8);
  SVDC_ROR_MAX(4);
  SVDC_ROR_MAX(2);
  SVDC_ROR_MAX(1);
#undef SVDC_ROR_MAX
  return v;
}

}  // namespace svdc
