// The 4-bit cache's format on the device (specmoe_kv4.h): codes and scale bytes
// to values and back.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "specmoe_kv4.h"

namespace kv4 {

// The 16-byte aligned members of a cache, as the kernels take them
struct Cache {
  char* k_codes;
  char* k_scales;
  char* v_codes;
  char* v_scales;
};

// A scale byte as the fp32 number whose exponent is it: what the conversions
// of this GPU take as a scale (0 stands for 2^-127 there, 255 for NaN).
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Codes of byte BYTE of a word as two bfloat16 (the low code low), times their
// scale: exact, as bfloat16 has every value of a code and the exponents of the
// scales.
template <int BYTE>
__device__ __forceinline__ uint32_t bf16_of(uint32_t word, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, BYTE));
}

// Scale byte of a block whose largest magnitude has the fp32 bits `most`: the
// unit is 2^(k - 2) for most in [2^k, 1.75 2^k), 2^(k - 1) from there on, so that
// most / unit < 7, and at least 2^-126.
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
  if (most >= 0x7f800000u) return 255u;   // (an infinity or NaN)
  const int e = (int)(most >> 23) - 2 + ((most & 0x7fffffu) >= 0x600000u ? 1 : 0);
  return (uint32_t)max(e, 1);
}

// 8 values of a block as codes, with the block's scale byte.  The conversion
// rounds to nearest, ties to the even code.
__device__ __forceinline__ uint32_t codes_of(const float (&x)[8], uint32_t byte) {
  if (byte == 255u) return 0u;
  const float s = scale_of(byte);
  uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
}

// An fp64 value in fp32 such that every comparison with a number of fewer than
// 24 significant bits, so the rounding to a code too, comes out as the fp64
// value's would: what is not exact is rounded to the odd neighbour.
__device__ __forceinline__ float to_odd(double x) {
  const float f = (float)x;
  const double rest = x - (double)f;
  uint32_t u = __float_as_uint(f);
  if (rest != 0.0 && !(u & 1u) && u << 1 < 0xff000000u) {   // (not of an infinity or NaN)
    if (f == 0.f) u = rest > 0.0 ? 1u : 0x80000001u;
    else u += (rest > 0.0) == (f > 0.f) ? 1u : 0xffffffffu;
  }
  return __uint_as_float(u);
}

}  // namespace kv4
