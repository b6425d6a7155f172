// Eight bits with scales: e4m3 codes, and for 32 consecutive elements of a row one power of
// two 2^(byte - 127), the smallest that brings the largest of them to 448 (the largest e4m3
// number) or below, at least 2^-126.  So nothing saturates, and a code is off by at most half
// an e4m3 step (2^-4 of its value, 2^-10 of the scale below its normal numbers).
#pragma once

#include "ec_common.h"

namespace ec {

constexpr int MX_BLOCK = 32;         // elements of a scale
constexpr uint32_t MX_NAN = 255;     // the scale of a block that holds a NaN or an infinity

// Magnitude bits of a value: as integers they order NaN above infinity above every number.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// The scale's byte, from the largest magnitude of the block: with it 1.m 2^(x - 127), the
// exponent e solves 1.m 2^(x - 127) <= 1.75 2^8 2^e.
__device__ __forceinline__ uint32_t mx_byte(uint32_t top) {
  if (top >= 0x7f800000u) return MX_NAN;
  const uint32_t x = (top >> 23) + ((top & 0x7fffffu) > 0x600000u);
  return x > 9 ? x - 8 : 1;
}

// What a value is multiplied by before its rounding, 2^(127 - byte): exact.  A NaN makes every
// code of its block NaN.
__device__ __forceinline__ float mx_inverse(uint32_t byte) {
  return __uint_as_float(byte == MX_NAN ? 0x7fc00000u : (254 - byte) << 23);
}

// Four codes (round to nearest, ties to even).
__device__ __forceinline__ uint32_t mx_codes4(const float* v, float inverse) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inverse, v[1] * inverse, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inverse, v[3] * inverse, w, true);
  return (uint32_t)w;
}

// The largest over the 32 / VEC neighbouring lanes that hold a block, VEC elements each.
template <int VEC>
__device__ __forceinline__ uint32_t mx_block_max(uint32_t t) {
  static_assert(VEC == 8 || VEC == 4, "");
  t = max(t, dpp_u32<0xB1>(t));
  t = max(t, dpp_u32<0x4E>(t));
  if (VEC == 4) t = max(t, dpp_u32<0x141>(t));   // the other quad of eight lanes
  return t;
}

// The codes of VEC elements.
template <int VEC>
__device__ __forceinline__ void mx_store(uint8_t* q, const float* v, float inverse) {
  if constexpr (VEC == 8)
    *reinterpret_cast<uint2*>(q) = make_uint2(mx_codes4(v, inverse), mx_codes4(v + 4, inverse));
  else
    *reinterpret_cast<uint32_t*>(q) = mx_codes4(v, inverse);
}

}  // namespace ec
