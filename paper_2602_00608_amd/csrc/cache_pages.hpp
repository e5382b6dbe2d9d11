// Keys and values in four bits: where they lie, and how eight of them become numbers.
//
// Blocks of 32 channels of a head of a token share a power of two 2^e, kept as the byte e + 127 (255: not a number); a value is a sign and one of
// 0, 0.5, 1, 1.5, 2, 3, 4, 6 times that, in a code of four bits (the matrix cores' and conversions' own format of that width).  A value has two significant
// bits: bf16 holds it to the bit, and f16 if it was f16 before.  The conversions below round nothing where that is so.
//
// A page holds `page_tokens` tokens, head by head, so that what a workgroup reads of a head lies together:
//   [head][ keys' codes | values' codes | keys' exponents | values' exponents ]
// with 16 bytes of codes a block, an odd channel in the high half of its byte, channels past the last one zero, and room for 1, 2, 4 or 8 exponents a token.
#pragma once
#include "conv_device.hpp"

namespace wmdec {

__host__ __device__ constexpr int exponent_bytes(int blocks) { return blocks <= 1 ? 1 : blocks <= 2 ? 2 : blocks <= 4 ? 4 : 8; }

// head h's part of page `number`; null where that is no page
__device__ __forceinline__ unsigned char* head_of_page(const CachePages& p, int number, int h) {
  return (unsigned)number < (unsigned)p.pages ? p.data + (unsigned long)number * p.page_bytes + (unsigned long)((unsigned)h * p.head_bytes) : nullptr;
}

// eight channels: a 32-bit word of codes -> four words of two values each, times the power of two
template <typename T> __device__ __forceinline__ u32x4 widen(unsigned codes, float unit);
template <> __device__ __forceinline__ u32x4 widen<bf16_t>(unsigned codes, float unit) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 0)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 2)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 3))};
}
template <> __device__ __forceinline__ u32x4 widen<f16_t>(unsigned codes, float unit) {
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, unit, 0)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, unit, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, unit, 2)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, unit, 3))};
}
__device__ __forceinline__ float unit_of(unsigned exponent) { return __uint_as_float(exponent << 23); }   // (255 is infinite here and not a number to the conversions)

// floats -> their codes, in order from the low bits: times 1 / unit, to the nearest value, ties to the even code, 6 for what is above
__device__ __forceinline__ unsigned narrow(const float (&x)[4], float unit) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(__builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], unit, 0), x[2], x[3], unit, 1);
}
__device__ __forceinline__ unsigned narrow(const float (&x)[8], float unit) {
  unsigned w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], unit, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], unit, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], unit, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], unit, 3);
}

}  // namespace wmdec
