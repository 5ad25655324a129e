// Rows held in 4 bits, on the device: E2M1 elements (magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign), element 2 i in the low
// half of byte i, and a scale byte for every kFp4Block of them, 2^(byte - 127).  The matrix unit's own conversions do the
// rounding (to nearest, ties to the even code) and the way back, with the scale as the exponent of a float: exact for every
// byte, denormal inputs included, and NaN for byte 255 (all 4096 (byte, code) pairs and 9429 inputs on and around the borders
// between codes compared with the definition).
#pragma once
#include <utility>

#include "common.hpp"

namespace vec {

constexpr int kFp4Block = VECTOR_FP4_BLOCK;
constexpr int fp4_code_bytes(int head_dim) { return head_dim / 2; }
constexpr int fp4_scale_bytes(int head_dim) { return head_dim / kFp4Block; }

typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(2))) short s16x2;

// f(0), f(1), .. with the number as a constant, which the conversions' byte selectors have to be
template <typename F, int... I> __device__ __forceinline__ void for_constants(std::integer_sequence<int, I...>, F f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F> __device__ __forceinline__ void for_each_constant(F f) { for_constants(std::make_integer_sequence<int, N>{}, f); }

// The scale of a block whose largest |x| has these bits: the smallest power of two with 7 of it no less than that, so that nothing is
// off by more than one unit (6 is the largest code: what lies between 6 and 7 loses no more than what lies between 4 and 6).  Its
// exponent is that of the largest magnitude, one more if the mantissa is above 1.75, less 2; 125 at most, since four of the next unit are
// infinite as a float.  An infinite or NaN element: 255.
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t top_bits) {
  if (top_bits >= 0x7f800000u) return 255u;
  return (uint32_t)min(max((int)((top_bits + 0x1fffffu) >> 23) - 2, 1), 252);
}
__device__ __forceinline__ float fp4_unit(uint32_t byte) { return __uint_as_float(byte << 23); }

// eight consecutive elements -> four bytes of codes; of a block that is NaN, zeros
__device__ __forceinline__ uint32_t fp4_codes(const float* x, uint32_t byte) {
  if (byte == 255u) return 0u;
  const float unit = fp4_unit(byte);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], unit, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], unit, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], unit, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], unit, 3);
  return c;
}
// elements 2 BYTE and 2 BYTE + 1 of eight, times the scale: as two bf16 (exact, an element has two significant bits), or floats
template <int BYTE> __device__ __forceinline__ uint32_t fp4_pair_bf16(uint32_t codes, float unit) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, BYTE));
}
template <int BYTE> __device__ __forceinline__ f32x2 fp4_pair_f32(uint32_t codes, float unit) {
  return __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, BYTE));
}

// Eight consecutive elements of a row of T as floats
template <typename T> __device__ __forceinline__ void load8(const T* at, float* x) {
  if constexpr (sizeof(T) == 2) {
    Unpack16<bf16_t>::run(load_chunk(at), x);
  } else {
    Unpack16<float>::run(load_chunk(at), x);
    Unpack16<float>::run(load_chunk(at + 4), x + 4);
  }
}
__device__ __forceinline__ uint32_t top_bits8(const float* x) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  return top;
}

// the largest of four adjacent lanes
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, false));    // lanes 1 0 3 2 of the four
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, false));  // lanes 2 3 0 1
}

}  // namespace vec
