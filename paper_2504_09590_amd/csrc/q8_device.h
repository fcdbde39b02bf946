// Device helpers of the 8-bit cache: rows of 128 values held as e4m3 codes with
// one power-of-two scale 2^e per slot and KV head, kept as the byte e + 127.
//
// e is the least integer with max |x| <= 448 * 2^e over the row's finite values
// (448 is the largest e4m3 value), so nothing saturates; a code is x * 2^-e
// rounded to the nearest e4m3 value, ties to even. e4m3 is a floating format: a
// finer scale than a power of two would gain no relative precision, and with it a
// value code * 2^e is exact in bf16 and the conversion to bf16 applies it for
// nothing. One scale per slot, because the slot is what a request owns here: two
// requests fill a block from its two ends, and single slots are checkpointed,
// overwritten and put back, so a scale of a whole block would have two writers.
#pragma once

#include "bros_device.h"

namespace bros {
namespace q8 {

typedef unsigned v2u_t __attribute__((ext_vector_type(2)));
typedef unsigned v4u_t __attribute__((ext_vector_type(4)));
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2_t;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float float2_t;

// Exponents a row may take. The smallest code, 2^-9, times 2^e stays a normal bf16 value down to
// e = -117; -100 is that with a margin. Above 120 no finite fp32 row reaches.
constexpr int kMinExp = -100, kMaxExp = 120;
constexpr uint32_t kNaNBits = 0x7fc00000u;

// Scale exponent of a row whose largest finite magnitude is amax (448 = 1.75 * 2^8).
__device__ __forceinline__ int row_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, kMinExp), kMaxExp);
}
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// |x| where x is finite, else 0 (infinities and NaNs take no part in the scale).
__device__ __forceinline__ float finite_magnitude(float x) {
  const float m = fabsf(x);
  return m < INFINITY ? m : 0.0f;
}
// Four e4m3 codes of x * mul (mul = 2^-e); a value that is not finite becomes the NaN code.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float mul) {
  const auto v = [&](float x) { return fabsf(x) < INFINITY ? x * mul : __uint_as_float(kNaNBits); };
  int r = 0;
  r = __builtin_amdgcn_cvt_pk_fp8_f32(v(a), v(b), r, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(v(c), v(d), r, true);
  return (uint32_t)r;
}

// The values of a scale byte and of codes.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }
// A byte that marks, added to the magnitude of a row's code (below 128), the sum's top bit where
// the value is not finite in bf16 and fp32: the NaN code, a scale of 255 (none), and values from
// 2^128 on. These are codes 2^(x - 7) (1 + m / 8), x their exponent field, with x >= 262 - byte: of the
// scales that an append writes only the largest, 247, has any (256, for a
// finite value of 1.9375 * 2^127 or more).
__device__ __forceinline__ uint32_t not_finite_mark(uint32_t byte) {
  return byte < 247u ? 1u : byte < 255u ? 8u * (byte - 246u) : 128u;
}
// The bytes of w whose values are not finite, as their top bits.
__device__ __forceinline__ uint32_t not_finite(uint32_t w, uint32_t byte) {
  return ((w & 0x7f7f7f7fu) + not_finite_mark(byte) * 0x01010101u) & 0x80808080u;
}
// Two codes (the low or the high half of w) times the scale, as bf16 (exact).
template <bool HI>
__device__ __forceinline__ uint32_t values2_bf16(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}
__device__ __forceinline__ uint32_t pack2_bf16(float lo, float hi) {   // round to nearest even
  const float2_t f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
}

}  // namespace q8
}  // namespace bros
