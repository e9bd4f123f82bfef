// Device-side helpers of the kernels on the cache in 4 bits (gfx950 only): codes to fp16 values, masks on those.
#pragma once

#include "sc_attend_device.h"
#include "sc_packed.h"

#pragma clang fp contract(off)

namespace sc {

typedef _Float16 half2 __attribute__((ext_vector_type(2)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ uint32_t bits_of(half2 v) { return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ half2 half2_of(uint32_t v) { return __builtin_bit_cast(half2, v); }

// fp16 round-to-nearest-even of two floats, packed.
__device__ __forceinline__ uint32_t pack2h(float a, float b) { return bits_of(__builtin_convertvector(floatx2{a, b}, half2)); }

// Of a word whose 16-bit halves hold a code each in bits 0..3 (4..7): the codes as fp16. An fp16 number with the code in its mantissa's last
// bits is 1024 + code (in bits 4..7 and exponent 6: 64 + code), exactly, so one logical operation and one packed addition make two. The
// logical one takes its masks from registers: two literals would make it two.
struct CodeBits {
  uint32_t low_mask, low_bits, high_mask, high_bits;
};
__device__ __forceinline__ CodeBits code_bits() {
  CodeBits b = {0x000f000fu, 0x64006400u, 0x00f000f0u, 0x54005400u};
  asm volatile("" : "+s"(b.low_mask), "+s"(b.high_mask), "+v"(b.low_bits), "+v"(b.high_bits));
  return b;
}
__device__ __forceinline__ half2 codes_low(uint32_t w, const CodeBits& b) { return half2_of((w & b.low_mask) | b.low_bits) + half2{-1024.0f16, -1024.0f16}; }
__device__ __forceinline__ half2 codes_high(uint32_t w, const CodeBits& b) { return half2_of((w & b.high_mask) | b.high_bits) + half2{-64.0f16, -64.0f16}; }

// The values of two codes: one rounding, as the format has it.
__device__ __forceinline__ uint32_t values2(half2 codes, half2 scale, half2 low) { return bits_of(__builtin_elementwise_fma(codes, scale, low)); }

// (a's, b's) scale, and minimum, of two (scale, minimum) words.
__device__ __forceinline__ half2 scales2(uint32_t a, uint32_t b) { return half2_of(__builtin_amdgcn_perm(b, a, 0x05040100u)); }
__device__ __forceinline__ half2 lows2(uint32_t a, uint32_t b) { return half2_of(__builtin_amdgcn_perm(b, a, 0x07060302u)); }

// The eight values of a word of codes, in the order 0 4 1 5 2 6 3 7 (what one mask leaves side by side). pair: its (scale, minimum).
__device__ __forceinline__ half8 values8(uint32_t w, uint32_t pair, const CodeBits& b) {
  const half2 s = scales2(pair, pair), m = lows2(pair, pair);
  const uint4 v{values2(codes_low(w, b), s, m), values2(codes_high(w, b), s, m), values2(codes_low(w >> 8, b), s, m), values2(codes_high(w >> 8, b), s, m)};
  return __builtin_bit_cast(half8, v);
}

// A row of queries comes into fp16's range by a power of two: lift_of that which takes its largest element into [2^14, 2^15) (a row of zeros or subnormal
// numbers: 2^141, below it), factor_of what takes its scores, formed of the lifted row, to powers of two. The factor stays a normal number: as zero it
// would make a masked score, minus infinity, NaN, and as infinity a score of zero. Below 2^-126 the row's scores are under 2^-87 either way (lifted ones
// are 2^39 at most) and count as nothing; past 2^128 two that differ (by 2^-48 at least, lifted) do so by 2^80 or more.
__device__ __forceinline__ int lift_of(float most) { return 141 - (int)((__float_as_uint(most) >> 23) & 255u); }
__device__ __forceinline__ float factor_of(float scale_log2, int lift) {
  return fminf(fmaxf(ldexpf(scale_log2, -lift), 0x1p-126f), 0x1.fffffep127f);
}

// Of two packed fp16 values those outside the mask become zero, and so do those that are infinite or NaN, which set *odd.
__device__ __forceinline__ uint32_t finite2h(uint32_t v, uint32_t mask, int* odd) {
  v &= mask;
  uint32_t f = v;
  if ((v & 0x7c00u) == 0x7c00u) f &= 0xffff0000u;
  if ((v & 0x7c000000u) == 0x7c000000u) f &= 0x0000ffffu;
  if (f != v) *odd = 1;
  return f;
}

// The value, not known to the compiler to be the same as before: an offset that is widened to 64 bits where it is used, not ahead of the loop,
// stays the 32-bit lane offset of a load with a scalar base; a scalar taken out of a block of arguments is kept by itself.
__device__ __forceinline__ uint32_t here(uint32_t v) {
  asm volatile("" : "+v"(v));
  return v;
}
__device__ __forceinline__ uint32_t alone(uint32_t v) {
  v = (uint32_t)uniform((int)v);
  asm volatile("" : "+s"(v));
  return v;
}

}  // namespace sc
