// fp32 products on the bf16 matrix cores (gfx950).
//
// The fp32 MFMA runs at 1/16 of the bf16 rate.  An fp32 value is instead
// written exactly as the sum of three bf16 values,
//
//   x = h + m + l,  h = bf16(x), m = bf16(x - h), l = x - h - m
//
// (each difference is exact, |m| <= 2^-8 |x|, |l| <= 2^-17 |x|), and a product
// x y is the six terms l h' + h l' + m m' + m h' + h m' + h h'; the three left
// out reach 2^-24 |x y| at worst, the fp32 rounding of one product.  An MFMA
// rounds its sum about once per 8 products: h h' has a sum of its own and the
// five small terms another, so that the large one is rounded 4 times per 32
// values, less often than in a chain of fp32 products.  (Values below 2^-110
// run out of bf16's exponents: absolute precision 2^-133.)
//
// A workgroup that meets a value of kHuge or more (an infinity has no such
// split, and terms of opposite sign could overflow where the sum does not)
// takes its tile again with fp32 MFMAs.  A NaN is one in every term.
#pragma once

#include "group.h"

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2_any __attribute__((ext_vector_type(2), aligned(4)));

constexpr float kHuge = 1.125899906842624e15f;  // 2^50: products below 2^100, and any sum of them finite

// Two values -> their three parts, packed.
__device__ __forceinline__ void split2(float a, float b, uint32_t (&p)[3]) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    p[i] = pack2_bf16(a, b);
    a -= __uint_as_float(p[i] << 16);
    b -= __uint_as_float(p[i] & 0xffff0000u);
  }
}

__device__ __forceinline__ f32x16_t mma(const u32x4 &a, const u32x4 &b, const f32x16_t &c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0,
                                                 0, 0);
}

}  // namespace
