// The 4-bit format of cached vectors: groups of 32 components, each with a scale of one byte.
//
// A component is (u - 8) s, u its 4 bits and s the group's scale.  Byte b of a scale stands for
// (4 + b % 4) 2^(b / 4 - 40), b < 252; 252 to 255 mark a group that holds no numbers.  s has three
// significant bits and u - 8 four at most, so that every product is a bf16 value exactly.  Bits of
// a vector: component c at bits 4 (c % 8) of its 32-bit word c / 8.
//
// Widening takes two instructions for two components beside the shift: 0x4300 | u are the bits of
// 128 + u in bf16, and (128 + u) s - 136 s is one fused multiply-add whose result needs no rounding.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

namespace dcl {

constexpr int Q4_GROUP = 32;    // components that share a scale
constexpr int Q4_SCALES = 252;  // bytes from here on: a group that holds no numbers
constexpr int Q4_NONE = 255;    // (the one that is written)

__device__ __forceinline__ uint32_t q4_mul(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t q4_fma(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}

// The scales of two groups, as two bf16, from their bytes in bits 0 - 7 and 16 - 23.  The bytes are put
// below the exponents' top, where 252 to 255 become infinity and NaN, and the product brings the
// others down to where they belong.
struct Q4Scale {
  uint32_t s, off;  // s; -136 s
};
__device__ __forceinline__ Q4Scale q4_scale(uint32_t bytes) {
  const uint32_t s = q4_mul(bytes * 32u + 0x60006000u, 0x0c000c00u);  // 2^-103
  return Q4Scale{s, q4_mul(s, 0xc308c308u)};                          // -136
}
__device__ __forceinline__ Q4Scale q4_scale_twice(uint32_t byte) { return q4_scale(byte * 0x10001u); }

// The components i (in the lower half) and i + 4 of a word's eight, i < 4.
// (One instruction for the mask and the exponents: left to the compiler they were two, and the integer pipe is
// what bounds the attention.)
__device__ __forceinline__ uint32_t q4_widen(uint32_t w, int i, const Q4Scale& f) {
  uint32_t x;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(x) : "r"(w >> (4 * i)), "r"(0x000f000fu), "r"(0x43004300u));
  return q4_fma(x, f.s, f.off);
}

}  // namespace dcl
