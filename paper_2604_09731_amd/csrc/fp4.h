// The 4-bit cache's number format and page layout.  An element is an E2M1 code (OCP microscaling formats: sign, two exponent
// bits with bias 1, one mantissa bit; 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), and the 32 codes of consecutive head
// dims of one token share a scale 2^(byte - 127), byte 255 meaning that all of them are NaN.  The conversions are the
// processor's: they agree with the definition for all 256 scale bytes and 16 codes, and for every rounding tie.
//
// A page (one block and kv head) is made of 16-byte vectors, each one load of a lane, and the scale bytes behind them:
//   K: 32 head dims of one token, which share a scale; the scales lie token by token.
//   V: 4 head dims of 8 consecutive tokens (two bytes a token): what a lane of the output product contracts over.  Two
//      codes that are converted together belong to one token, so they share a scale; the scales of 8 tokens lie together.
#ifndef SMART_FP4_H_
#define SMART_FP4_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace smart {

typedef __attribute__((ext_vector_type(2))) __bf16 fp4_bf16x2;
typedef __attribute__((ext_vector_type(2))) float fp4_floatx2;

// Byte offsets in a page of bs slots of D head dims.  The vector that holds (slot, d), and where in it.
__device__ inline int fp4_k_vector(int bs, int slot, int d) { return ((d >> 5) * bs + slot) * 16; }
__device__ inline int fp4_v_vector(int D, int slot, int d) { return ((slot >> 3) * (D >> 2) + (d >> 2)) * 16; }
__device__ inline int fp4_k_code(int bs, int slot, int d) { return fp4_k_vector(bs, slot, d) + ((d & 31) >> 1); }
__device__ inline int fp4_v_code(int D, int slot, int d) { return fp4_v_vector(D, slot, d) + (slot & 7) * 2 + ((d & 3) >> 1); }
__device__ inline int fp4_k_scale(int bs, int D, int slot, int d) { return bs * (D >> 1) + slot * (D >> 5) + (d >> 5); }
__device__ inline int fp4_v_scale(int bs, int D, int slot, int d) { return bs * (D >> 1) + (d >> 5) * bs + slot; }

// A scale byte as the binary32 the conversions take its exponent from.
__device__ inline float fp4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// The same out of byte kByte of a dword, with what lies beside the byte left where it is: the conversions look at the exponent
// bits alone (checked for all bytes against 256 patterns of sign and mantissa bits).
template <int kByte>
__device__ inline float fp4_scale_of(uint32_t w) { return __uint_as_float(kByte == 3 ? w >> 1 : w << (23 - 8 * kByte)); }

// One element of a page, as binary32 (exact).
__device__ inline float fp4_element(uint8_t pair, uint8_t scale, int d) {
  const fp4_floatx2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)pair, fp4_scale(scale), 0);
  return d & 1 ? x[1] : x[0];
}
__device__ inline float fp4_k_element(const uint8_t* page, int bs, int D, int slot, int d) {
  return fp4_element(page[fp4_k_code(bs, slot, d)], page[fp4_k_scale(bs, D, slot, d)], d);
}
__device__ inline float fp4_v_element(const uint8_t* page, int bs, int D, int slot, int d) {
  return fp4_element(page[fp4_v_code(D, slot, d)], page[fp4_v_scale(bs, D, slot, d)], d);
}

// The scale byte of 32 elements, of which `top` is the largest absolute value as bits.  2^(e - 2) puts a largest value in
// [1, 2) 2^e at 4 .. 8 steps of the grid that ends at 6.  Up to 7 the nearest value is 6, at most one step off, half of the
// distance from 4 to 6 as everywhere up there; beyond, the next scale is taken, so that nothing is cut off by more than rounding
// would cost.  Kept within 2^-125 .. 2^125: then no stored value is subnormal or infinite (larger ones become 6 2^125).
__device__ inline uint32_t fp4_scale_byte(uint32_t top) {
  if (top > 0x7F800000u) return 255u;  // a NaN among them
  const int e = (int)(top >> 23) - 2 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return (uint32_t)(e < 2 ? 2 : (e > 252 ? 252 : e));
}

// Four pairs of elements -> four bytes of codes: nearest, ties to the even code, infinities and what lies beyond 6 become 6.
__device__ inline uint32_t fp4_codes8(const float* x, float scale) {
  uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}

}  // namespace smart
#endif
