// Wavefront helpers shared by the attention kernels.
#ifndef SMART_WAVE_H_
#define SMART_WAVE_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace smart {

__device__ inline int64_t readlane64(int64_t v, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)v, lane);
  const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)((uint64_t)v >> 32), lane);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// A value every lane agrees on, moved to scalar registers.
__device__ inline int64_t uniform64(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)v >> 32));
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// Inclusive add scan over the 64 lanes with data-parallel-primitive moves (no LDS traffic):
// shifts by 1, 2, 4, 8 inside each row of 16 lanes, then lane 15 of rows 0 and 2 is added to
// rows 1 and 3, then lane 31 to the upper half.  Lanes without a source add zero.
template <int kCtrl, int kRowMask>
__device__ inline int64_t dpp_add(int64_t v) {
  const int lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, kCtrl, kRowMask, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)((uint64_t)v >> 32), kCtrl, kRowMask, 0xf, false);
  return v + (int64_t)(((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo);
}

// One wavefront: exclusive scan of v and (uniform) the total.
__device__ inline int64_t wave_excl_scan(int64_t v, int lane, int64_t* total) {
  int64_t incl = v;
  incl = dpp_add<0x111, 0xf>(incl);  // row_shr:1
  incl = dpp_add<0x112, 0xf>(incl);  // row_shr:2
  incl = dpp_add<0x114, 0xf>(incl);  // row_shr:4
  incl = dpp_add<0x118, 0xf>(incl);  // row_shr:8
  incl = dpp_add<0x142, 0xa>(incl);  // row_bcast:15 into rows 1 and 3
  incl = dpp_add<0x143, 0xc>(incl);  // row_bcast:31 into rows 2 and 3
  *total = readlane64(incl, 63);
  return incl - v;
}

// Over the two lanes with the same lane % 32, and over the four with the same lane % 16: the result in each of them.
__device__ inline float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ inline float max_quarters(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ inline float sum_quarters(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return sum_halves(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// `sum` and the two bf16 of a pair: one dot product with two ones, rounded to nearest.
__device__ inline float add_pair(uint32_t pair, float sum) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3F803F80u), sum, false);
}

}  // namespace smart
#endif
