// Reductions over the 64 lanes of a wave, in the vector ALU.
#pragma once

#include "common.hpp"

namespace grace {

// ---------------------------------------------------------------------------
// wave reductions over 64 lanes, every lane gets the result.  Partners are
// lanes l ^ 32, 16, 8, 4, 2, 1 in that order; all six steps stay in the vector
// ALU (half and row swaps, row rotations, quad permutes) instead of going
// through LDS.  A rotation by 4 within 16 lanes reaches l ^ 4 because lanes l
// and l ^ 8 already agree.
// ---------------------------------------------------------------------------
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __builtin_bit_cast(
      float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
// The six steps for NR values of each lane at once (NR = 1, 2 or 4), sharing
// the swaps and all later steps: row j's result ends in the lanes of group
// lane_of_row<NR>(j) (all lanes for NR = 1, a half for 2, 16 lanes for 4).  Each
// row's order of operations is that of NR = 1.
template <int NR>
__device__ __forceinline__ constexpr int lane_of_row(int j) {
  return NR == 1 ? 0 : (NR == 2 ? 32 * j : 32 * (j & 1) + 16 * (j >> 1));
}
template <int NR>
__device__ __forceinline__ int row_of_lane(int lane) {
  return NR == 1 ? 0 : (NR == 2 ? lane >> 5 : (lane >> 5) + 2 * ((lane >> 4) & 1));
}
template <class Op>
__device__ __forceinline__ float swap_halves(float a, float b, Op op) {
  const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return op(__uint_as_float(h[0]), __uint_as_float(h[1]));
}
template <int NR, class Op>
__device__ __forceinline__ float reduce_rows(const float (&v)[NR], Op op) {
  static_assert(NR == 1 || NR == 2 || NR == 4, "rows per wave");
  const float y = swap_halves(v[0], v[NR > 1 ? 1 : 0], op);
  float w = y;
  if constexpr (NR == 4) w = swap_halves(v[2], v[3], op);
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(w), false, false);
  float x = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  x = op(x, dpp<0x128>(x));   // row_ror:8
  x = op(x, dpp<0x124>(x));   // row_ror:4
  x = op(x, dpp<0x4E>(x));    // quad_perm 2,3,0,1
  return op(x, dpp<0xB1>(x)); // quad_perm 1,0,3,2
}
template <int NR>
__device__ __forceinline__ float max_rows(const float (&v)[NR]) {
  return reduce_rows<NR>(v, [](float a, float b) { return max3(a, b, b); });
}
template <int NR>
__device__ __forceinline__ float sum_rows(const float (&v)[NR]) {
  return reduce_rows<NR>(v, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float wave_max(float x) { return max_rows<1>({x}); }
__device__ __forceinline__ float wave_sum(float x) { return sum_rows<1>({x}); }
// x of lane l, in a scalar register
__device__ __forceinline__ float lane_value(float x, int l) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), l));
}

// x where bit e of `bits` is set, else -inf (one bit-field extract, one bit select)
__device__ __forceinline__ float keep_bit(float x, uint32_t bits, int e) {
  const uint32_t m = (uint32_t)((int32_t)(bits << (31 - e)) >> 31);
  return __uint_as_float((__float_as_uint(x) & m) | (0xff800000u & ~m));
}

}  // namespace grace
