// What the kernels that rank a row's experts share: ordered bit patterns and reductions over the
// 16 lanes of a row.
#pragma once

#include "common.h"

namespace mla {

__device__ __forceinline__ uint32_t total_order_bits(float x) {
  const uint32_t u = __float_as_uint(x);
  return (u >> 31) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ float from_total_order_bits(uint32_t t) {
  return __uint_as_float((t >> 31) ? (t & 0x7FFFFFFFu) : ~t);
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}

__device__ __forceinline__ uint32_t max_u32(uint32_t x, uint32_t y) { return x > y ? x : y; }
__device__ __forceinline__ uint32_t med_u32(uint32_t x, uint32_t y, uint32_t z) {
  uint32_t m;
  asm("v_med3_u32 %0, %1, %2, %3" : "=v"(m) : "v"(x), "v"(y), "v"(z));
  return m;
}
// maximum over each row of 16 lanes, in every lane
__device__ __forceinline__ uint32_t row_max_u32(uint32_t v) {
  v = max_u32(v, dpp<0xB1>(v));
  v = max_u32(v, dpp<0x4E>(v));
  v = max_u32(v, dpp<0x141>(v));
  return max_u32(v, dpp<0x140>(v));
}
__device__ __forceinline__ uint32_t row_sum_u32(uint32_t v) {
  v += dpp<0xB1>(v);
  v += dpp<0x4E>(v);
  v += dpp<0x141>(v);
  return v + dpp<0x140>(v);
}
// lane J of each row of 16, in every lane of the row (row_newbcast)
template <int J>
__device__ __forceinline__ float row_bcast(float v) {
  return __uint_as_float(dpp<0x150 + J>(__float_as_uint(v)));
}

}  // namespace mla
