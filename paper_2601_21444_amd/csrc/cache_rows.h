// Rows of the cache in registers (device code): eight elements of a block to their codes and back, and where a row lies.
#pragma once
#include "cache.h"

namespace apbv {
namespace {

// Absolute value of a bf16 pattern as it is held: NaN counts as zero, infinity as the largest finite value.
__device__ __forceinline__ uint32_t held(uint32_t x) {
  const uint32_t a = x & 0x7fffu;
  return a > 0x7f80u ? 0u : (a == 0x7f80u ? (x & 0x8000u) | 0x7f7fu : x);
}
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, false);      // quad_perm [1,0,3,2]
  x = x > y ? x : y;
  const uint32_t z = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, false);      // quad_perm [2,3,0,1]
  return x > z ? x : z;
}

// Eight elements of a block (its other lanes hold the rest) -> eight codes, and the block's scale byte.
__device__ __forceinline__ uint32_t encode(u32x4 x, uint32_t& scale) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = held(x[i] & 0xffffu), hi = held(x[i] >> 16);
    x[i] = lo | (hi << 16);
    const uint32_t a = lo & 0x7fffu, b = hi & 0x7fffu;
    m = m > a ? m : a;
    m = m > b ? m : b;
  }
  m = quad_max(m);
  int e = (int)(m >> 7) - 2 + ((m & 0x7fu) > 0x60u ? 1 : 0);       // one more from 1.75 * 2^n (fraction 0x60 of 0x80) on
  e = e < 2 ? 2 : (e > 252 ? 252 : e);
  scale = (uint32_t)e;
  const float s = __uint_as_float((uint32_t)e << 23);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[0]), s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[1]), s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[2]), s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[3]), s, 3);
  return c;
}
__device__ __forceinline__ u32x4 decode(uint32_t c, uint32_t scale) {
  const float s = __uint_as_float(scale << 23);
  u32x4 x;
  x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
  x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
  x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
  x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
  return x;
}

// A row's place: offsets of its codes and scales, or not in the pool.
struct RowPlace {
  int64_t page;
  int row;
  bool held;
  __device__ __forceinline__ RowPlace(const CacheView& c, int slot, int head) {
    page = slot >> c.page_log2;
    held = slot >= 0 && page < c.n_pages;
    row = (head << c.page_log2) + (slot & ((1 << c.page_log2) - 1));
  }
};

}  // namespace
}  // namespace apbv
