// Elements of tensors in 32 and 16 bits, four at a time, for the kernels that
// walk over them.
#pragma once

#include "device.h"

namespace fr {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float as_f(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t as_u(float f) { return __builtin_bit_cast(uint32_t, f); }

// Elements i ... i + 3 of the n > 0 at p, zeros behind them; kFull: all four are
// there.  Else each comes by a load of its own, from the last one's place where
// there is none: without branches all loads are in flight together.  (A load
// within a branch is waited for before the branch ends: a step of 20,000
// tensors of 1 to 4,096 elements took 81 us instead of 62.)
template <bool kFull>
__device__ __forceinline__ u32x4 load4(const void* p, uint32_t i, uint32_t n) {
  const uint32_t* q = static_cast<const uint32_t*>(p);
  if constexpr (kFull) return ld_nt(reinterpret_cast<const u32x4*>(q + i));
  u32x4 x;
#pragma unroll
  for (uint32_t j = 0; j < 4; j++) x[j] = q[i + j < n ? i + j : n - 1];
#pragma unroll
  for (uint32_t j = 0; j < 4; j++) x[j] = i + j < n ? x[j] : 0u;
  return x;
}
// The same of bf16 elements, in the first two words.
template <bool kFull>
__device__ __forceinline__ u32x4 load4h(const void* p, uint32_t i, uint32_t n) {
  const uint16_t* q = static_cast<const uint16_t*>(p);
  u32x4 x = {0, 0, 0, 0};
  if constexpr (kFull) {
    x.xy = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(q + i));
    return x;
  }
  uint32_t h[4];
#pragma unroll
  for (uint32_t j = 0; j < 4; j++) h[j] = q[i + j < n ? i + j : n - 1];
#pragma unroll
  for (uint32_t j = 0; j < 4; j++) h[j] = i + j < n ? h[j] : 0u;
  x.xy = u32x2{h[0] | h[1] << 16, h[2] | h[3] << 16};
  return x;
}
// Their fp32 patterns.
__device__ __forceinline__ u32x4 widen(const u32x4& x) {
  return u32x4{x.x << 16, x.x & 0xFFFF0000u, x.y << 16, x.y & 0xFFFF0000u};
}
template <bool kFull>
__device__ __forceinline__ void store4(void* p, u32x4 x, uint32_t i, uint32_t n) {
  uint32_t* q = static_cast<uint32_t*>(p) + i;
  if (kFull || i + 4 <= n) return st_nt(x, reinterpret_cast<u32x4*>(q));
  for (int j = 0; j < 4; j++)
    if (i + j < n) q[j] = x[j];
}
template <bool kFull>
__device__ __forceinline__ void store4h(void* p, u32x2 x, uint32_t i, uint32_t n) {
  uint16_t* q = static_cast<uint16_t*>(p) + i;
  if (kFull || i + 4 <= n) return st_nt2(x, reinterpret_cast<u32x2*>(q));
  for (int j = 0; j < 4; j++)
    if (i + j < n) q[j] = uint16_t(x[j / 2] >> (16 * (j & 1)));
}

// Four fp32 patterns to bf16, two a word: v_cvt_pk_bf16_f32 rounds every
// pattern as rne_bf16 does, NaNs included.
__device__ __forceinline__ u32x2 to_bf16(const f32x4& x) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(x.xy, bf16x2)),
               __builtin_bit_cast(uint32_t, __builtin_convertvector(x.zw, bf16x2))};
}

}  // namespace
}  // namespace fr
