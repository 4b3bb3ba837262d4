// Elements of tensors in 32 and 16 bits, four at a time, and sums over a wave,
// for the kernels that walk over tensors.
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

// Vectors at any element's address: the memory system takes accesses that are not
// aligned, and the compiler makes one of each (which it does not of a structure of
// elements).
typedef uint32_t u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_at2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));

// Four fp32 patterns to bf16, two a word: v_cvt_pk_bf16_f32 rounds every
// pattern as rne_bf16 does, NaNs included.
__device__ __forceinline__ u32x2 to_bf16(const f32x4& x) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(x.xy, bf16x2)),
               __builtin_bit_cast(uint32_t, __builtin_convertvector(x.zw, bf16x2))};
}

// Sums over a wave of eight 64-bit values at once.  Each of the first steps
// brings the lanes together in pairs that keep one half of the values each, so
// that they take 4 + 2 + 1 exchanges and the last three steps are of one value:
// 10 exchanges instead of 48.  Lane l ends with the total of value l / 8.
template <int kCtrl>
__device__ __forceinline__ u64 dpp64(u64 x) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0u, uint32_t(x), kCtrl, 0xF, 0xF, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0u, uint32_t(x >> 32), kCtrl, 0xF, 0xF, true);
  return u64(hi) << 32 | lo;
}
// The sums of a with the lanes 32 (or 16) apart in the lanes whose bit 5 (4) is
// clear, those of b in the others.
template <int kLanes>
__device__ __forceinline__ u64 halve(u64 a, u64 b) {
  const uint32_t al = uint32_t(a), ah = uint32_t(a >> 32), bl = uint32_t(b), bh = uint32_t(b >> 32);
  if constexpr (kLanes == 32) {
    const auto lo = __builtin_amdgcn_permlane32_swap(al, bl, false, false);
    const auto hi = __builtin_amdgcn_permlane32_swap(ah, bh, false, false);
    return (u64(hi[0]) << 32 | lo[0]) + (u64(hi[1]) << 32 | lo[1]);
  } else {
    const auto lo = __builtin_amdgcn_permlane16_swap(al, bl, false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap(ah, bh, false, false);
    return (u64(hi[0]) << 32 | lo[0]) + (u64(hi[1]) << 32 | lo[1]);
  }
}
__device__ __forceinline__ u64 wave_totals(u64 (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; i++) x[i] = halve<32>(x[i], x[i + 4]);
#pragma unroll
  for (int i = 0; i < 2; i++) x[i] = halve<16>(x[i], x[i + 2]);
  const bool upper = threadIdx.x & 8;
  const u64 keep = upper ? x[1] : x[0], send = upper ? x[0] : x[1];
  u64 t = keep + dpp64<0x128>(send);  // row_ror:8
  t += dpp64<0x141>(t);               // row_half_mirror
  t += dpp64<0x4E>(t);                // quad_perm: lanes 2 apart
  return t + dpp64<0xB1>(t);          // and neighbours
}

}  // namespace
}  // namespace fr
