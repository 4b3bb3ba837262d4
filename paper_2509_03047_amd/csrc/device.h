// Device helpers shared by the kernel sources.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace fr {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned long long u64;

__device__ __forceinline__ u32x4 ld_nt(const u32x4* p) { return __builtin_nontemporal_load(p); }
__device__ __forceinline__ void st_nt(u32x4 v, u32x4* p) { __builtin_nontemporal_store(v, p); }
__device__ __forceinline__ void st_nt2(u32x2 v, u32x2* p) { __builtin_nontemporal_store(v, p); }

// FRSUM-128 contribution of four consecutive words whose 0-based word index
// within the chunk starts at i0: sum += w, wsum += (index + 1) * w.
__device__ __forceinline__ void acc4(const u32x4& x, uint32_t i0, u64& s, u64& ws) {
  s += (u64)x.x + (u64)x.y + (u64)x.z + (u64)x.w;
  ws += (u64)(i0 + 1) * x.x + (u64)(i0 + 2) * x.y + (u64)(i0 + 3) * x.z + (u64)(i0 + 4) * x.w;
}

__device__ __forceinline__ void acc2(const u32x2& x, uint32_t i0, u64& s, u64& ws) {
  s += (u64)x.x + (u64)x.y;
  ws += (u64)(i0 + 1) * x.x + (u64)(i0 + 2) * x.y;
}

// fp32 bit pattern -> bf16 bit pattern, round to nearest, ties to even, in
// integer arithmetic (no flush of denormals): adding 0x7FFF plus the lowest
// kept bit carries into the kept half exactly when the dropped half is above
// the midpoint, or at it with an odd kept half.  NaN keeps its top bits with
// the quiet bit set.
__device__ __forceinline__ uint32_t rne_bf16(uint32_t u) {
  const uint32_t r = (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
  return ((u & 0x7FFFFFFFu) > 0x7F800000u) ? ((u >> 16) | 0x40u) : r;
}

}  // namespace
}  // namespace fr
